"""Plain float64 statements of cache_append, tree_attention and logits_rules, node by node, and what a call may be off by.

Bounds, with u = 2^-24 (one rounding of fp32):
  append  the reduced angle is off by at most 2^-23 (half a step below pi), sine and cosine by 2 steps more, products and
          their sum by 3 roundings: 8 u (|x| + |y|) covers them; then the rounding of the result
  attend  a score is a sum of D products, added up in groups of 16 by the tensor cores, whose additions lose up to 2^-23 of
          the magnitude at each: (D/16 + 16) 2 u A, A = scale sum |q| |k| (fp32: one by one, (D + 8) u A), and a few u of
          its own magnitude from scale and base-2 exponent.  A weight is off by that relative to itself, as is the sum, and by
          4 u from the exponential; in bf16 calls a weight is cut to two bf16 numbers, 2^-17 of itself, or above 16 queries per
          cached head to one, 2^-8.  Sums over n keys add (n/16 + 64) 2 u (fp32: (n + 64) u).  All of these are relative to
          sum p |v|.  Then the rounding of the result.
  rules   five roundings of the terms' magnitudes, then the rounding of the result
"""
import math

import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def path(parents, i):
    """Node i and those before it on its path."""
    out = []
    while i >= 0:
        out.append(i)
        i = i - 1 if parents is None else int(parents[i])
    return out


def make_tree(B, T, g, roots=0.15):
    parents = torch.full((B, T), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(1, T):
            if torch.rand(1, generator=g) > roots:
                parents[b, i] = int(torch.randint(max(0, i - 5), i, (1,), generator=g))
    return parents


def make_pages(B, most, spare, g):
    n = B * most + spare
    return torch.randperm(n, generator=g)[:B * most].view(B, most).to(torch.int32), n


def used_nodes(lens, counts, b, T):
    if int(lens[b]) < 0:
        return 0
    return T if counts is None else min(max(int(counts[b]), 0), T)


def append(q, k, v, k_cache, v_cache, page_table, lens, inv_freq, interleaved, counts, parents, slots):
    """(q_out, k_cache, v_cache) in float64 and what they may be off by, from CPU tensors."""
    B, T, _, D = k.shape
    page = k_cache.shape[2]
    kc, vc = k_cache.double(), v_cache.double()
    k_tol, v_tol = torch.zeros_like(kc), torch.zeros_like(vc)
    qo = torch.zeros(q.shape, dtype=torch.float64) if q is not None else None
    q_tol = torch.zeros_like(qo) if q is not None else None
    r = 0 if inv_freq is None else inv_freq.numel()

    def turned(x, a):
        x, h = x.double(), half(x.dtype)
        y, tol = x.clone(), torch.zeros_like(x)
        if r:
            first = slice(0, 2 * r, 2) if interleaved else slice(0, r)
            second = slice(1, 2 * r, 2) if interleaved else slice(r, 2 * r)
            c, s = torch.cos(a), torch.sin(a)
            y[:, first] = x[:, first] * c - x[:, second] * s
            y[:, second] = x[:, second] * c + x[:, first] * s
            both = 8 * U * (x[:, first].abs() + x[:, second].abs())
            tol[:, first], tol[:, second] = both, both
            tol[:, :2 * r] += h * y[:, :2 * r].abs()
        return y, tol

    for b in range(B):
        par = None if parents is None else parents[b].tolist()
        for i in range(used_nodes(lens, counts, b, T)):
            depth = len(path(par, i)) - 1
            a = (int(lens[b]) + depth) * inv_freq.double() if r else None
            if q is not None:
                qo[b, i], q_tol[b, i] = turned(q[b, i], a)
            slot = int(lens[b]) + i if slots is None else int(slots[b, i])
            if slot < 0:
                continue
            at = int(page_table[b, slot // page])
            kc[at, :, slot % page], k_tol[at, :, slot % page] = turned(k[b, i], a)
            vc[at, :, slot % page] = v[b, i].double()
    return (qo, kc, vc), (q_tol, k_tol, v_tol)


def attend(q, k_cache, v_cache, page_table, lens, counts, parents, scale):
    """(out, what it may be off by) in float64; any device."""
    B, T, Hq, D = q.shape
    Hkv, page = k_cache.shape[1], k_cache.shape[2]
    G, dev = Hq // Hkv, q.device
    bf16 = q.dtype == torch.bfloat16
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    tol = torch.zeros_like(out)
    for b in range(B):
        n = used_nodes(lens, counts, b, T)
        if n == 0:
            continue
        length = int(lens[b])
        slot = torch.arange(length + n, device=dev)
        pages = page_table[b].to(dev).long()[slot // page]
        k, v = k_cache[pages, :, slot % page].double(), v_cache[pages, :, slot % page].double()   # [keys, Hkv, D]
        par = None if parents is None else parents[b].tolist()
        seen = torch.zeros((n, length + n), dtype=torch.bool)
        seen[:, :length] = True
        for i in range(n):
            seen[i, [length + j for j in path(par, i)]] = True
        seen = seen.to(dev)[None, None]                                       # [1, 1, n, keys]
        qq = q[b, :n].double().view(n, Hkv, G, D).permute(1, 2, 0, 3)         # [Hkv, G, n, D]
        k, v = k.permute(1, 0, 2)[:, None], v.permute(1, 0, 2)[:, None]       # [Hkv, 1, keys, D]
        k0 = torch.where(seen.any(2)[..., None], k, 0.0)                      # what nobody sees is not looked at
        v0 = torch.where(seen.any(2)[..., None], v, 0.0)
        s = scale * (qq @ k0.transpose(2, 3))
        s = s.masked_fill(~seen, -math.inf)
        p = torch.softmax(s, -1)
        # a value that a row does not see has no part in it, not even as 0 times infinity
        y, a = torch.zeros(Hkv, G, n, D, dtype=torch.float64, device=dev), torch.zeros(Hkv, G, n, D, dtype=torch.float64, device=dev)
        if bool(torch.isfinite(v0).all()):
            y, a = p @ v0, p @ v0.abs()
        else:
            for i in range(n):
                at = seen[0, 0, i].nonzero()[:, 0]
                y[:, :, i] = (p[:, :, i:i + 1, at] @ v0[:, :, at])[:, :, 0]
                a[:, :, i] = (p[:, :, i:i + 1, at] @ v0[:, :, at].abs())[:, :, 0]
        mag = abs(scale) * (qq.abs() @ k0.abs().transpose(2, 3))
        worst = mag.masked_fill(~seen, 0.0).amax(-1)
        d_score = worst * ((D / 16 + 16) * 2 * U if bf16 else (D + 8) * U) + 4 * U * s.masked_fill(~seen, 0.0).abs().amax(-1)
        keys = length + n
        cut = 2.0 ** -17 if T * G <= 16 else 2.0 ** -8
        rel = 2 * d_score + 8 * U + (cut + (keys / 16 + 64) * 2 * U if bf16 else (keys + 64) * U)
        out[b, :n] = y.permute(2, 0, 1, 3).reshape(n, Hq, D)
        tol[b, :n] = (a * rel[..., None] + half(q.dtype) * y.abs()).permute(2, 0, 1, 3).reshape(n, Hq, D)
    return out, tol + 1e-30


def rules(logits, V, history, history_len, tokens, parents, counts, penalties, bias_tokens, bias_values, masks, mask_rows):
    """(rows, what they may be off by) in float64, from CPU tensors; [B,T,V]."""
    B, T = logits.shape[:2]
    out = logits[..., :V].double().clone()
    tol = torch.zeros_like(out)
    for b in range(B):
        n = T if counts is None else min(max(int(counts[b]), 0), T)
        par = None if parents is None else parents[b].tolist()
        base = {}
        if penalties is not None and history is not None:
            for t in history[b, :max(int(history_len[b]), 0)].tolist():
                base[t] = base.get(t, 0) + 1
        for i in range(n):
            c = dict(base)
            if penalties is not None and tokens is not None:
                for j in path(par, i):
                    t = int(tokens[b, j])
                    c[t] = c.get(t, 0) + 1
            for t, times in c.items():
                if not 0 <= t < V:
                    continue
                r, f, s = penalties[b].double().tolist()
                x = float(out[b, i, t])
                out[b, i, t] = (x / r if x > 0 else x * r) - f * times - s
                tol[b, i, t] += 5 * U * (abs(x) * max(r, 1 / r) + abs(f * times) + abs(s))
            if bias_tokens is not None:
                for t, w in dict(zip(bias_tokens[b].tolist(), bias_values[b].tolist())).items():
                    if 0 <= t < V:
                        out[b, i, t] += w
                        tol[b, i, t] += 5 * U * (abs(w) + abs(float(out[b, i, t])))
            changed = tol[b, i] > 0
            tol[b, i] += torch.where(changed, half(logits.dtype) * out[b, i].abs(), 0.0)
            if masks is not None and 0 <= int(mask_rows[b, i]) < masks.shape[0]:
                words = masks[int(mask_rows[b, i])].long()
                v = torch.arange(V)
                out[b, i][((words[v // 32] >> (v % 32)) & 1) == 0] = -math.inf
    return out, tol


def within(got, want, tol):
    """Whether every entry is within its bound: infinities and NaN stand where they should."""
    got, want = got.double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    ok = same | ((got - want).abs() <= tol)
    return bool(ok.all())


def worst(got, want, tol):
    d = (got.double() - want.double()).abs() / tol.clamp(min=1e-300)
    return float(torch.where(want.isfinite(), d, 0.0).max())
