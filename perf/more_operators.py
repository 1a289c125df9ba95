"""Cases and plain forms of the operators around the target model's pass over drafted tokens.

  append  cache_append     rotates the drafted tokens' queries and keys by their positions and puts keys
                           and values into a paged cache (or a prompt's, many at once)
  attend  tree_attention   attention of the drafted tokens, a chain or a tree, over that cache
  rules   logits_rules     penalties for repeated tokens, biases and grammar masks on the rows of logits that
                           sd_verify and replace_sample read

B sequences have T nodes each: the tokens that one pass works on.  parents [B,T] gives each node's parent
(-1: the cached prefix), no parents mean a chain, counts [B] says how many of the T a sequence uses.  Node i of
sequence b lies in the cache's slot lens[b] + i, at position lens[b] + depth, and sees the prefix and its path.
Caches are [pages, kv heads, page size, D]; slot s of sequence b is entry s % page size of page
page_table[b, s / page size].
"""
import math

import torch

own = False

THETA = 10000.0         # base of the rotation's frequencies
NONE = -1


def listed():
    return [
        # one new token of one sequence, fp32: the call's latency
        dict(name="append 1x1 4/4x64 f32", op="append", dt="f32", B=1, T=1, Hq=4, Hkv=4, D=64, L=100, page=16, tree=False,
             rot=64, interleaved=False, fused=False),
        # a verification pass: 256 sequences, 16 draft tokens and the last one before them
        dict(name="append 256x17 32/8x128", op="append", dt="bf16", B=256, T=17, Hq=32, Hkv=8, D=128, L=2048, page=16, tree=False,
             rot=128, interleaved=False, fused=True),
        # prompts of four sequences
        dict(name="append 4x8000 32/8x128", op="append", dt="bf16", B=4, T=8000, Hq=32, Hkv=8, D=128, L=200, page=64, tree=False,
             rot=128, interleaved=True, fused=True),
        # four draft tokens of one sequence, fp32: the call's latency
        dict(name="attend 1x4 4/2x64 f32", op="attend", dt="f32", B=1, T=4, Hq=4, Hkv=2, D=64, L=300, page=16, tree=False),
        # single tokens: ordinary decoding of a batch
        dict(name="attend 64x1 32/8x128", op="attend", dt="bf16", B=64, T=1, Hq=32, Hkv=8, D=128, L=4096, page=16, tree=False),
        # eight draft tokens under heads of their own (d = 768)
        dict(name="attend 32x9 12/12x64", op="attend", dt="bf16", B=32, T=9, Hq=12, Hkv=12, D=64, L=1000, page=16, tree=False),
        # 16 draft tokens
        dict(name="attend 128x17 32/8x128", op="attend", dt="bf16", B=128, T=17, Hq=32, Hkv=8, D=128, L=2048, page=32, tree=False),
        # trees of 64 drafted tokens
        dict(name="attend 16x64 tree 32/8x128", op="attend", dt="bf16", B=16, T=64, Hq=32, Hkv=8, D=128, L=8192, page=64, tree=True),
        # one sequence with a long prefix: the prefix is what there is to split
        dict(name="attend 1x8 131072 32/8x128", op="attend", dt="bf16", B=1, T=8, Hq=32, Hkv=8, D=128, L=131072, page=16, tree=True),
        # the rows of one sequence's four draft tokens, fp32: the call's latency
        dict(name="rules 1x4x1000 f32", op="rules", dt="f32", B=1, T=4, V=1000, L=50, tree=False, bias=4, masked=0.0),
        # rows of odd length, half of the sequences under a grammar
        dict(name="rules 32x9x50257", op="rules", dt="bf16", B=32, T=9, V=50257, L=1000, tree=False, bias=16, masked=0.5),
        # rows for the exact check of 16 draft tokens and the row behind them
        dict(name="rules 256x17x128256", op="rules", dt="bf16", B=256, T=17, V=128256, L=2048, tree=False, bias=32, masked=0.25),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend", "rules"])
    dt = rng.choice(["bf16", "bf16", "f32"])
    if op == "rules":
        while True:
            B, T, V = size(1, 256), size(1, 64), size(500, 128256)
            if B * T * V <= 256 * 17 * 128256 // (1 if dt == "bf16" else 2):
                break
        return dict(op=op, dt=dt, B=B, T=T, V=V, L=size(1, 8192), tree=rng.random() < 0.4, bias=rng.choice([0, 1, 7, 64, 300]),
                    masked=rng.choice([0.0, 0.3, 1.0]))
    Hkv, G, page = rng.choice([1, 2, 3, 4, 8, 12, 16]), rng.choice([1, 1, 2, 3, 4, 5, 8]), rng.choice([8, 16, 24, 32, 64, 128])
    D, tree = rng.choice([64, 64, 80, 96, 128, 128]), rng.random() < 0.5
    if op == "append":
        while True:
            B, T = size(1, 256), size(1, 64 if tree else 8192)
            if B * T * (G + 2) * Hkv * D <= 4 * 8000 * 48 * 128 // (1 if dt == "bf16" else 2):
                break
        return dict(op=op, dt=dt, B=B, T=T, Hq=G * Hkv, Hkv=Hkv, D=D, L=size(1, 2048), page=page, tree=tree,
                    rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.5, fused=rng.random() < 0.5)
    while True:
        B, T, L = size(1, 128), size(1, 64), size(1, 131072)
        flops, kv = 4 * B * T * G * Hkv * D * (L + T), 2 * B * Hkv * D * (L + T)
        if kv <= 2 * 8 * 128 * 131072 // (1 if dt == "bf16" else 2) and flops <= 4 * 16 * 64 * 32 * 128 * 8192 // (1 if dt == "bf16" else 16):
            break
    return dict(op=op, dt=dt, B=B, T=T, Hq=G * Hkv, Hkv=Hkv, D=D, L=L, page=page, tree=tree)


def _type(case):
    return torch.float32 if case["dt"] == "f32" else torch.bfloat16


def _ragged(B, most, g):
    """Lengths of up to `most`, the first as long as that: prefixes of sequences that came at different times."""
    n = (torch.rand(B, generator=g, device="cuda") * 0.5 + 0.5) * most
    n[0] = most
    return n.round().to(torch.int32)


def _tree(case, g):
    """parents [B,T] and counts [B], or two times None for a chain."""
    B, T = case["B"], case["T"]
    if not case["tree"]:
        return None, None
    i = torch.arange(T, device="cuda")
    # a node's parent is one of the few before it: trees some T / 3 deep with a few branches
    back = 1 + (torch.rand(B, T, generator=g, device="cuda") ** 2 * 5).long()
    parents = torch.where(i >= back, i - back, NONE).to(torch.int32)
    counts = (T - (torch.rand(B, generator=g, device="cuda") * 0.25 * T).long()).clamp(min=1).to(torch.int32)
    return parents, counts


def _pages(case, g, lens):
    """page_table [B, pages a sequence may have]: pages in the order in which a pool hands them out."""
    B, page = case["B"], case["page"]
    most = (case["L"] + case["T"] + page - 1) // page
    return torch.randperm(B * most + 3, generator=g, device="cuda")[:B * most].view(B, most).to(torch.int32), B * most + 3


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    ty, op, B, T = _type(case), case["op"], case["B"], case["T"]
    s = {"case": dict(case), "ws": None}
    s["parents"], s["counts"] = _tree(case, g)
    if op == "rules":
        V, L = case["V"], case["L"]
        s["logits"] = (randn(B, T, V) * 3.0).to(ty)
        # tokens repeat as they do in text: rank r about as often as 1 / r
        rank = torch.exp(torch.rand(B, L + T, generator=g, device="cuda") * math.log(V)).long().clamp(max=V) - 1
        text = (rank * 7919 + 13) % V
        s["history"], s["tokens"] = text[:, :L].to(torch.int32).contiguous(), text[:, L:].to(torch.int32).contiguous()
        s["history_len"] = _ragged(B, L, g)
        u = torch.rand(B, 3, generator=g, device="cuda")
        s["penalties"] = torch.stack([1.0 + 0.3 * u[:, 0], 0.5 * u[:, 1], 0.5 * u[:, 2]], 1).contiguous()
        s["bias_tokens"] = s["bias_values"] = s["masks"] = s["mask_rows"] = None
        if case["bias"]:
            s["bias_tokens"] = torch.randint(0, V, (B, case["bias"]), generator=g, device="cuda", dtype=torch.int32)
            s["bias_values"] = randn(B, case["bias"]) * 4.0
        if case["masked"]:
            n = 32              # states of the grammars in use; some allow a handful of tokens, some nearly all
            keep = torch.rand(n, (V + 31) // 32 * 32, generator=g, device="cuda") < torch.rand(n, 1, generator=g, device="cuda")
            bits = keep.view(n, -1, 32).long() << torch.arange(32, device="cuda")
            s["masks"] = bits.sum(-1).to(torch.int32)
            some = torch.rand(B, 1, generator=g, device="cuda") < case["masked"]
            s["mask_rows"] = torch.where(some, torch.randint(0, n, (B, T), generator=g, device="cuda"), NONE).to(torch.int32)
        s["out"] = torch.empty_like(s["logits"])
        return s
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    s["lens"] = _ragged(B, case["L"], g)
    s["page_table"], pages = _pages(case, g, s["lens"])
    if op == "append":
        s["k_cache"], s["v_cache"] = randn(pages, Hkv, page, D, dtype=ty), randn(pages, Hkv, page, D, dtype=ty)
        if case["fused"]:       # one projection gives all three, side by side
            x = randn(B, T, Hq + 2 * Hkv, D).to(ty)
            s["q"], s["k"], s["v"] = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
        else:
            s["q"], s["k"], s["v"] = randn(B, T, Hq, D).to(ty), randn(B, T, Hkv, D).to(ty), randn(B, T, Hkv, D).to(ty)
        r = case["rot"] // 2
        s["inv_freq"] = (THETA ** (-torch.arange(r, device="cuda", dtype=torch.float64) / r)).float()
        s["q_out"] = torch.empty(B, T, Hq, D, device="cuda", dtype=ty)
        return s
    # scores N(0, 1.5^2): some keys count for much, most for little
    s["q"] = (randn(B, T, Hq, D) * 1.5).to(ty)
    s["k_cache"] = randn(pages, Hkv, page, D, dtype=ty)
    s["v_cache"] = randn(pages, Hkv, page, D, dtype=ty)
    s["out"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------------------- plain forms


def _paths(s, B, T):
    """[B,T,T] of 0 and 1: whether node j is node i or before it on its path.  (I - P)^-1 = I + P + P^2 + ..."""
    one = torch.eye(T, device="cuda").expand(B, T, T)
    if s["parents"] is None:
        return torch.ones(T, T, device="cuda").tril().expand(B, T, T)
    P = (s["parents"][:, :, None] == torch.arange(T, device="cuda", dtype=torch.int32)).float()
    return torch.linalg.solve_triangular(one - P, one, upper=False, unitriangular=True)


def _used(s, B, T):
    if s["counts"] is None:
        return torch.ones(B, T, dtype=torch.bool, device="cuda")
    return torch.arange(T, device="cuda") < s["counts"][:, None]


def _rotated(x, c, n, interleaved):
    """x [B,T,H,D] with its first 2 n elements rotated; c = cos and sin [B,T,1,n]."""
    x = x.float()
    if interleaved:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack([a * c[0] - b * c[1], b * c[0] + a * c[1]], -1).flatten(-2)
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        turned = torch.cat([a * c[0] - b * c[1], b * c[0] + a * c[1]], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_append(s):
    case = s["case"]
    B, T, page, n = case["B"], case["T"], case["page"], case["rot"] // 2
    used = _used(s, B, T)
    i = torch.arange(T, device="cuda").expand(B, T)
    depth = i if s["parents"] is None else _paths(s, B, T).sum(-1).long() - 1
    angle = (s["lens"][:, None] + depth).double()[..., None, None] * s["inv_freq"].double()
    c = (torch.cos(angle).float(), torch.sin(angle).float())
    q = torch.where(used[..., None, None], _rotated(s["q"], c, n, case["interleaved"]), 0.0)
    s["q_out"].copy_(q)
    slot = s["lens"][:, None].long() + i
    at = s["page_table"].gather(1, slot // page).long() * page + slot % page
    at, k = at[used], _rotated(s["k"], c, n, case["interleaved"])[used]
    s["k_cache"][at // page, :, at % page] = k.to(s["k_cache"].dtype)
    s["v_cache"][at // page, :, at % page] = s["v"][used]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_attend(s):
    case = s["case"]
    B, T, Hq, Hkv, D = case["B"], case["T"], case["Hq"], case["Hkv"], case["D"]
    keys = s["page_table"].shape[1] * case["page"]
    used, lens = _used(s, B, T), s["lens"].long()[:, None, None]
    j = torch.arange(keys, device="cuda")
    seen = (j < lens).expand(B, T, keys)
    nodes = torch.nn.functional.pad(_paths(s, B, T), (0, 1)) > 0
    at = (j - lens).clamp(min=-1, max=T).expand(B, T, keys)
    seen = torch.where(at >= 0, nodes.gather(2, at.clamp(min=0)), seen) & used[..., None]

    def laid_out(cache):        # [B,Hkv,keys,D]
        return cache[s["page_table"].long()].transpose(1, 2).reshape(B, Hkv, keys, D).float()

    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    score = ((q @ laid_out(s["k_cache"]).transpose(2, 3)) / math.sqrt(D)).view(B, Hkv, T, -1, keys)
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p.view(B, Hkv, -1, keys) @ laid_out(s["v_cache"])).view(B, Hkv, T, -1, D) / total.clamp(min=1e-30)
    return out.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(s["q"].dtype)


def _plain_rules(s):
    case = s["case"]
    B, T, V, L = case["B"], case["T"], case["V"], case["L"]
    x = s["logits"].float()
    known = (torch.arange(L, device="cuda") < s["history_len"][:, None]).float()
    base = torch.zeros(B, V, device="cuda").scatter_add_(1, s["history"].long(), known)
    paths = _paths(s, B, T)
    count = base[:, None].repeat(1, T, 1).scatter_add_(2, s["tokens"].long()[:, None].expand(B, T, T), paths)
    repeat, often, there = (s["penalties"][:, k, None, None] for k in range(3))
    y = torch.where(x > 0, x / repeat, x * repeat) - often * count - there
    y = torch.where(count > 0, y, x)
    if s["bias_tokens"] is not None:
        t, n = s["bias_tokens"], case["bias"]
        again = (t[:, :, None] == t[:, None]) & torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        bias = torch.zeros(B, V, device="cuda").scatter_add_(1, t.long(), torch.where(again.any(-1), 0.0, s["bias_values"]))
        y = y + bias[:, None]
    if s["masks"] is not None:
        rows = s["mask_rows"].long()
        bit = torch.arange(32, device="cuda", dtype=torch.int32)
        allowed = ((s["masks"][..., None] >> bit) & 1).view(s["masks"].shape[0], -1)[:, :V].bool()
        y = y.masked_fill(~(allowed[rows.clamp(min=0)] | (rows < 0)[..., None]), -math.inf)
    y = torch.where(_used(s, B, T)[..., None], y, x)
    s["out"].copy_(y)
    return s["out"]


def _plain(s):
    return {"append": _plain_append, "attend": _plain_attend, "rules": _plain_rules}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------- the library's calls


def _workspace(s):
    """The workspace that a program keeps beside its weights, made at the state's first pass."""
    import paper_2502_04557_b200 as spr
    if s["ws"] is None:
        c = s["case"]
        op = {"append": spr.OP_CACHE_APPEND, "attend": spr.OP_TREE_ATTENTION, "rules": spr.OP_LOGITS_RULES}[c["op"]]
        s["ws"] = spr.Workspace(spr.workspace_bytes(op, c["B"], c["T"], c.get("V", 1), c.get("D", 1), c.get("Hq", 0),
                                                    spr.F32 if c["dt"] == "f32" else spr.BF16))
    return s["ws"]


def _own(s):
    import paper_2502_04557_b200 as spr
    case, ws = s["case"], _workspace(s)
    if case["op"] == "append":
        spr.cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"], s["lens"], ws, q=s["q"],
                         inv_freq=s["inv_freq"], interleaved=case["interleaved"], counts=s["counts"], parents=s["parents"],
                         q_out=s["q_out"])
        return s["q_out"], s["k_cache"], s["v_cache"]
    if case["op"] == "attend":
        return spr.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lens"], ws, counts=s["counts"],
                                  parents=s["parents"], out=s["out"])
    return spr.logits_rules(s["logits"], case["V"], ws, history=s["history"], history_len=s["history_len"], tokens=s["tokens"],
                            parents=s["parents"], counts=s["counts"], penalties=s["penalties"], bias_tokens=s["bias_tokens"],
                            bias_values=s["bias_values"], masks=s["masks"], mask_rows=s["mask_rows"], out=s["out"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Ragged batches are three quarters as long as their longest on average, trees use seven eighths of their nodes."""
    es, B, T = 4 if case["dt"] == "f32" else 2, case["B"], case["T"]
    nodes = B * T * (0.875 if case["tree"] else 1.0)
    if case["op"] == "rules":
        V = case["V"]
        return {"bytes": 2 * es * B * T * V + 4 * B * (0.75 * case["L"] + 2 * T + 2 * case["bias"]) + case["masked"] * min(32, B * T) * V / 8,
                "flops": B * T * V}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "append":
        return {"bytes": 2 * es * nodes * (Hq + 2 * Hkv) * D + 8 * nodes, "flops": 6 * nodes * (Hq + Hkv) * case["rot"] / 2}
    prefix = case["L"] * (0.75 if B > 1 else 1.0)
    return {"bytes": 2 * es * (B * prefix + nodes) * Hkv * D + 2 * es * nodes * Hq * D,
            "flops": 4 * nodes * Hq * D * (prefix + T / 2)}


# ---------------------------------------------------------------------------- 64 bits, from the definitions


def _path_list(parents, i):
    """Node i and the nodes before it on its path, the last first."""
    path = [i]
    while (parents[path[-1]] if parents is not None else path[-1] - 1) >= 0:
        path.append(parents[path[-1]] if parents is not None else path[-1] - 1)
    return path


def exact(case, seed):
    s, f64 = prepare(case, seed), torch.float64
    B, T, op = case["B"], case["T"], case["op"]
    counts = [T] * B if s["counts"] is None else s["counts"].tolist()
    parents = [None] * B if s["parents"] is None else s["parents"].tolist()
    if op == "rules":
        V, out = case["V"], s["logits"].to(f64)
        for b in range(B):
            seen = torch.bincount(s["history"][b, :int(s["history_len"][b])].long(), minlength=V).to(f64)
            repeat, often, there = s["penalties"][b].to(f64)
            bias = torch.zeros(V, dtype=f64, device="cuda")
            if case["bias"]:
                last = dict(zip(s["bias_tokens"][b].tolist(), s["bias_values"][b].tolist()))
                bias[list(last)] = torch.tensor(list(last.values()), dtype=f64, device="cuda")
            for i in range(counts[b]):
                c = seen + torch.bincount(s["tokens"][b, _path_list(parents[b], i)].long(), minlength=V)
                x = out[b, i]
                y = torch.where(x > 0, x / repeat, x * repeat) - often * c - there
                x = torch.where(c > 0, y, x) + bias
                if case["masked"] and int(s["mask_rows"][b, i]) >= 0:
                    words = s["masks"][int(s["mask_rows"][b, i])].long()
                    v = torch.arange(V, device="cuda")
                    x[((words[v // 32] >> (v % 32)) & 1) == 0] = -math.inf
                out[b, i] = x
        return out
    lens, table, page, D = s["lens"].tolist(), s["page_table"].long(), case["page"], case["D"]
    if op == "append":
        r = case["rot"]
        first, second = (torch.arange(0, r, 2), torch.arange(1, r, 2)) if case["interleaved"] else (torch.arange(r // 2), torch.arange(r // 2, r))
        first, second = first.cuda(), second.cuda()
        k_cache, v_cache = s["k_cache"].to(f64), s["v_cache"].to(f64)
        q_out = torch.zeros(B, T, case["Hq"], D, dtype=f64, device="cuda")
        for b in range(B):
            n = counts[b]
            depth = torch.arange(n) if parents[b] is None else torch.tensor([len(_path_list(parents[b], i)) - 1 for i in range(n)])
            turn = torch.polar(torch.ones((), dtype=f64, device="cuda"), (lens[b] + depth).cuda().to(f64)[:, None] * s["inv_freq"].to(f64))
            slot = lens[b] + torch.arange(n, device="cuda")
            where, within = table[b, slot // page], slot % page
            for x, take in ((s["q"], True), (s["k"], False)):
                x = x[b, :n].to(f64)
                z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
                x[..., first], x[..., second] = z.real, z.imag
                if take:
                    q_out[b, :n] = x
                else:
                    k_cache[where, :, within] = x
            v_cache[where, :, within] = s["v"][b, :n].to(f64)
        return q_out, k_cache, v_cache
    Hq, Hkv = case["Hq"], case["Hkv"]
    if B * counts[0] * Hq * (case["L"] + T) > 1 << 32:
        return None
    out = torch.zeros(B, T, Hq, D, dtype=f64, device="cuda")
    for b in range(B):
        n, l = counts[b], lens[b]
        slot = torch.arange(l + n, device="cuda")
        k, v = (s[c][table[b, slot // page], :, slot % page].to(f64) for c in ("k_cache", "v_cache"))
        hidden = torch.ones(n, n, dtype=torch.bool)
        for i in range(n):
            hidden[i, _path_list(parents[b], i)] = False
        hidden = torch.cat([torch.zeros(n, l, dtype=torch.bool), hidden], 1).cuda()
        for h in range(Hq):
            a = (s["q"][b, :n, h].to(f64) @ k[:, h * Hkv // Hq].T) * D ** -0.5
            out[b, :n, h] = torch.softmax(a.masked_fill(hidden, -math.inf), -1) @ v[:, h * Hkv // Hq]
    return out
