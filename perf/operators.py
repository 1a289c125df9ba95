"""Cases and plain forms of the operators that fit a draft model's head and the verifier.

  loss    head_loss            softmax cross entropy of hidden states under a vocabulary head
                               (logits = hidden W^T are never kept): loss and log-sum-exp per token
  grad    head_loss_grad       its gradient with respect to hidden states and head
  labels  verifier_labels_head training labels 1[q(x)/p(x) <= lambda] of the verifier from the
                               hidden states and heads of both models
  pack    hidden_pack8 / hidden_unpack8   hidden states kept in 8 bits and read back
  step    verifier_train_step8 one Adam step of the verifier on hidden states kept in 8 bits

Packed hidden states: a row of d elements is d signed bytes q followed by ceil(d / 32) signed
bytes e (one for each block of 32 elements), padded with zeros to a multiple of 16 bytes; an
element stands for q * 2^e, e = max(floor(log2 of the block's largest magnitude) - 6, -126),
q = clamp(round-to-even(x * 2^-e), -127, 127).
"""
import math

import torch

own = False

BLOCK = 32              # elements that share an exponent
LAMBDAS = (1.0, 1.2, 1.5)
LR, BETA1, BETA2, EPS, STEP = 1e-3, 0.9, 0.999, 1e-8, 100


def listed():
    return [
        # one sequence of four draft tokens, fp32: the call's latency
        dict(name="loss tiny f32", op="loss", dt="f32", N=4, d=256, V=1000, ignore=False),
        # a decode batch's tokens (32 x 8) under a 50257-entry head
        dict(name="loss 256x768x50257", op="loss", dt="bf16", N=256, d=768, V=50257, ignore=True),
        # a training batch under a 128256-entry head
        dict(name="loss 4096x2048x128256", op="loss", dt="bf16", N=4096, d=2048, V=128256, ignore=True),
        # fp32 with odd sizes everywhere
        dict(name="grad 67x257x1003 f32", op="grad", dt="f32", N=67, d=257, V=1003, ignore=True),
        # a small batch: the head's gradient (77 MB written) counts as much as the products
        dict(name="grad 256x768x50257", op="grad", dt="bf16", N=256, d=768, V=50257, ignore=True),
        # an ordinary batch (128 x 8)
        dict(name="grad 1024x2048x32000", op="grad", dt="bf16", N=1024, d=2048, V=32000, ignore=True),
        # a training batch: the vocabulary goes by in pieces
        dict(name="grad 4096x2048x128256", op="grad", dt="bf16", N=4096, d=2048, V=128256, ignore=True),
        # labels for a decode batch, target twice as wide as the draft
        dict(name="labels 256 768+1536 50257", op="labels", dt="bf16", N=256, dq=768, dp=1536, V=50257),
        # labels for a batch of 128 x 8 draft tokens
        dict(name="labels 1024 2048+4096 32000", op="labels", dt="bf16", N=1024, dq=2048, dp=4096, V=32000),
        # one batch's hidden states go into the training set and come back
        dict(name="pack 4096x2048", op="pack", dt="bf16", N=4096, d=2048),
        # a small fitting batch of narrow states
        dict(name="step 4096x768", op="step", dt="bf16", N=4096, d=768),
        # a whole training set of 2^18 samples in one step
        dict(name="step 262144x2048", op="step", dt="bf16", N=262144, d=2048),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["loss", "grad", "labels", "pack", "step"])
    dt = rng.choice(["bf16", "bf16", "f32"])
    if op == "pack":
        return dict(op=op, dt=dt, N=size(1, 16384), d=size(1, 4096))
    if op == "step":
        return dict(op=op, dt=dt, N=size(1, 200000), d=16 * size(1, 128))
    while True:
        N, d, V = size(1, 4096), size(32, 4096), size(1000, 128256)
        if rng.random() < 0.6:
            d = (d + 63) // 64 * 64
        if N * d * V <= (1024 * 2048 * 128256 if dt == "f32" else 4096 * 2048 * 128256) / (1 if op != "labels" else 4):
            break
    if op == "labels":
        return dict(op=op, dt=dt, N=N, dq=d, dp=d + rng.choice([0, d, size(1, 512)]), V=V)
    return dict(op=op, dt=dt, N=N, d=d, V=V, ignore=rng.random() < 0.5)


def _type(case):
    return torch.float32 if case["dt"] == "f32" else torch.bfloat16


def _tokens(logits, g):
    """Tokens distributed as softmax(logits)."""
    u = torch.rand(logits.shape, generator=g, device="cuda").clamp_(1e-20, 1.0 - 1e-7)
    return (logits - torch.log(-torch.log(u))).argmax(-1).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    ty, op, N = _type(case), case["op"], case["N"]
    s = {"op": op}
    if op in ("loss", "grad"):
        d, V = case["d"], case["V"]
        s["hidden"] = randn(N, d).to(ty)
        s["W"] = (randn(V, d) * (3.0 / math.sqrt(d))).to(ty)            # logits N(0, 3^2)
        logits = s["hidden"].float() @ s["W"].float().T
        s["targets"] = _tokens(logits, g)
        if case["ignore"]:                                               # padding of ragged sequences
            s["targets"] = torch.where(torch.rand(N, generator=g, device="cuda") < 0.125,
                                       torch.full_like(s["targets"], -1), s["targets"])
        if op == "grad":
            s["lse"] = torch.logsumexp(logits, -1)
            s["grad_loss"] = torch.full((N,), 1.0 / N, device="cuda") * (0.5 + torch.rand(N, generator=g, device="cuda"))
    elif op == "labels":
        dq, dp, V = case["dq"], case["dp"], case["V"]
        hq, wq = randn(N, dq), randn(V, dq) * (3.0 / math.sqrt(dq))      # draft logits N(0, 3^2)
        hp = torch.cat([hq, randn(N, dp - dq)], 1)
        wp = randn(V, dp) * (3.0 * math.sqrt(0.19 / dp))                 # target logits correlate 0.9 with them
        wp[:, :dq] += 0.9 * wq
        s.update(p_hidden=hp.to(ty), p_W=wp.to(ty), q_hidden=hq.to(ty), q_W=wq.to(ty))
        lq = s["q_hidden"].float() @ s["q_W"].float().T
        s["tokens"] = _tokens(lq, g)
        at = s["tokens"].long()[:, None]
        log_q = lq.gather(1, at)[:, 0] - torch.logsumexp(lq, -1)
        lp = s["p_hidden"].float() @ s["p_W"].float().T
        ratio = (log_q - lp.gather(1, at)[:, 0] + torch.logsumexp(lp, -1)).exp()
        # each threshold in the middle of the widest gap of the ratios within 1 % of it
        s["lambdas"] = [_clear_of(ratio, lam) for lam in LAMBDAS]
    elif op == "pack":
        s["hidden"] = (randn(N, case["d"]) * randn(N, 1).exp()).to(ty)
    else:
        d = case["d"]
        # hidden states whose packed form depends on the type they came in
        hidden = randn(N, d).to(ty)
        teacher = randn(d) / math.sqrt(d)
        s["labels"] = (hidden.float() @ teacher + 0.5 * randn(N) > 0.1).to(torch.uint8)
        s["packed"], s["d"] = _pack(hidden), d
        s["theta"] = randn(d + 1) / math.sqrt(d)                         # a fit in progress: step 100
        s["m"], s["v"] = randn(d + 1) * 1e-3, torch.rand(d + 1, generator=g, device="cuda") * 1e-6 + 1e-7
    if op in ("loss", "grad", "labels", "step"):
        s["ws"] = torch.empty(0, device="cuda")
        s["case"] = dict(case)
    return s


def _clear_of(ratio, lam):
    near = ratio[(ratio > 0.99 * lam) & (ratio < 1.01 * lam)].sort().values.double()
    edge = torch.cat([near.new_tensor([0.99 * lam]), near, near.new_tensor([1.01 * lam])])
    k = int((edge[1:] - edge[:-1]).argmax())
    return float(torch.tensor(float(0.5 * (edge[k] + edge[k + 1])), dtype=torch.float32))


# ---------------------------------------------------------------------------- plain forms


def _pow2(e):
    """2^e for int32 -126 <= e <= 127, exactly: the exponent field of a float."""
    return ((e + 127) << 23).view(torch.float32)


def _pack(x):
    N, d = x.shape
    nb = (d + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - d)).view(N, nb, BLOCK)
    e = (torch.frexp(x.abs().amax(-1)).exponent - 7).clamp(min=-126)
    e = torch.where((x == 0).all(-1), torch.full_like(e, -126), e)
    q = (x * _pow2(-e)[..., None]).round().clamp(-127, 127)
    row = torch.cat([q.view(N, nb * BLOCK)[:, :d].to(torch.int8), e.to(torch.int8)], 1)
    return torch.nn.functional.pad(row, (0, -(d + nb) % 16)).view(torch.uint8)


def _unpack(packed, d):
    N, nb = packed.shape[0], (d + BLOCK - 1) // BLOCK
    row = packed.view(torch.int8)
    q = torch.nn.functional.pad(row[:, :d].float(), (0, nb * BLOCK - d)).view(N, nb, BLOCK)
    e = row[:, d:d + nb].to(torch.int32)[..., None]
    return (q * _pow2(e)).view(N, nb * BLOCK)[:, :d]


def _log_prob(hidden, W, tokens):
    lse = torch.logsumexp(hidden.float() @ W.float().T, -1)
    at = (hidden.double() * W[tokens.long().clamp(min=0)].double()).sum(-1)     # a ratio e^(a - b) shows every bit
    return at - lse.double(), lse


def _plain(s):
    op = s["op"]
    if op == "loss":
        log_prob, lse = _log_prob(s["hidden"], s["W"], s["targets"])
        return torch.where(s["targets"] >= 0, -log_prob.float(), torch.zeros_like(lse)), lse
    if op == "grad":
        keep = (s["targets"] >= 0)[:, None]
        H, W = torch.where(keep, s["hidden"].float(), 0.0), s["W"].float()
        P = torch.exp(H @ W.T - s["lse"][:, None])
        at = s["targets"].long().clamp(min=0)[:, None]
        P.scatter_add_(1, at, torch.full_like(P[:, :1], -1.0))
        P = torch.where(keep, P * s["grad_loss"][:, None], 0.0)
        return (P @ W).to(s["hidden"].dtype), (P.T @ H).to(s["W"].dtype)
    if op == "labels":
        log_p, _ = _log_prob(s["p_hidden"], s["p_W"], s["tokens"])
        log_q, _ = _log_prob(s["q_hidden"], s["q_W"], s["tokens"])
        ratio = torch.exp(log_q - log_p)
        lam = torch.tensor(s["lambdas"], dtype=torch.float64).to(ratio.device)
        return (ratio[None, :] <= lam[:, None]).to(torch.uint8), ratio.float()
    if op == "pack":
        return _unpack(_pack(s["hidden"]), s["hidden"].shape[1]).to(s["hidden"].dtype)
    S, w, y = _unpack(s["packed"], s["d"]), s["theta"], s["labels"].float()
    z = (S @ w[:-1] + w[-1]).double()
    loss = (torch.nn.functional.relu(z) + torch.log1p(torch.exp(-z.abs())) - y * z).mean()
    r = torch.sigmoid(z) - y
    grad = torch.cat([(r.float() @ S).double(), r.sum()[None]]) / S.shape[0]
    m = BETA1 * s["m"].double() + (1 - BETA1) * grad
    v = BETA2 * s["v"].double() + (1 - BETA2) * grad * grad
    step = LR * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
    s["theta"].copy_(w.double() - step)
    s["m"].copy_(m)
    s["v"].copy_(v)
    return loss.float()[None], s["theta"], s["m"], s["v"]


# ---------------------------------------------------------------------------- the library's calls


def _workspace(s):
    """The workspace that a program keeps beside its weights, made at the state's first pass."""
    import paper_2502_04557_b200 as spr
    if not isinstance(s["ws"], spr.Workspace):
        c = s["case"]
        code = spr.F32 if c["dt"] == "f32" else spr.BF16
        op = {"loss": spr.OP_HEAD_LOSS, "grad": spr.OP_HEAD_LOSS_GRAD, "labels": spr.OP_VERIFIER_LABELS_HEAD,
              "step": spr.OP_VERIFIER_TRAIN8}[c["op"]]
        n = spr.workspace_bytes(op, c["N"], 1, c.get("V", 1), c.get("d", c.get("dp")), c.get("dq", 0), code)
        s["ws"] = spr.Workspace(n)
    return s["ws"]


def _own(s):
    import paper_2502_04557_b200 as spr
    op = s["op"]
    if op == "loss":
        return spr.head_loss(s["hidden"], s["W"], s["targets"], _workspace(s))
    if op == "grad":
        return spr.head_loss_grad(s["hidden"], s["W"], s["targets"], s["lse"], s["grad_loss"], _workspace(s))
    if op == "labels":
        return spr.verifier_labels_head(s["p_hidden"], s["p_W"], s["q_hidden"], s["q_W"], s["tokens"], s["lambdas"],
                                        _workspace(s))
    if op == "pack":
        d = s["hidden"].shape[1]
        return spr.hidden_unpack8(spr.hidden_pack8(s["hidden"]), d, s["hidden"].dtype)
    loss = spr.verifier_train_step8(s["packed"], s["d"], s["labels"], s["theta"], s["m"], s["v"], STEP, LR,
                                    _workspace(s), beta1=BETA1, beta2=BETA2, eps=EPS)
    return loss, s["theta"], s["m"], s["v"]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    es, N, op = 4 if case["dt"] == "f32" else 2, case["N"], case["op"]
    if op == "loss":
        d, V = case["d"], case["V"]
        return {"bytes": es * d * (N + V) + 12 * N, "flops": 2 * N * d * V}
    if op == "grad":           # the logits' product again, and the two products of the gradient
        d, V = case["d"], case["V"]
        return {"bytes": 2 * es * d * (N + V) + 12 * N, "flops": 6 * N * d * V}
    if op == "labels":
        w = case["dq"] + case["dp"]
        return {"bytes": es * w * (N + case["V"]) + (8 + len(LAMBDAS)) * N, "flops": 2 * N * w * case["V"]}
    d = case["d"]
    row = (d + (d + BLOCK - 1) // BLOCK + 15) // 16 * 16
    if op == "pack":           # read, write packed; read packed, write
        return {"bytes": N * (2 * es * d + 2 * row), "flops": 4 * N * d}
    return {"bytes": N * (row + 1) + 24 * (d + 1), "flops": 4 * N * d}


# ---------------------------------------------------------------------------- 64 bits, from the definitions


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    f64 = torch.float64
    if op == "loss":
        l = s["hidden"].to(f64) @ s["W"].to(f64).T
        m = l.max(1).values
        lse = m + (l - m[:, None]).exp_().sum(1).log()
        t = s["targets"].long()
        loss = lse - (s["hidden"].to(f64) * s["W"][t.clamp(min=0)].to(f64)).sum(1)
        return loss.masked_fill(t < 0, 0.0), lse
    if op == "grad":
        rows = (s["targets"] >= 0).nonzero()[:, 0]
        H, W, t = s["hidden"][rows].to(f64), s["W"].to(f64), s["targets"][rows].long()
        D = ((H @ W.T) - s["lse"][rows].to(f64)[:, None]).exp_()
        D[torch.arange(len(rows), device=D.device), t] -= 1.0
        D *= s["grad_loss"][rows].to(f64)[:, None]
        dh = torch.zeros(s["hidden"].shape, dtype=f64, device=D.device)
        dh[rows] = D @ W
        return dh, D.T @ H
    if op == "labels":
        lp = torch.log_softmax(s["p_hidden"].to(f64) @ s["p_W"].to(f64).T, 1)
        lq = torch.log_softmax(s["q_hidden"].to(f64) @ s["q_W"].to(f64).T, 1)
        i = torch.arange(case["N"], device=lp.device)
        ratio = (lq[i, s["tokens"].long()] - lp[i, s["tokens"].long()]).exp()
        return torch.stack([(ratio <= lam).to(torch.uint8) for lam in s["lambdas"]]), ratio
    if op == "pack":
        x = s["hidden"].to(f64)
        out = torch.empty_like(x)
        powers = torch.tensor([2.0 ** e for e in range(-126, 128)], dtype=f64, device=x.device)
        for b in range(0, case["d"], BLOCK):
            y = x[:, b:b + BLOCK]
            top = y.abs().amax(1, keepdim=True)
            e = (torch.frexp(top).exponent.long() - 7).clamp(min=-126)
            step = powers[torch.where(top > 0, e, -126) + 126]
            out[:, b:b + BLOCK] = (y / step).round().clamp(-127, 127) * step
        return out
    d, N = s["d"], case["N"]
    raw = s["packed"].view(torch.int8).to(f64)
    powers = torch.tensor([2.0 ** e for e in range(-128, 128)], dtype=f64, device=raw.device)
    S = raw[:, :d] * powers[raw[:, d:d + (d + BLOCK - 1) // BLOCK].long() + 128].repeat_interleave(BLOCK, 1)[:, :d]
    theta, m, v, y = (s[k].to(f64) for k in ("theta", "m", "v", "labels"))
    z = (S * theta[:d]).sum(1) + theta[d]
    loss = (torch.logaddexp(z, torch.zeros_like(z)) - y * z).sum() / N
    r = 1.0 / (1.0 + torch.exp(-z)) - y
    grad = torch.cat([(S * r[:, None]).sum(0), r.sum().reshape(1)]) / N
    m = BETA1 * m + (1.0 - BETA1) * grad
    v = BETA2 * v + (1.0 - BETA2) * grad ** 2
    theta = theta - LR * (m / (1.0 - BETA1 ** STEP)) / ((v / (1.0 - BETA2 ** STEP)).sqrt() + EPS)
    return loss.reshape(1), theta, m, v
