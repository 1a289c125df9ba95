"""head_loss, head_loss_grad and verifier_labels_head against plain float64.

Bounds, with u = 2^-23 (an accumulator that rounds or truncates loses at most u of its running
magnitude per addition) and A = |hidden| |W|^T:
  logit   a product of d terms is added up in groups of 16: off by at most (d/16 + 16) u A (fp32
          operands: the three bf16 parts leave 2^-24 of each factor, inside the 16)
  lse     as the worst logit of the row, plus a few u of |lse| and of the exponentials
  D       exp(l - lse) is off by the two above; D is then rounded to bf16: 2^-8 |D| (bf16 operands)
  dH, dW  the sum over |D| |W| or |D| |hidden| of these, (terms/16 + 16) u of the sum for the additions,
          and the rounding of the result, 2^-8 in bf16
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
IDS = {torch.bfloat16: "bf16", torch.float32: "f32"}


@pytest.fixture(scope="module")
def spr():
    import paper_2502_04557_b200 as s
    s.lib()
    return s


def problem(N, d, V, dtype, seed, ignore=0.2, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn((N, d), generator=g).to(dtype).cuda()
    w = (torch.randn((V, d), generator=g) * (scale / d ** 0.5)).to(dtype).cuda()
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    if ignore:
        t[torch.rand(N, generator=g) < ignore] = -1
    gl = (torch.rand(N, generator=g) + 0.1) / max(N, 1)
    return h, w, t.cuda(), gl.cuda()


def code(spr, dtype):
    return spr.F32 if dtype == torch.float32 else spr.BF16


def workspace(spr, op, N, V, d, dtype, h=0):
    n = spr.workspace_bytes(op, N, 1, V, d, h, code(spr, dtype))
    assert n > 0
    return spr.Workspace(n)


def logit_bound(h, w):
    d = h.shape[1]
    return (d / 16 + 16) * U * (h.double().abs() @ w.double().abs().T)


def reference_loss(h, w, t):
    l = h.double() @ w.double().T
    lse = torch.logsumexp(l, 1)
    pick = l.gather(1, t.long().clamp(min=0)[:, None])[:, 0]
    return l, lse, torch.where(t >= 0, lse - pick, torch.zeros_like(lse))


def check_loss(spr, h, w, t, ws=None):
    N, d = h.shape
    ws = ws or workspace(spr, spr.OP_HEAD_LOSS, N, w.shape[0], d, h.dtype)
    loss, lse = spr.head_loss(h, w, t, ws)
    assert ws.device_status() == 0
    _, want_lse, want = reference_loss(h, w, t)
    tol = logit_bound(h, w).amax(1) + 16 * U * (1 + want_lse.abs())
    assert bool(((lse.double() - want_lse).abs() <= tol).all()), float(((lse.double() - want_lse).abs() / tol).max())
    assert bool(((loss.double() - want).abs() <= 2 * tol).all())
    assert bool((loss[t < 0] == 0).all()) and bool((loss >= 0).all())
    return loss, lse


def check_grad(spr, h, w, t, gl, lse, ws=None, d_rounding=2.0 ** -8, **kw):
    N, d = h.shape
    V = w.shape[0]
    ws = ws or workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, h.dtype)
    dh, dw = spr.head_loss_grad(h, w, t, lse, gl, ws, **kw)
    assert ws.device_status() == 0
    keep = (t >= 0)[:, None]
    H, W = torch.where(keep, h.double(), 0.0), w.double()
    p = torch.exp(H @ W.T - lse.double()[:, None])
    hot = torch.zeros_like(p).scatter_(1, t.long().clamp(min=0)[:, None], 1.0)
    g = gl.double()[:, None]
    D = torch.where(keep, g * (p - hot), 0.0)
    # what D may be off by: the logit's error, exp and its argument, and the rounding to bf16
    dD = torch.where(keep, g.abs() * p * (logit_bound(H, W) + (8 + lse.double().abs()[:, None] * 2) * U), 0.0) + 4 * U * D.abs()
    # a probability below the smallest normal number, 2^-126, counts as zero (and products of g with one as
    # small): off by less than (1 + g) 2^-126, which is all there is where the true value is of that size
    dD += torch.where(keep, (1 + g.abs()) * 2.0 ** -126, 0.0)
    dD += (d_rounding if h.dtype == torch.bfloat16 else 2.0 ** -23) * D.abs()
    for got, X, off, k in ((dh, W, dD, V), (dw, H, dD.T, N)):
        if got is None:
            continue
        Dm = D if got is dh else D.T
        want = Dm @ X
        tol = off @ X.abs() + (k / 16 + 16 + 40) * U * (Dm.abs() @ X.abs()) + 1.01 * HALF[h.dtype] * want.abs() + 1e-40
        bad = (got.double() - want).abs() / tol
        assert bool((bad <= 1).all()), float(bad.max())
    return dh, dw


SHAPES = [
    (1, 1, 1), (1, 8, 3), (3, 64, 256), (4, 256, 1000), (129, 72, 257), (257, 200, 511), (300, 768, 1025),
    (64, 2048, 700), (5, 7, 5000), (1000, 33, 300), (2, 4104, 130), (520, 136, 9001),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
@pytest.mark.parametrize("N,d,V", SHAPES)
def test_loss_and_gradient(spr, N, d, V, dtype):
    h, w, t, gl = problem(N, d, V, dtype, seed=N * 7 + d * 3 + V)
    _, lse = check_loss(spr, h, w, t)
    check_grad(spr, h, w, t, gl, lse)


@pytest.mark.parametrize("N,d,V", [(20, 40, 17001), (500, 8, 1001), (33, 900, 1500), (9, 1001, 2003), (257, 257, 257), (31, 513, 33),
                                   (8, 770, 1001), (7, 1, 3), (1, 4001, 999)])
def test_small_fp32_heads(spr, N, d, V):
    """Contractions of one round and of several, cut among CTAs or not; and a handful of tokens of a small head."""
    h, w, t, gl = problem(N, d, V, torch.float32, seed=N + d + V)
    _, lse = check_loss(spr, h, w, t)
    check_grad(spr, h, w, t, gl, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
@pytest.mark.parametrize("N,d,V", [(1, 2048, 32000), (2, 136, 20011), (4, 1001, 12007), (8, 264, 15013), (3, 100, 9999), (4, 4096, 10007)])
def test_a_handful_of_tokens_of_a_large_head(spr, N, d, V, dtype):
    """Every CTA goes round its rows of W more than once."""
    h, w, t, gl = problem(N, d, V, dtype, seed=N + d + V)
    _, lse = check_loss(spr, h, w, t)
    check_grad(spr, h, w, t, gl, lse)


@pytest.mark.parametrize("N,d,V", [(9, 1024, 16401), (16, 2048, 8200), (17, 1001, 17011), (24, 520, 32300), (25, 520, 32300)])
def test_fp32_tokens_in_several_passes(spr, N, d, V):
    """Eight tokens at a time under a head of 2^24 elements: the loss up to 24 tokens, the gradient, which adds to its dW,
    up to 16; the workspace of one call serves the next."""
    h, w, t, gl = problem(N, d, V, torch.float32, seed=N + d)
    _, lse = check_loss(spr, h, w, t)
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.float32)
    first = check_grad(spr, h, w, t, gl, lse, ws=ws)
    again = spr.head_loss_grad(h, w, t, lse, gl, ws)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    dh, none = spr.head_loss_grad(h, w, t, lse, gl, ws, want_W=False)
    none2, dw = spr.head_loss_grad(h, w, t, lse, gl, ws, want_hidden=False)
    assert none is None and none2 is None and torch.equal(dh, first[0]) and torch.equal(dw, first[1])


@pytest.mark.parametrize("N,d,V,dtype", [(2048, 512, 30011, torch.bfloat16), (4096, 256, 128256, torch.bfloat16),
                                         (700, 264, 50257, torch.bfloat16), (1500, 136, 33000, torch.float32)],
                         ids=lambda v: str(v).replace("torch.", ""))
def test_vocabulary_pieces_and_split_contractions(spr, N, d, V, dtype):
    """Sizes at which the vocabulary goes by in several pieces, or dH's contraction is cut."""
    h, w, t, gl = problem(N, d, V, dtype, seed=5)
    _, lse = check_loss(spr, h, w, t)
    check_grad(spr, h, w, t, gl, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
def test_one_gradient_alone_equals_both(spr, dtype):
    h, w, t, gl = problem(130, 96, 700, dtype, seed=3)
    _, lse = check_loss(spr, h, w, t)
    dh, dw = check_grad(spr, h, w, t, gl, lse)
    a, none = check_grad(spr, h, w, t, gl, lse, want_W=False)
    assert none is None and torch.equal(a, dh)
    none, b = check_grad(spr, h, w, t, gl, lse, want_hidden=False)
    assert none is None and torch.equal(b, dw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
@pytest.mark.parametrize("d", [64, 67])
def test_padding_rows_hold_anything(spr, d, dtype):
    """Rows without a target hold NaN and infinities: no other row and no sum sees them."""
    N, V = 300, 515
    h, w, t, gl = problem(N, d, V, dtype, seed=8, ignore=0.0)
    pad = torch.arange(N, device="cuda") % 3 == 1
    t[pad] = -100
    _, clean_lse = check_loss(spr, h, w, t)
    clean = check_grad(spr, h, w, t, gl, clean_lse)
    dirty = h.clone()
    dirty[pad] = float("nan")
    dirty[4] = float("inf")
    gl2, lse2 = gl.clone(), clean_lse.clone()
    gl2[pad], lse2[pad] = float("nan"), float("-inf")
    ws = workspace(spr, spr.OP_HEAD_LOSS, N, V, d, dtype)
    loss, lse = spr.head_loss(dirty, w, t, ws)
    assert bool((loss[pad] == 0).all())
    assert torch.equal(lse[~pad], clean_lse[~pad])
    wg = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, dtype)
    got = spr.head_loss_grad(dirty, w, t, lse2, gl2, wg)
    assert wg.device_status() == 0
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    assert bool((got[0][pad] == 0).all())
    # a live row that is not finite is its own affair in the loss
    bad = h.clone()
    bad[5] = float("nan")
    loss, lse = spr.head_loss(bad, w, t, ws)
    assert bool(lse[5].isnan()) and bool(loss[5].isnan())
    other = torch.arange(N, device="cuda") != 5
    assert torch.equal(lse[other & ~pad], clean_lse[other & ~pad])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
def test_all_padding_and_empty_batches(spr, dtype):
    N, d, V = 70, 72, 400
    h, w, t, gl = problem(N, d, V, dtype, seed=8, ignore=0.0)
    t.fill_(-1)
    _, lse = check_loss(spr, h, w, t)
    dh, dw = check_grad(spr, h, w, t, gl, lse)
    assert not dh.any() and not dw.any()
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, 1, V, d, dtype)
    empty = torch.empty((0, d), dtype=dtype, device="cuda")
    none_t, none_f = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = spr.head_loss(empty, w, none_t, ws)
    assert loss.shape == (0,) and lse.shape == (0,)
    dw = torch.full((V, d), 7.0, dtype=dtype, device="cuda")
    dh, dw = spr.head_loss_grad(empty, w, none_t, none_f, none_f, ws, out=(None, dw))
    assert dh.shape == (0, d) and not dw.any()


def test_bad_targets_are_reported_and_have_no_gradient(spr):
    N, d, V = 40, 64, 300
    h, w, t, gl = problem(N, d, V, torch.bfloat16, seed=9, ignore=0.0)
    _, lse = check_loss(spr, h, w, t)
    pad = t.clone()
    pad[7] = -1
    want = check_grad(spr, h, w, pad, gl, lse)
    t[7] = V
    ws = workspace(spr, spr.OP_HEAD_LOSS, N, V, d, h.dtype)
    loss, lse2 = spr.head_loss(h, w, t, ws)
    assert ws.device_status() == 6 and ws.device_status() == 0
    assert float(loss[7]) == -1.0 and torch.equal(lse, lse2)
    wg = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, h.dtype)
    got = spr.head_loss_grad(h, w, t, lse, gl, wg)
    assert wg.device_status() == 6
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_extreme_logits(spr):
    """One column far above the rest (loss 0 or huge), and logits that spread over hundreds."""
    N, d, V = 6, 64, 1000
    h = torch.zeros((N, d), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    h[:, 0] = torch.tensor([1.0, 1.0, 30.0, -30.0, 0.0, 200.0])
    w[:, 0] = torch.linspace(-8, 8, V).to(torch.bfloat16)
    w[3, 0] = 100.0
    t = torch.tensor([3, 4, 3, 3, 0, 10], dtype=torch.int32, device="cuda")
    gl = torch.full((N,), 0.5, device="cuda")
    loss, lse = check_loss(spr, h, w, t)
    assert float(loss[0]) == 0.0 and float(loss[2]) == 0.0
    assert float(loss[5]) == pytest.approx(200.0 * (100.0 - float(w[10, 0])), rel=1e-6)
    check_grad(spr, h, w, t, gl, lse)


def test_gradient_against_differences(spr):
    """A step along a random direction changes sum(g loss) as the gradient says: fp32, the loss in
    float64 (the operator's own loss has too few digits for a difference)."""
    N, d, V = 33, 50, 211
    h, w, t, gl = problem(N, d, V, torch.float32, seed=4)
    ws = workspace(spr, spr.OP_HEAD_LOSS, N, V, d, torch.float32)
    _, lse = spr.head_loss(h, w, t, ws)
    wg = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.float32)
    dh, dw = spr.head_loss_grad(h, w, t, lse, gl, wg)
    g = torch.Generator().manual_seed(1)
    eh, ew = torch.randn((N, d), generator=g).double().cuda(), torch.randn((V, d), generator=g).double().cuda()

    def total(s):
        l = (h.double() + s * eh) @ (w.double() + s * ew).T
        loss = torch.logsumexp(l, 1) - l.gather(1, t.long().clamp(min=0)[:, None])[:, 0]
        return float((gl.double() * torch.where(t >= 0, loss, 0.0)).sum())
    s = 1e-4
    slope = (total(s) - total(-s)) / (2 * s)
    assert slope == pytest.approx(float((dh.double() * eh).sum() + (dw.double() * ew).sum()), rel=1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
def test_runs_are_identical_and_one_workspace_serves_every_call(spr, dtype):
    N, d, V = 333, 136, 3001
    h, w, t, gl = problem(N, d, V, dtype, seed=12)
    n = max(spr.workspace_bytes(op, N, 1, V, d, 0, code(spr, dtype)) for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD))
    ws = spr.Workspace(n)
    first = spr.head_loss(h, w, t, ws)
    grads = spr.head_loss_grad(h, w, t, first[1], gl, ws)
    for _ in range(3):
        ws.buf[256:].random_(0, 255)          # what an earlier call left behind does not matter
        again = spr.head_loss(h, w, t, ws)
        ws.buf[256:].random_(0, 255)
        g2 = spr.head_loss_grad(h, w, t, again[1], gl, ws)
        assert all(torch.equal(a, b) for a, b in zip(first + grads, again + g2))
    assert ws.device_status() == 0


def test_captured_and_replayed_with_new_inputs_and_on_another_stream(spr):
    N, d, V = 200, 128, 2100
    h, w, t, gl = problem(N, d, V, torch.bfloat16, seed=13)
    h2, w2, t2, gl2 = problem(N, d, V, torch.bfloat16, seed=14)
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.bfloat16)
    out = (torch.empty(N, device="cuda"), torch.empty(N, device="cuda"))
    gout = (torch.empty_like(h), torch.empty_like(w))
    want = []
    for a in ((h, w, t, gl), (h2, w2, t2, gl2)):
        loss, lse = spr.head_loss(*a[:3], ws)
        want.append((loss, lse) + spr.head_loss_grad(*a[:3], lse, a[3], ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        spr.head_loss(h, w, t, ws, out=out)
        spr.head_loss_grad(h, w, t, out[1], gl, ws, out=gout)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out + gout, want[0]))
    for a, b in zip((h, w, t, gl), (h2, w2, t2, gl2)):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out + gout, want[1]))
    with torch.cuda.stream(side):
        loss, lse = spr.head_loss(h, w, t, ws)
    side.synchronize()
    assert torch.equal(loss, want[1][0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
def test_bounded_waits_run_out_and_the_workspace_survives(spr, dtype):
    """Nothing is loaded (test hook): the first wait of every CTA pair expires after a few thousand polls, the calls
    end by themselves and report SPR_ERR_TIMEOUT, loss and lse are NaN, labels 0; normal calls follow."""
    N, d, V = 300, 200, 2001
    h, w, t, gl = problem(N, d, V, dtype, seed=15)
    n = max(spr.workspace_bytes(op, N, 1, V, d, 200, code(spr, dtype))
            for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD, spr.OP_VERIFIER_LABELS_HEAD))
    ws = spr.Workspace(n)
    want = spr.head_loss(h, w, t, ws)
    grads = spr.head_loss_grad(h, w, t, want[1], gl, ws)
    labels = spr.verifier_labels_head(h, w, h, w, t.clamp(min=0), [1.5], ws)
    assert ws.device_status() == 0
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    spr.lib().spr_test_pair_kernels(1, 4000)
    try:
        a.record()
        loss, lse = spr.head_loss(h, w, t, ws)
        b.record()
        assert ws.device_status() == 5 and ws.device_status() == 0
        assert bool(loss.isnan().all()) and bool(lse.isnan().all())
        assert a.elapsed_time(b) < 50.0
        spr.head_loss_grad(h, w, t, want[1], gl, ws)
        assert ws.device_status() == 5
        none, ratio = spr.verifier_labels_head(h, w, h, w, t.clamp(min=0), [1.5], ws)
        assert ws.device_status() == 5 and not none.any() and bool(ratio.isnan().all())
    finally:
        spr.lib().spr_test_pair_kernels(0, 0)
    again = spr.head_loss(h, w, t, ws) + spr.head_loss_grad(h, w, t, want[1], gl, ws)
    again += spr.verifier_labels_head(h, w, h, w, t.clamp(min=0), [1.5], ws)
    assert ws.device_status() == 0
    assert all(torch.equal(x, y) for x, y in zip(again, want + grads + labels))


# ---------------------------------------------------------------------------- labels


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
@pytest.mark.parametrize("N,dp,dq,V", [(1, 8, 8, 2), (5, 16, 8, 1000), (40, 72, 64, 513), (300, 256, 136, 5003),
                                       (64, 33, 64, 257), (17, 128, 257, 700), (260, 2048, 1024, 4000)])
def test_labels_from_hidden_states(spr, N, dp, dq, V, dtype):
    g = torch.Generator().manual_seed(N + dp + dq + V)
    ph, pw, x, _ = problem(N, dp, V, dtype, seed=N + V, ignore=0.0)
    qh, qw, _, _ = problem(N, dq, V, dtype, seed=N + V + 1)
    x[torch.rand(N, generator=g).cuda() < 0.1] = V + 2
    lambdas = [1.0, 1.2, 1.5, 0.25, 1e30]
    ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, dp, dtype, h=dq)
    labels, ratio = spr.verifier_labels_head(ph, pw, qh, qw, x, lambdas, ws)
    ok = x < V
    assert ws.device_status() == (0 if bool(ok.all()) else 6)
    at = x.long().clamp(max=V - 1)[:, None]
    lp, lq = ph.double() @ pw.double().T, qh.double() @ qw.double().T
    off = logit_bound(ph, pw).amax(1) + logit_bound(qh, qw).amax(1)
    off += 16 * U * (2 + torch.logsumexp(lp, 1).abs() + torch.logsumexp(lq, 1).abs())
    want = torch.exp(torch.log_softmax(lq, 1).gather(1, at)[:, 0] - torch.log_softmax(lp, 1).gather(1, at)[:, 0])
    err = (ratio.double() / want - 1).abs()
    assert bool((err[ok] <= 2 * off[ok]).all()), float((err / off)[ok].max())
    assert bool((ratio[~ok] == -1).all()) and not labels[:, ~ok].any()
    for i, lam in enumerate(lambdas):
        lam = float(np.float32(lam))
        clear = ok & ((want / lam - 1).abs() > 2 * off)
        assert torch.equal(labels[i][clear].bool(), (want <= lam)[clear])
        assert int((ok & ~clear).sum()) <= max(1, N // 20)


def test_labels_agree_with_those_from_kept_logits(spr):
    """The same batch through verifier_labels on fp32 logits and through the heads."""
    B, K, d, V = 6, 5, 128, 4001
    N = B * K
    ph, pw, x, _ = problem(N, d, V, torch.float32, seed=1, ignore=0.0)
    qh, qw, _, _ = problem(N, d, V, torch.float32, seed=2)
    lp, lq = (ph.double() @ pw.double().T).float(), (qh.double() @ qw.double().T).float()
    w0 = spr.Workspace(spr.workspace_bytes(spr.binding.OP_VERIFIER_LABELS, B, K, V, 0, 0, spr.F32))
    a, ra = spr.binding.verifier_labels(lp.view(B, K, V), lq.view(B, K, V), V, x.view(B, K), [1.0, 1.2, 1.5], w0)
    ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, d, torch.float32, h=d)
    b, rb = spr.verifier_labels_head(ph, pw, qh, qw, x, [1.0, 1.2, 1.5], ws)
    assert bool(((ra.view(-1) / rb - 1).abs() < 2e-4).all())
    clear = torch.stack([(rb / lam - 1).abs() > 2e-4 for lam in (1.0, 1.2, 1.5)])
    assert torch.equal(a.view(3, N)[clear], b[clear])


@pytest.mark.parametrize("N,d,V", [(67, 257, 1003), (33, 64, 31), (100, 3, 20000), (32, 129, 2048), (1, 40, 33), (500, 65, 900)])
def test_fp32_problems_small_enough_for_the_cuda_cores(spr, N, d, V):
    h, w, t, gl = problem(N, d, V, torch.float32, seed=N + d)
    _, lse = check_loss(spr, h, w, t)
    dh, dw = check_grad(spr, h, w, t, gl, lse)
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.float32)
    for _ in range(3):                                       # the tickets are back at zero after every call
        again = spr.head_loss_grad(h, w, t, lse, gl, ws)
        assert torch.equal(again[0], dh) and torch.equal(again[1], dw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
def test_labels_with_heads_on_different_kernels(spr, dtype):
    """A draft head small enough for the CUDA cores (fp32) beside a target head that is not."""
    N, dp, dq, V = 64, 640, 40, 3001
    ph, pw, x, _ = problem(N, dp, V, dtype, seed=1, ignore=0.0)
    qh, qw, _, _ = problem(N, dq, V, dtype, seed=2)
    for a in ((ph, pw, qh, qw), (qh, qw, ph, pw)):
        ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, a[0].shape[1], dtype, h=a[2].shape[1])
        _, ratio = spr.verifier_labels_head(*a, x, [1.0], ws)
        l = [b.double() @ c.double().T for b, c in ((a[0], a[1]), (a[2], a[3]))]
        off = logit_bound(a[0], a[1]).amax(1) + logit_bound(a[2], a[3]).amax(1) + 64 * U * 10
        p, q = (torch.log_softmax(m, 1).gather(1, x.long()[:, None])[:, 0] for m in l)
        assert bool(((ratio.double() / torch.exp(q - p) - 1).abs() <= 2 * off).all()) and ws.device_status() == 0


@pytest.mark.parametrize("N,d,V,dtype", [
    (1, 768, 50257, torch.bfloat16), (1, 4096, 9001, torch.bfloat16), (1, 8, 70000, torch.bfloat16), (4, 1001, 8000, torch.bfloat16),
    (3, 4095, 3001, torch.bfloat16), (2, 30, 40000, torch.bfloat16), (1, 9000, 2000, torch.bfloat16),
    (8, 2048, 5003, torch.float32), (7, 1028, 9000, torch.float32), (5, 513, 33000, torch.float32), (2, 100, 99999, torch.float32),
    (1, 2047, 6001, torch.float32), (4, 4096, 3000, torch.float32), (8, 40, 50257, torch.float32)],
    ids=lambda v: str(v).replace("torch.", ""))
def test_a_handful_of_tokens(spr, N, d, V, dtype):
    """One pass over W: widths that leave lanes or threads idle, rows that start anywhere, a token padded."""
    h, w, t, gl = problem(N, d, V, dtype, seed=N + d, ignore=0.0)
    if N > 2:
        t[1] = -1
        h[1] = float("nan")
        clean = h.clone()
        clean[1] = 0.0
        ws = workspace(spr, spr.OP_HEAD_LOSS, N, V, d, dtype)
        loss, lse = spr.head_loss(h, w, t, ws)
        want = check_loss(spr, clean, w, t)
        ok = torch.arange(N, device="cuda") != 1
        assert torch.equal(loss, want[0]) and torch.equal(lse[ok], want[1][ok])
        wg = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, dtype)
        got = spr.head_loss_grad(h, w, t, want[1], gl, wg)
        ref = check_grad(spr, clean, w, t, gl, want[1])
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    else:
        _, lse = check_loss(spr, h, w, t)
        dh, dw = check_grad(spr, h, w, t, gl, lse)
        assert torch.equal(check_grad(spr, h, w, t, gl, lse, want_W=False)[0], dh)
        assert torch.equal(check_grad(spr, h, w, t, gl, lse, want_hidden=False)[1], dw)


@pytest.mark.parametrize("N,d,V", [(3, 768, 4001), (9, 256, 5000), (64, 768, 3001), (128, 264, 9001), (100, 1001, 700), (128, 72, 128256)])
def test_few_tokens_keep_their_gradient_of_the_logits(spr, N, d, V):
    """Up to 128 bf16 tokens D has two bf16 parts: rounding the first leaves at most 2^-8 of D, and rounding that
    at most 2^-8 of it again: 2^-16 in all."""
    h, w, t, gl = problem(N, d, V, torch.bfloat16, seed=V)
    _, lse = check_loss(spr, h, w, t)
    check_grad(spr, h, w, t, gl, lse, d_rounding=2.0 ** -16)


def framed(shape, dtype):
    """A contiguous tensor of this shape in the middle of a buffer of sevens, 64 of them on either side."""
    n = int(np.prod(shape))
    buf = torch.full((n + 128,), 7.0, device="cuda").to(dtype)
    return buf, buf[64:64 + n].view(shape)


def untouched(buf):
    return bool((buf[:64] == 7).all()) and bool((buf[-64:] == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=IDS.get)
@pytest.mark.parametrize("N,d,V", [(130, 72, 515), (257, 264, 1025), (33, 100, 700), (2, 72, 515), (300, 8, 9001), (129, 67, 300)])
def test_nothing_is_written_beside_the_outputs(spr, N, d, V, dtype):
    h, w, t, gl = problem(N, d, V, dtype, seed=N + V)
    ws = workspace(spr, spr.OP_HEAD_LOSS, N, V, d, dtype)
    (lb, loss), (zb, lse) = framed((N,), torch.float32), framed((N,), torch.float32)
    spr.head_loss(h, w, t, ws, out=(loss, lse))
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, dtype)
    (hb, dh), (wb, dw) = framed((N, d), dtype), framed((V, d), dtype)
    check_grad(spr, h, w, t, gl, lse, ws=ws, out=(dh, dw))
    assert all(untouched(b) for b in (lb, zb, hb, wb))


def test_two_calls_at_once(spr):
    """Two streams, a workspace each: the results are those of the calls alone."""
    a = problem(300, 264, 9001, torch.bfloat16, seed=1)
    b = problem(67, 257, 1003, torch.float32, seed=2)
    def both(h, w, t, gl, ws1, ws2):
        loss, lse = spr.head_loss(h, w, t, ws1)
        return (loss, lse) + tuple(spr.head_loss_grad(h, w, t, lse, gl, ws2))
    def spaces(h, w):
        return [workspace(spr, op, h.shape[0], w.shape[0], h.shape[1], h.dtype) for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD)]
    spaces_a, spaces_b = spaces(a[0], a[1]), spaces(b[0], b[1])
    want = both(*a, *spaces_a), both(*b, *spaces_b)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(s1):
            x = both(*a, *spaces_a)
        with torch.cuda.stream(s2):
            y = both(*b, *spaces_b)
        got.append((x, y))
    torch.cuda.synchronize()
    for x, y in got:
        assert all(torch.equal(p, q) for p, q in zip(x, want[0])) and all(torch.equal(p, q) for p, q in zip(y, want[1]))


def test_a_draft_head_fitted_labelled_and_its_verifier_fitted(spr):
    """The operators one after the other, as they are used: a step on the draft's head along its gradient, labels from
    the new head, states packed, a step of the verifier on them, each against float64 on what it was given."""
    from oracle import training
    N, d, V = 600, 128, 3001
    h, w, t, gl = problem(N, d, V, torch.float32, seed=21, ignore=0.1)
    loss, lse = check_loss(spr, h, w, t)
    dh, dw = check_grad(spr, h, w, t, gl, lse)
    new = (w - 0.5 * dw).to(torch.bfloat16)
    hb, pw = h.to(torch.bfloat16), w.to(torch.bfloat16)
    x = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).cuda()
    ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, d, torch.bfloat16, h=d)
    labels, ratio = spr.verifier_labels_head(hb, pw, hb, new, x, [1.0], ws)
    assert ws.device_status() == 0
    logp = [torch.log_softmax(hb.double() @ m.double().T, 1).gather(1, x.long()[:, None])[:, 0] for m in (pw, new)]
    want = torch.exp(logp[1] - logp[0])
    off = 2 * (logit_bound(hb, pw).amax(1) + logit_bound(hb, new).amax(1)) + 64 * U * (1 + logp[0].abs() + logp[1].abs())
    assert bool(((ratio.double() - want).abs() <= want * (torch.exp(off) - 1) + U).all())
    clear = (want - 1).abs() > want * (torch.exp(off) - 1)
    assert torch.equal(labels[0][clear].bool(), (want <= 1)[clear])
    packed = spr.hidden_pack8(hb)
    S = spr.hidden_unpack8(packed, d, dtype=torch.float32)
    st = [torch.zeros(d + 1, device="cuda") for _ in range(3)]
    ws = spr.Workspace(spr.workspace_bytes(spr.OP_VERIFIER_TRAIN8, 0, 0, 0, d, 0, spr.BF16))
    got = spr.verifier_train_step8(packed, d, labels[0].contiguous(), *st, 1, 0.01, ws)
    zero = np.zeros(d + 1)
    ref, theta, _, _ = training.verifier_train_step(S.cpu().double().numpy(), labels[0].cpu().numpy(), zero, zero, zero, 1, 0.01)
    # all logits are zero: the loss is ln 2 to a rounding; a first step of Adam is lr g / (|g| + eps), and the bound of
    # tests/test_gpu_pack8.py for one step
    assert float(got) == pytest.approx(ref, rel=1e-6)
    assert np.abs(st[0].cpu().double().numpy() - theta).max() <= 1e-3 * 0.01


@pytest.mark.parametrize("grad", [False, True], ids=["loss", "gradient"])
def test_two_host_threads_with_heads_of_different_widths(spr, grad):
    """Two threads, a stream and a workspace each, call the kernel for a handful of tokens over and over, one with 64 KB and
    more of states in shared memory and one with 8 KB: neither call depends on what the other asked for.  (The calls are made
    without the binding's checks, so that the threads spend their time in the library.)"""
    import threading
    N, V, L = 8, 64, spr.lib()
    jobs = []
    for d in (2048 if grad else 4096, 256):
        h, w, t, gl = problem(N, d, V, torch.float32, seed=d)
        # small enough for one round of a CTA or two
        ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD if grad else spr.OP_HEAD_LOSS, N, V, d, torch.float32)
        loss, lse = check_loss(spr, h, w, t)
        want = check_grad(spr, h, w, t, gl, lse) if grad else (loss, lse)
        out = tuple(torch.empty_like(x) for x in want)
        stream = torch.cuda.Stream()
        p = lambda x: x.data_ptr()
        tail = (N, d, V, spr.F32, p(out[0]), p(out[1]), p(ws.buf), ws.nbytes, stream.cuda_stream)
        args = (p(h), p(w), p(t), p(lse), p(gl)) + tail if grad else (p(h), p(w), p(t)) + tail
        jobs.append((args, stream, (h, w, t, gl, lse, ws), out, want))
    torch.cuda.synchronize()
    call, failed = L.head_loss_grad if grad else L.head_loss, []

    def run(args, *rest):
        for _ in range(20000):
            rc = call(*args)
            if rc != 0:
                failed.append(rc)
                return

    threads = [threading.Thread(target=run, args=j) for j in jobs]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    torch.cuda.synchronize()
    assert not failed
    for _, _, (*_, ws), out, want in jobs:
        assert ws.device_status() == 0 and all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("sizes,d,V,dtype", [((150, 128, 3), 768, 50257, torch.bfloat16), ((300, 256, 1), 2048, 32000, torch.bfloat16),
                                             ((600, 512, 130), 100, 5000, torch.bfloat16), ((25, 24, 16, 8, 4), 520, 32300, torch.float32),
                                             ((400, 129, 67, 9), 64, 1003, torch.float32)], ids=lambda v: str(v).replace("torch.", ""))
def test_a_workspace_made_for_the_largest_batch_serves_smaller_ones(spr, sizes, d, V, dtype):
    """A training run's last batch is a short one."""
    spaces = [workspace(spr, op, sizes[0], V, d, dtype, h=d)
              for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD, spr.OP_VERIFIER_LABELS_HEAD)]
    for N in sizes:
        h, w, t, gl = problem(N, d, V, dtype, seed=N)
        _, lse = check_loss(spr, h, w, t, ws=spaces[0])
        check_grad(spr, h, w, t, gl, lse, ws=spaces[1])
        _, ratio = spr.verifier_labels_head(h, w, h, w, t.clamp(min=0), [1.0], spaces[2])
        assert bool((ratio == 1).all()) and spaces[2].device_status() == 0


def mean_offset(h, w, t, gl, lse, dw):
    """Mean relative error of the rows of dW from the ninth on, none of which is a target's: sums of one sign."""
    want = torch.zeros((w.shape[0] - 8, h.shape[1]), dtype=torch.float64, device="cuda")
    for n in range(0, len(h), 1 << 16):
        x, z, g = (a[n:n + (1 << 16)].double() for a in (h, lse, gl))
        want += (torch.exp(x @ w[8:].double().T - z[:, None]) * g[:, None]).T @ x
    return float((dw[8:].double() / want - 1).mean()), want.numel()


def test_a_gradient_over_a_million_tokens_is_not_off_to_one_side(spr):
    """The tensor pipe truncates what it adds up, by up to 2^-23 of the running sum per 16 tokens and always towards zero: a sum
    of one sign over 2^20 tokens in one accumulator would come out some 1.4e-3 low.  One takes at most 2^15 of them, which is
    2^11 2^-23 = 2^-12 at the very most.  Beside it D (a factor of two and more apart from token to token) and the result are
    rounded to bf16, to either side: the mean of n results is off by less than five deviations, 5 2^-8 / sqrt(3 n)."""
    N, d, V = 1 << 20, 8, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    h = (torch.rand((N, d), generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    w = (torch.randn((V, d), generator=g, device="cuda") * 0.5).to(torch.bfloat16)
    t = torch.randint(0, 8, (N,), generator=g, dtype=torch.int32, device="cuda")
    gl = torch.full((N,), 1.0 / N, device="cuda")
    _, lse = spr.head_loss(h, w, t, workspace(spr, spr.OP_HEAD_LOSS, N, V, d, torch.bfloat16))
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.bfloat16)
    _, dw = spr.head_loss_grad(h, w, t, lse, gl, ws, want_hidden=False)
    assert ws.device_status() == 0
    off, n = mean_offset(h, w, t, gl, lse, dw)
    assert abs(off) <= 2.0 ** -12 + 5 * 2.0 ** -8 / (3 * n) ** 0.5


def test_the_gradient_of_wide_states_is_not_off_to_one_side(spr):
    """Logits of 20 as sums of one sign over 65536 columns: an accumulator takes at most 4096 of them, so a logit is low by at
    most 2^8 2^-23 of itself, 6.1e-4, and D by as much (in one accumulator: some 1.8e-3; 64 tokens keep D in two parts).
    The mean of 10^7 results, rounded to bf16 to either side, adds less than 1e-5."""
    N, d, V = 64, 65536, 200
    g = torch.Generator(device="cuda").manual_seed(1)
    h = (torch.rand((N, d), generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    w = ((torch.rand((V, d), generator=g, device="cuda") + 0.5) * (20.0 / d)).to(torch.bfloat16)
    t = torch.randint(0, 8, (N,), generator=g, dtype=torch.int32, device="cuda")
    gl = torch.rand(N, generator=g, device="cuda") + 0.5
    _, lse = spr.head_loss(h, w, t, workspace(spr, spr.OP_HEAD_LOSS, N, V, d, torch.bfloat16))
    ws = workspace(spr, spr.OP_HEAD_LOSS_GRAD, N, V, d, torch.bfloat16)
    _, dw = spr.head_loss_grad(h, w, t, lse, gl, ws, want_hidden=False)
    assert ws.device_status() == 0
    logit = float((h.double() @ w.double().T).max())
    off, _ = mean_offset(h, w, t, gl, lse, dw)
    assert abs(off) <= logit * 2.0 ** -15 + 1e-5


@pytest.mark.parametrize("p_wide", [True, False], ids=["target", "draft"])
def test_a_ratio_from_two_kernels_is_as_exact_as_from_one(spr, p_wide):
    """Four tokens of one model are too wide for the pass over W and take the tensor pipe, which truncates what it adds up; in a
    ratio to a model that does not, nothing of that cancels.  It is held to what the shortest chunks that are used anywhere,
    of two blocks, would leave: a truncation takes half a unit on average, at most 2^-24 of the running sum, and there are
    eight to a chunk, on average of half the chunk's share of a logit: 4 2^-24 of the mean logit under the softmax, beside
    2^-21 for the roundings of both models' statistics."""
    N, V, wide, narrow = 4, 32000, 20480, 2048
    ph, pw, x, _ = problem(N, wide, V, torch.bfloat16, seed=1, ignore=0.0)
    qh, qw, _, _ = problem(N, narrow, V, torch.bfloat16, seed=2)
    a = (ph, pw, qh, qw) if p_wide else (qh, qw, ph, pw)
    ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, a[0].shape[1], torch.bfloat16, h=a[2].shape[1])
    _, ratio = spr.verifier_labels_head(*a, x, [1.0], ws)
    assert ws.device_status() == 0
    l = [h.double() @ w.double().T for h, w in ((a[0], a[1]), (a[2], a[3]))]
    p, q = (torch.log_softmax(m, 1).gather(1, x.long()[:, None])[:, 0] for m in l)
    off = float((ratio.double() / torch.exp(q - p) - 1).mean())
    logit = max(float((torch.softmax(m, 1) * m).sum(1).mean()) for m in l)
    assert abs(off) <= 4 * 2.0 ** -24 * logit + 2.0 ** -21


@pytest.mark.parametrize("dq,dp", [(128, 256), (192, 384), (256, 768), (320, 640), (768, 1536)])
def test_ratios_of_narrow_models_are_not_off_to_one_side(spr, dq, dp):
    """Both models' logits are added up in chunks of one length, so what truncation takes off their log-sum-exps is the same and
    the mean of many ratios shows none of it.  What is left goes either way: a logit is rounded at most twice per model behind
    its chunks, 2^-24 of itself each (the softmax of logits this far apart is that of the few largest), so a ratio is off by at
    most 4 2^-24 of the mean logit under the softmax, and the mean of N of them by less than five times that over sqrt(N)."""
    N, V = 2000, 3000
    ph, pw, x, _ = problem(N, dp, V, torch.bfloat16, seed=dp, ignore=0.0, scale=8.0)
    qh, qw, _, _ = problem(N, dq, V, torch.bfloat16, seed=dq + 1, scale=8.0)
    ws = workspace(spr, spr.OP_VERIFIER_LABELS_HEAD, N, V, dp, torch.bfloat16, h=dq)
    _, ratio = spr.verifier_labels_head(ph, pw, qh, qw, x, [1.0], ws)
    assert ws.device_status() == 0
    l = [h.double() @ w.double().T for h, w in ((ph, pw), (qh, qw))]
    p, q = (torch.log_softmax(m, 1).gather(1, x.long()[:, None])[:, 0] for m in l)
    ok = (q - p).abs() < 60                          # a ratio is a float: larger ones are rounded to infinity or nothing
    off = (ratio.double() / torch.exp(q - p) - 1)[ok]
    logit = max(float((torch.softmax(m, 1) * m).sum(1).mean()) for m in l)
    assert int(ok.sum()) > N // 2
    assert abs(float(off.mean())) <= 5 * 4 * 2.0 ** -24 * logit / float(ok.sum()) ** 0.5


@pytest.mark.parametrize("N,d,V", [(40000, 67, 300), (33000, 72, 300), (256, 8192, 70000), (300, 8200, 700), (20, 4200, 3000), (20, 4203, 3000)])
def test_long_bf16_contractions_in_every_form(spr, N, d, V):
    """Contractions of more than one chunk: dW over the tokens, stored as boxes or from rows that start anywhere; dH over the
    vocabulary, in ranges that are added up; logits of wide states, with D in one part and in two."""
    h, w, t, gl = problem(N, d, V, torch.bfloat16, seed=N + d)
    _, lse = check_loss(spr, h, w, t)
    dh, dw = check_grad(spr, h, w, t, gl, lse, d_rounding=2.0 ** -8 if N > 128 else 2.0 ** -16)
    assert torch.equal(check_grad(spr, h, w, t, gl, lse, want_W=False)[0], dh)
    assert torch.equal(check_grad(spr, h, w, t, gl, lse, want_hidden=False)[1], dw)
