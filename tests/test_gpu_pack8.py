"""hidden_pack8 / hidden_unpack8 and verifier_train_step8.

Packing is compared bit for bit with a numpy statement of the format (nothing in it is inexact but
the one rounding it defines); training with the float64 oracle on the values the packed rows stand for.
"""
import numpy as np
import pytest
import torch

from helpers import to_np
from oracle import training
from test_gpu_fit import teacher_problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spr():
    import paper_2502_04557_b200 as s
    s.lib()
    return s


def pack_ref(x):
    """float64 [N,d] -> packed bytes [N, pitch]"""
    N, d = x.shape
    nb = (d + 31) // 32
    out = np.zeros((N, (d + nb + 15) // 16 * 16), np.int8)
    for b in range(nb):
        blk = x[:, 32 * b:32 * b + 32]
        finite = np.isfinite(blk).all(1)
        blk = np.where(finite[:, None], blk, 0.0)
        top = np.abs(blk).max(1)
        e = np.maximum(np.frexp(top)[1] - 7, -126)
        e[top == 0] = -126
        q = np.clip(np.rint(np.ldexp(blk, -e[:, None])), -127, 127)
        out[:, 32 * b:32 * b + blk.shape[1]] = np.where(finite[:, None], q, 0)
        out[:, d + b] = np.where(finite, e, -128)
    return out.view(np.uint8)


def unpack_ref(p, d):
    p = p.view(np.int8)
    nb = (d + 31) // 32
    e = p[:, d:d + nb].astype(np.int32).repeat(32, 1)[:, :d]
    return np.where(e == -128, np.nan, np.ldexp(p[:, :d].astype(np.float64), e))


def values(N, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((N, d), generator=g) * torch.exp(3 * torch.randn((N, 1), generator=g))
    x[torch.rand((N, d), generator=g) < 0.05] = 0.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 255), (4, 256), (3, 257), (2, 1000), (9, 768),
                                 (300, 2048), (2, 4099), (3000, 40)])
def test_pack_and_unpack(spr, N, d, dtype):
    x = values(N, d, dtype, seed=N + d)
    packed = spr.hidden_pack8(x.cuda())
    assert packed.shape == (N, spr.pack8_pitch(d)) == (N, (d + (d + 31) // 32 + 15) // 16 * 16)
    want = pack_ref(x.double().numpy())
    assert np.array_equal(packed.cpu().numpy(), want)
    for ty in (torch.float32, torch.bfloat16):
        back = spr.hidden_unpack8(packed, d, ty)
        assert np.array_equal(back.cpu().double().numpy(), unpack_ref(want, d))
    # at most half a step off, a whole one where the byte is clamped
    off = np.abs(unpack_ref(want, d) - x.double().numpy())
    e = want.view(np.int8)[:, d:d + (d + 31) // 32].astype(np.int32).repeat(32, 1)[:, :d]
    clamped = np.abs(np.ldexp(x.double().numpy(), -e)) > 127.5
    assert np.all(off <= np.ldexp(np.where(clamped, 1.0, 0.5), e))


def test_pack_extremes(spr):
    big, tiny = 3.3895313892515355e38, 2.0 ** -133
    x = torch.zeros((8, 64), dtype=torch.bfloat16)
    x[0, 0], x[0, 1] = big, -big
    x[1, 5] = tiny
    x[2, :] = 2.0 ** -126
    x[3, 3] = float("inf")
    x[4, 40] = float("nan")
    x[5, :] = torch.arange(64) - 31.5
    x[6, 0] = -0.0
    x[7, :3] = torch.tensor([127.0, 127.5, 0.5])
    packed = spr.hidden_pack8(x.cuda())
    assert np.array_equal(packed.cpu().numpy(), pack_ref(x.double().numpy()))
    back = spr.hidden_unpack8(packed, 64).cpu()
    assert back[3, :32].isnan().all() and not back[3, 32:].isnan().any()
    assert back[4, 32:].isnan().all() and not back[4, :32].isnan().any()
    assert float(back[7, 1]) == 127.0 or float(back[7, 1]) == 128.0


def test_pack_of_an_unaligned_view_and_of_nothing(spr):
    x = values(6, 512, torch.bfloat16, 3).cuda().flatten()
    view = x[1:1 + 5 * 512].view(5, 512)                      # contiguous, two bytes past a 16-byte boundary
    assert np.array_equal(spr.hidden_pack8(view).cpu().numpy(), pack_ref(view.cpu().double().numpy()))
    buf = torch.empty(5 * 512 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(5, 512)
    packed = spr.hidden_pack8(view)
    assert torch.equal(spr.hidden_unpack8(packed, 512, out=buf), spr.hidden_unpack8(packed, 512))
    none = spr.hidden_pack8(torch.empty((0, 40), device="cuda"))
    assert none.shape == (0, 48) and spr.hidden_unpack8(none, 40).shape == (0, 40)


def step_ws(spr, d):
    return spr.Workspace(spr.workspace_bytes(spr.OP_VERIFIER_TRAIN8, 0, 0, 0, d, 0, spr.BF16))


@pytest.mark.parametrize("N,d", [(1, 16), (7, 64), (5000, 768), (20000, 256), (3000, 2048), (2000, 4096), (4001, 1008),
                                 (60000, 512), (30001, 1024), (24000, 2048), (9000, 2560), (12000, 4096), (70001, 128),
                                 (50003, 528), (8000, 1536), (33, 1040)])
def test_training_steps_match_the_oracle(spr, N, d):
    """As for verifier_train_step: fp32 sums against float64, loss to 2e-5, and a relative gradient error e
    moves a parameter by about lr e per step: bound 1e-3 lr t.  The loss of a step is that of the parameters
    before it, which already differ by some delta (at most that bound): ln(1 + e^z) - y z changes by no more
    than z does, so the mean loss by at most mean_i sum_j |s_ij| |delta_j|, and by the rounding of the fp32
    dot product, 2^-24 (d/32 + 16) sum_j |s_ij theta_j| (a lane adds d/32 terms).  Once a small set is
    separated the loss is tiny, and these terms, not 2e-5 of it, are what it can be held to."""
    S, y = teacher_problem(N, d, torch.bfloat16, seed=N + d)
    packed = spr.hidden_pack8(S.cuda())
    Sn = unpack_ref(packed.cpu().numpy(), d)
    lr, steps = 0.02, 8
    ws = step_ws(spr, d)
    theta, m, v = (torch.zeros(d + 1, device="cuda") for _ in range(3))
    rt, rm, rv = np.zeros(d + 1), np.zeros(d + 1), np.zeros(d + 1)
    for t in range(1, steps + 1):
        before = theta.cpu().double().numpy()
        slack = np.mean(np.abs(Sn) @ np.abs(before - rt)[:d]) + abs(before[d] - rt[d])
        slack += 2.0 ** -24 * (d / 32 + 16) * (np.mean(np.abs(Sn) @ np.abs(rt[:d])) + abs(rt[d]))
        loss = spr.verifier_train_step8(packed, d, y.cuda(), theta, m, v, t, lr, ws)
        want, rt, rm, rv = training.verifier_train_step(Sn, y.numpy(), rt, rm, rv, t, lr)
        assert abs(float(loss) - want) < 2e-5 * want + slack
        assert np.abs(theta.cpu().double().numpy() - rt).max() <= 1e-3 * lr * t
    assert ws.device_status() == 0


@pytest.mark.parametrize("N,d", [(5000, 768), (9001, 2048), (3000, 4096), (700, 128)])
def test_a_step_equals_the_step_on_unpacked_states(spr, N, d):
    """The packed values are bf16 numbers, so verifier_train_step on the unpacked states is the same
    problem: the two differ by the order of their sums alone.  Loss: a mean of N terms, fp32 logits."""
    S, y = teacher_problem(N, d, torch.bfloat16, seed=N)
    packed = spr.hidden_pack8(S.cuda())
    U = spr.hidden_unpack8(packed, d)
    g = torch.Generator().manual_seed(1)
    theta = (0.05 * torch.randn(d + 1, generator=g)).cuda()
    state = [(theta.clone(), torch.zeros_like(theta), torch.zeros_like(theta)) for _ in range(2)]
    ws = step_ws(spr, d)
    w2 = spr.Workspace(spr.workspace_bytes(spr.binding.OP_VERIFIER_TRAIN, 0, 0, 0, d, 0, spr.BF16))
    a = spr.verifier_train_step8(packed, d, y.cuda(), *state[0], 1, 0.01, ws)
    b = spr.binding.verifier_train_step(U, y.cuda(), *state[1], 1, 0.01, w2)
    assert float(a) == pytest.approx(float(b), rel=2e-6)
    # m = 0.1 g: compared to the size of the gradient's terms, mean |s_ij|, over N / teams of them in fp32
    scale = U.float().abs().mean(0).amax()
    assert float((state[0][1] - state[1][1]).abs().max()) <= 0.1 * 1e-5 * max(1.0, float(scale))


def test_a_step_is_reproducible_and_a_marked_block_shows(spr):
    S, y = teacher_problem(6000, 768, torch.bfloat16, seed=9)
    packed = spr.hidden_pack8(S.cuda())
    ws, yg = step_ws(spr, 768), y.cuda()
    runs = []
    for _ in range(2):
        st = [torch.zeros(769, device="cuda") for _ in range(3)]
        loss = [spr.verifier_train_step8(packed, 768, yg, *st, t, 0.02, ws).clone() for t in (1, 2, 3)]
        runs.append(loss + st)
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    S[17, 100] = float("nan")
    st = [torch.zeros(769, device="cuda") for _ in range(3)]
    assert bool(spr.verifier_train_step8(spr.hidden_pack8(S.cuda()), 768, yg, *st, 1, 0.02, ws).isnan().all())


def test_a_captured_step(spr):
    S, y = teacher_problem(3000, 512, torch.bfloat16, seed=19)
    packed, yg, ws = spr.hidden_pack8(S.cuda()), y.cuda(), step_ws(spr, 512)
    a, b = ([torch.zeros(513, device="cuda") for _ in range(3)] for _ in range(2))
    loss = torch.empty(1, device="cuda")
    spr.verifier_train_step8(packed, 512, yg, *a, 1, 0.02, ws, loss=loss)
    want = [x.clone() for x in a] + [loss.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spr.verifier_train_step8(packed, 512, yg, *b, 1, 0.02, ws, loss=loss)
    for x in b:
        x.zero_()
    loss.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(b + [loss], want))


@pytest.mark.parametrize("N,d", [(5000, 768), (9000, 2048), (4000, 4096), (9, 64), (30001, 256)])
def test_bounded_wait_runs_out_and_nothing_is_stepped(spr, N, d):
    """No tile is ever fetched (test flag): the first wait of every CTA expires after a few thousand polls, the
    launch ends by itself, reports SPR_ERR_TIMEOUT and takes no step; the next call is a normal step."""
    S, y = teacher_problem(N, d, torch.bfloat16, seed=21)
    packed, yg, ws = spr.hidden_pack8(S.cuda()), y.cuda(), step_ws(spr, d)
    g = torch.Generator().manual_seed(22)
    state = [(0.05 * torch.randn(d + 1, generator=g)).cuda(), torch.rand(d + 1, generator=g).cuda() * 1e-3,
             torch.rand(d + 1, generator=g).cuda() * 1e-6]
    before, want = [x.clone() for x in state], [x.clone() for x in state]
    loss_ok = spr.verifier_train_step8(packed, d, yg, *want, 3, 0.01, ws).clone()
    assert ws.device_status() == 0
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    loss = spr.verifier_train_step8(packed, d, yg, *state, 3, 0.01, ws, test_flags=1, spin_limit=4000)
    b.record()
    assert ws.device_status() == 5 and ws.device_status() == 0
    assert bool(loss.isnan().all()) and all(torch.equal(x, r) for x, r in zip(state, before))
    assert a.elapsed_time(b) < 50.0
    loss = spr.verifier_train_step8(packed, d, yg, *state, 3, 0.01, ws)
    assert ws.device_status() == 0
    assert torch.equal(loss, loss_ok) and all(torch.equal(x, w) for x, w in zip(state, want))


@pytest.mark.parametrize("N,d", [(400001, 48), (330007, 512), (170001, 528), (90003, 1040), (85001, 2048), (50001, 2064)])
def test_many_tiles_per_cta(spr, N, d):
    """Rings of tiles go round several times, for every way the columns are dealt to warps.  Against float64: a
    logit is off by dz = 2^-24 (d/32 + 16) sum_j |s_ij w_j|, hence a residual by dz / 4 and two roundings of its
    own; residuals are written in 22 bits relative to the largest of a tile (at most 1), and at most 50 tiles are
    added up in fp32.  So m = 0.1 grad is off by at most 0.1 mean_i |s_ij| times all that."""
    g = torch.Generator(device="cuda").manual_seed(d)
    S = torch.randn((N, d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    y = (torch.rand(N, generator=g, device="cuda") < 0.3).to(torch.uint8)
    theta = torch.randn(d + 1, generator=g, device="cuda") / d ** 0.5
    packed = spr.hidden_pack8(S)
    X = spr.hidden_unpack8(packed, d, dtype=torch.float32).double()
    w = theta.double()
    z = X @ w[:d] + w[d]
    r = torch.sigmoid(z) - y
    state = [theta.clone(), torch.zeros_like(theta), torch.zeros_like(theta)]
    ws = step_ws(spr, d)
    loss = spr.verifier_train_step8(packed, d, y, *state, 1, 0.01, ws)
    assert ws.device_status() == 0
    A = X.abs()
    dz = float((A @ w[:d].abs()).max() + w[d].abs()) * 2.0 ** -24 * (d / 32 + 16)
    off = 2.0 ** -22 + 60 * 2.0 ** -24 + dz / 4
    want = torch.cat([X.t() @ r, r.sum().reshape(1)]) / N
    size = torch.cat([A.mean(0), torch.ones(1, device="cuda", dtype=torch.float64)])
    assert bool(((state[1].double() - 0.1 * want).abs() <= 0.1 * off * size).all())
    mean = float((torch.clamp(z, min=0) + torch.log1p(torch.exp(-z.abs())) - y * z).mean())
    assert abs(float(loss) - mean) <= dz + 4 * 2.0 ** -24 * mean


def test_weights_of_very_different_size_in_one_vector(spr):
    """The 32 weights of a block share a unit: the small ones beside a large one are held to 2^-23 of the large one, so a
    logit is off by at most sum_j |s_j| 2^-23 max|w| beside its fp32 roundings."""
    N, d = 64, 64
    g = torch.Generator().manual_seed(2)
    S = torch.randn((N, d), generator=g).to(torch.bfloat16)
    packed = spr.hidden_pack8(S.cuda())
    Sn = unpack_ref(packed.cpu().numpy(), d)
    theta = torch.randn(d + 1, generator=g) * torch.logspace(-6, 1, d + 1)[torch.randperm(d + 1, generator=g)]
    theta[5], theta[20] = 0.0, 1e-30
    th = theta.double().numpy()
    z = Sn @ th[:d] + th[d]
    y = (z > 0).astype(np.uint8)
    st = [theta.cuda(), torch.zeros(d + 1, device="cuda"), torch.zeros(d + 1, device="cuda")]
    loss = float(spr.verifier_train_step8(packed, d, torch.from_numpy(y).cuda(), *st, 1, 0.01, step_ws(spr, d)))
    want, _ = training.bce_loss_and_grad(Sn, y, th)
    top = np.abs(th[:d]).reshape(-1, 32).max(1).repeat(32)
    off = np.mean(np.abs(Sn) @ top) * 2.0 ** -23 + 2.0 ** -24 * 24 * np.mean(np.abs(Sn) @ np.abs(th[:d]) + abs(th[d]))
    assert abs(loss - want) <= off + 2.0 ** -22 * want


def test_widths_that_are_refused(spr):
    for d in (8, 40, 4112, 8192):
        packed = torch.zeros((4, spr.pack8_pitch(d)), dtype=torch.uint8, device="cuda")
        z = torch.zeros(d + 1, device="cuda")
        with pytest.raises(spr.SprinterError) as e:
            spr.verifier_train_step8(packed, d, torch.zeros(4, dtype=torch.uint8, device="cuda"), z, z.clone(), z.clone(), 1,
                                     0.01, step_ws(spr, d))
        assert e.value.status == 2


def test_states_labelled_packed_fitted_and_used(spr):
    """A run as it would be used: draft and target heads label the draft's tokens, the draft's states are
    packed, the verifier is fitted on them, and sprinter_verify scores with the fitted weights."""
    g = torch.Generator().manual_seed(3)
    N, d, V = 4096, 256, 2000
    qh = torch.randn((N, d), generator=g).to(torch.bfloat16).cuda()
    qw = (torch.randn((V, d), generator=g) * (3.0 / d ** 0.5)).to(torch.bfloat16).cuda()
    pw = (qw.float().cpu() + torch.randn((V, d), generator=g) * (1.0 / d ** 0.5)).to(torch.bfloat16).cuda()
    x = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
    wl = spr.Workspace(spr.workspace_bytes(spr.OP_VERIFIER_LABELS_HEAD, N, 1, V, d, d, spr.BF16))
    labels, ratio = spr.verifier_labels_head(qh, pw, qh, qw, x, [1.0], wl)
    assert wl.device_status() == 0
    packed = spr.hidden_pack8(qh)
    ws = step_ws(spr, d)
    theta, m, v = (torch.zeros(d + 1, device="cuda") for _ in range(3))
    losses = [float(spr.verifier_train_step8(packed, d, labels[0].contiguous(), theta, m, v, t, 0.05, ws)) for t in range(1, 5)]
    assert losses[0] == pytest.approx(np.log(2.0), rel=1e-6) and all(np.isfinite(losses))
    assert ws.device_status() == 0
    wv = spr.Workspace(spr.workspace_bytes(spr.binding.OP_SPRINTER_VERIFY, N // 8, 8, 1, d, 0, spr.BF16))
    scores, accept, first = spr.sprinter_verify(spr.hidden_unpack8(packed, d).view(N // 8, 8, d), theta[:d].to(torch.bfloat16),
                                                None, None, theta[d:].clone(), 0.5, wv)
    S = unpack_ref(packed.cpu().numpy(), d)
    z = S @ to_float(theta[:d].to(torch.bfloat16)) + float(theta[d])
    assert np.allclose(scores.cpu().numpy().reshape(-1), 1 / (1 + np.exp(-z)), rtol=1e-3)


def to_float(t):
    return t.cpu().double().numpy()


def framed(shape, dtype, fill=7):
    n = int(np.prod(shape))
    buf = torch.full((n + 128,), fill, device="cuda", dtype=dtype)
    return buf, buf[64:64 + n].view(shape)


def untouched(buf, fill=7):
    return bool((buf[:64] == fill).all()) and bool((buf[-64:] == fill).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 1), (3, 33), (5, 255), (7, 768), (130, 1000), (3, 2048)])
def test_nothing_is_written_beside_packed_and_unpacked_states(spr, N, d, dtype):
    x = values(N, d, dtype, seed=d).cuda()
    pb, p = framed((N, spr.pack8_pitch(d)), torch.uint8)
    spr.hidden_pack8(x, out=p)
    assert np.array_equal(p.cpu().numpy(), spr.hidden_pack8(x).cpu().numpy()) and untouched(pb)
    ub, u = framed((N, d), dtype)
    spr.hidden_unpack8(p, d, dtype=dtype, out=u)
    assert untouched(ub)


@pytest.mark.parametrize("N,d", [(1, 16), (33, 528), (500, 1040), (40, 2064)])
def test_nothing_is_written_beside_the_parameters(spr, N, d):
    S, y = teacher_problem(N, d, torch.bfloat16, seed=N)
    packed, ws = spr.hidden_pack8(S.cuda()), step_ws(spr, d)
    frames = [framed((d + 1,), torch.float32) for _ in range(3)] + [framed((1,), torch.float32)]
    for _, t in frames:
        t.zero_()
    spr.verifier_train_step8(packed, d, y.cuda(), frames[0][1], frames[1][1], frames[2][1], 1, 0.01, ws, loss=frames[3][1])
    assert all(untouched(b) for b, _ in frames) and float(frames[3][1]) == pytest.approx(np.log(2.0), rel=1e-6)


@pytest.mark.parametrize("d", [32, 96, 40], ids=lambda d: f"d{d}")
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_every_exponent_is_packed_and_unpacked_exactly(spr, dtype, d):
    """A row for each exponent that packing gives, -126 to 121, of numbers q 2^e with |q| <= 127 and a largest one of 64
    and more: nothing is rounded either way, through whole rows of blocks (d = 32, 96) and through the form for any width."""
    e = torch.arange(-126, 122).repeat_interleave(2)
    g = torch.Generator().manual_seed(d)
    q = torch.randint(-127, 128, (len(e), d), generator=g)
    q[:, ::32] = torch.where(torch.rand(q[:, ::32].shape, generator=g) < 0.5, -1, 1) * torch.randint(64, 128, q[:, ::32].shape, generator=g)
    q[:, 1::32] = 0
    x = torch.ldexp(q.double(), e[:, None].double())
    assert bool(x.isfinite().all()) and torch.equal(x.to(dtype).double(), x)
    packed = spr.hidden_pack8(x.to(dtype).cuda())
    assert np.array_equal(packed.cpu().numpy(), pack_ref(x.numpy()))
    assert torch.equal(packed[:, d].cpu().view(torch.int8), e.to(torch.int8))
    for ty in (torch.float32, torch.bfloat16):
        assert torch.equal(spr.hidden_unpack8(packed, d, ty).cpu().double(), x)


def test_all_of_the_extremes_come_back(spr):
    """The largest and smallest numbers of either type beside infinities and NaN: every element as its bytes say."""
    big = torch.finfo(torch.float32).max
    x = torch.zeros((6, 64))
    x[0, :3], x[1, 40:42], x[2, 5] = torch.tensor([big, -big, big / 2]), torch.tensor([2.0 ** 111, -1.0]), 2.0 ** -149
    x[3, 7], x[4, 33], x[5] = float("inf"), float("nan"), -2.0 ** 127
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype)
        packed = spr.hidden_pack8(y.cuda())
        want = pack_ref(y.double().numpy())
        assert np.array_equal(packed.cpu().numpy(), want)
        for ty in (torch.float32, torch.bfloat16):
            assert np.array_equal(spr.hidden_unpack8(packed, 64, ty).cpu().double().numpy(), unpack_ref(want, 64), equal_nan=True)


@pytest.mark.parametrize("factor", [10, 14, 18], ids=lambda f: f"2^{f}")
@pytest.mark.parametrize("N,d", [(96, 64), (130, 512), (96, 528), (200, 1040), (70, 2048), (100, 2064)])
def test_one_column_far_above_the_rest_costs_the_others_nothing(spr, N, d, factor):
    """In every sixteenth row one column is 2^factor times the others, as some channels of a model's states are, and those
    rows' residuals are near 1 while most others' are small.  The block's other bytes are zero in those rows, so the large
    numbers have no part in the other columns, and each column is held to its own terms:
      r      a logit's terms are added up in fp32 in runs of at most 8 blocks and 16 parts: off by dz = 30 2^-24 sum_j |s_ij w_j|,
             so r by dz / 4 and two roundings of its own
      r 2^e  in 46 bits relative to the largest of a tile: 2^-46 max_i 2^e_i |q_ij|
      sums   a rounding for each of at most two tiles and four more, 6 2^-24 of sum_i |r_i s_ij|
    m = 0.1 grad, rounded once more."""
    g = torch.Generator().manual_seed(N + d + factor)
    hot, col = torch.arange(3, N, 16), d // 2 + 5
    S = torch.randn((N, d), generator=g)
    w = 4.0 * torch.randn(d + 1, generator=g) / d ** 0.5
    S[hot, col] = 2.0 ** factor * (1 + torch.rand(len(hot), generator=g))
    w[col] = 2.0 ** -factor
    packed = spr.hidden_pack8(S.to(torch.bfloat16).cuda())
    X = torch.from_numpy(unpack_ref(packed.cpu().numpy(), d))
    z = X @ w[:d].double() + w[d].double()
    y = z > 0
    y[hot] = ~y[hot]
    r = torch.sigmoid(z) - y.double()
    ws = step_ws(spr, d)
    state = [w.cuda(), torch.zeros(d + 1, device="cuda"), torch.zeros(d + 1, device="cuda")]
    spr.verifier_train_step8(packed, d, y.to(torch.uint8).cuda(), *state, 1, 0.01, ws)
    assert ws.device_status() == 0
    u, A = 2.0 ** -24, X.abs()
    dz = 30 * u * (A @ w[:d].abs().double() + w[d].abs().double())
    dr = dz / 4 + 2 * u
    e = packed.cpu().view(torch.int8)[:, d:d + (d + 31) // 32].double().repeat_interleave(32, 1)[:, :d]
    q = packed.cpu().view(torch.int8)[:, :d].double().abs()
    tol = (A * dr[:, None]).mean(0) + 2.0 ** -46 * torch.exp2(e).amax(0) * q.mean(0) + 7 * u * (A * r.abs()[:, None]).mean(0)
    off = (state[1][:d].cpu().double() - 0.1 * (X * r[:, None]).mean(0)).abs()
    assert bool((off <= 0.1 * tol + 1e-45).all()), float((off / (0.1 * tol + 1e-45)).max())


@pytest.mark.parametrize("factor", [10, 16, 24], ids=lambda f: f"2^{f}")
@pytest.mark.parametrize("d", [64, 512, 1040, 2064])
def test_one_weight_far_above_the_rest_costs_the_others_nothing(spr, d, factor):
    """A weight 2^factor times the others of its block, in a column where the state is zero: the logit, seen through the loss
    of a single row (1 at most per unit of it), keeps what fp32 products keep: 30 2^-24 of its terms, and the weights
    46 bits relative to the largest, 2^-46 2^factor sum_j |s_j|, beside four roundings of the loss."""
    g = torch.Generator().manual_seed(d + factor)
    for _ in range(8):
        w = torch.randn(d + 1, generator=g) / d ** 0.5
        s = torch.randn((1, d), generator=g)
        w[d // 2 + 3], s[0, d // 2 + 3] = 2.0 ** factor, 0.0
        packed = spr.hidden_pack8(s.to(torch.bfloat16).cuda())
        x = torch.from_numpy(unpack_ref(packed.cpu().numpy(), d))[0]
        z = float(x @ w[:d].double() + w[d].double())
        state = [w.cuda(), torch.zeros(d + 1, device="cuda"), torch.zeros(d + 1, device="cuda")]
        loss = float(spr.verifier_train_step8(packed, d, torch.ones(1, dtype=torch.uint8).cuda(), *state, 1, 0.01, step_ws(spr, d)))
        want = np.log1p(np.exp(-z))
        terms = float((x * w[:d].double()).abs().sum() + w[d].double().abs())
        assert abs(loss - want) <= 30 * 2.0 ** -24 * terms + 2.0 ** (factor - 46) * float(x.abs().sum()) + 4 * 2.0 ** -24 * want


def test_a_step_on_no_samples_says_so(spr):
    """The mean loss of nothing is not a number, and nothing is stepped."""
    d = 64
    state = [torch.rand(d + 1, device="cuda") for _ in range(3)]
    before = [x.clone() for x in state]
    packed, y = (torch.empty(shape, dtype=torch.uint8, device="cuda") for shape in ((0, spr.pack8_pitch(d)), (0,)))
    ws = step_ws(spr, d)
    loss = torch.full((1,), 7.0, device="cuda")
    assert bool(spr.verifier_train_step8(packed, d, y, *state, 1, 0.01, ws, loss=loss).isnan().all())
    assert all(torch.equal(a, b) for a, b in zip(state, before)) and ws.device_status() == 0
