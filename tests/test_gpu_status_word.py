"""A wait that runs out inside a kernel shows in the status word and in the outputs whatever the word held before.

The word is sticky: a bad token of an earlier call may still stand there, unread, or be found earlier in the same call.
The waits are made to run out by the test hooks, which load nothing and give up after a few thousand polls."""
import pytest
import torch

import test_gpu_fit
import test_gpu_verifier_shapes

pytestmark = pytest.mark.gpu
TIMEOUT, BAD_TOKEN = 5, 6


@pytest.fixture(scope="module")
def spr():
    import paper_2502_04557_b200 as s
    s.lib()
    return s


@pytest.fixture
def nothing_loaded(spr):
    """Switches the loads of the head's products off for as long as it is called with True."""
    yield lambda on: spr.lib().spr_test_pair_kernels(1 if on else 0, 4000 if on else 0)
    spr.lib().spr_test_pair_kernels(0, 0)


def head(N=300, d=200, V=2001, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(N + d)
    h, w = torch.randn((N, d), generator=g).to(dtype).cuda(), (torch.randn((V, d), generator=g) * 0.2).to(dtype).cuda()
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
    return h, w, t


def head_bytes(spr, h, w):
    code = spr.F32 if h.dtype == torch.float32 else spr.BF16
    return max(spr.workspace_bytes(op, h.shape[0], 1, w.shape[0], h.shape[1], h.shape[1], code)
               for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD, spr.OP_VERIFIER_LABELS_HEAD))


def leave_a_bad_token(spr, ws):
    """A call with a target outside the vocabulary, whose status nobody reads."""
    h, w, t = head(64, 32, 100)
    t[3] = 100
    loss, _ = spr.head_loss(h, w, t, ws)
    assert float(loss[3]) == -1.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_head_calls(spr, dtype, nothing_loaded):
    h, w, t = head(dtype=dtype)
    ws = spr.Workspace(head_bytes(spr, h, w))
    want = spr.head_loss(h, w, t, ws) + spr.verifier_labels_head(h, w, h, w, t, [1.5], ws)
    assert ws.device_status() == 0
    for call in ("loss", "labels"):
        leave_a_bad_token(spr, ws)
        nothing_loaded(True)
        if call == "loss":
            loss, lse = spr.head_loss(h, w, t, ws)
            assert bool(loss.isnan().all()) and bool(lse.isnan().all())
        else:
            labels, ratio = spr.verifier_labels_head(h, w, h, w, t, [1.5], ws)
            assert not labels.any() and bool(ratio.isnan().all())
        nothing_loaded(False)
        assert ws.device_status() == TIMEOUT and ws.device_status() == 0
    again = spr.head_loss(h, w, t, ws) + spr.verifier_labels_head(h, w, h, w, t, [1.5], ws)
    assert ws.device_status() == 0 and all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_bad_target_of_the_same_call(spr, dtype, nothing_loaded):
    """head_loss_grad finds the target while it lays its operands out, before the products."""
    h, w, t = head(dtype=dtype)
    ws = spr.Workspace(head_bytes(spr, h, w))
    _, lse = spr.head_loss(h, w, t, ws)
    g = torch.full((len(t),), 0.01, device="cuda")
    t[5] = w.shape[0]
    spr.head_loss_grad(h, w, t, lse, g, ws)
    assert ws.device_status() == BAD_TOKEN
    nothing_loaded(True)
    spr.head_loss_grad(h, w, t, lse, g, ws)
    nothing_loaded(False)
    assert ws.device_status() == TIMEOUT and ws.device_status() == 0
    spr.head_loss_grad(h, w, t, lse, g, ws)
    assert ws.device_status() == BAD_TOKEN


@pytest.mark.parametrize("packed", [False, True], ids=["bf16", "packed"])
def test_steps_of_the_verifier(spr, packed):
    N, d = 5000, 768
    S, y = test_gpu_fit.teacher_problem(N, d, torch.bfloat16, seed=21)
    S, y = S.cuda(), y.cuda()
    h, w, _ = head(64, 32, 100)
    op = spr.OP_VERIFIER_TRAIN8 if packed else spr.binding.OP_VERIFIER_TRAIN
    ws = spr.Workspace(max(spr.workspace_bytes(op, 0, 0, 0, d, 0, spr.BF16), head_bytes(spr, h, w)))
    rows = spr.hidden_pack8(S) if packed else S

    def step(*state, **kw):
        if packed:
            return spr.verifier_train_step8(rows, d, y, *state, 3, 0.01, ws, **kw)
        return spr.binding.verifier_train_step(rows, y, *state, 3, 0.01, ws, **kw)

    g = torch.Generator().manual_seed(22)
    state = [(0.05 * torch.randn(d + 1, generator=g)).cuda()] + [torch.rand(d + 1, generator=g).cuda() * 1e-3 for _ in range(2)]
    before, want = [x.clone() for x in state], [x.clone() for x in state]
    step(*want)
    assert ws.device_status() == 0
    leave_a_bad_token(spr, ws)
    loss = step(*state, test_flags=1, spin_limit=4000)
    assert bool(loss.isnan().all()) and all(torch.equal(a, b) for a, b in zip(state, before))
    assert ws.device_status() == TIMEOUT and ws.device_status() == 0
    step(*state)
    assert ws.device_status() == 0 and all(torch.equal(a, b) for a, b in zip(state, want))


def test_the_verifier(spr):
    (B, K, d, h), shape = (40, 8, 512, 256), dict(bm=64, bn=64, splits=4, cluster_n=1)
    args, _ = test_gpu_verifier_shapes.problem(B, K, d, h)
    hh, w, _ = head(64, 32, 100)
    ws = spr.Workspace(max(spr.workspace_bytes(0, B, K, 1, d, h, spr.BF16), head_bytes(spr, hh, w)))
    want = spr.binding.sprinter_verify_shaped(*args, ws, **shape)
    assert ws.device_status() == 0
    leave_a_bad_token(spr, ws)
    scores, accept, first = spr.binding.sprinter_verify_shaped(*args, ws, flags=1, spin_limit=4000, **shape)
    assert bool((scores == -1).all()) and not accept.any() and bool((first == -1).all())
    assert ws.device_status() == TIMEOUT and ws.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(spr.binding.sprinter_verify_shaped(*args, ws, **shape), want))
