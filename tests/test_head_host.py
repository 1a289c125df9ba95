"""CPU-side checks of the vocabulary head's loss, its gradient and labels, and of the 8-bit hidden states: sizes,
types, pointers and workspaces are refused on the host, before any device call."""
import ctypes
import os
import re

import pytest
import torch

import paper_2502_04557_b200 as spr
from paper_2502_04557_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40          # a workspace size that never is the reason


@pytest.fixture(scope="module")
def mem():
    """Addresses that stand for tensors and are never read: 256-byte aligned, and off by 1, 4 and 8 bytes."""
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 255) // 256 * 256
    yield buf, a, a + 1, a + 4, a + 8


def loss(L, p, **kw):
    a = dict(hidden=p, W=p, targets=p, N=3, d=8, V=16, dt=1, loss=p, lse=p, ws=p, n=BIG)
    a.update(kw)
    return L.head_loss(a["hidden"], a["W"], a["targets"], a["N"], a["d"], a["V"], a["dt"], a["loss"], a["lse"], a["ws"], a["n"], None)


def grad(L, p, **kw):
    a = dict(hidden=p, W=p, targets=p, lse=p, g=p, N=3, d=8, V=16, dt=1, dh=p, dW=p, ws=p, n=BIG)
    a.update(kw)
    return L.head_loss_grad(a["hidden"], a["W"], a["targets"], a["lse"], a["g"], a["N"], a["d"], a["V"], a["dt"], a["dh"], a["dW"],
                            a["ws"], a["n"], None)


def labels(L, p, **kw):
    lam = (ctypes.c_float * 8)(*[1.0] * 8)
    a = dict(ph=p, pW=p, dp=8, qh=p, qW=p, dq=8, x=p, N=3, V=16, dt=1, lam=lam, n_lambda=2, labels=p, ratio=p, ws=p, n=BIG)
    a.update(kw)
    return L.verifier_labels_head(a["ph"], a["pW"], a["dp"], a["qh"], a["qW"], a["dq"], a["x"], a["N"], a["V"], a["dt"], a["lam"],
                                  a["n_lambda"], a["labels"], a["ratio"], a["ws"], a["n"], None)


def step(L, p, **kw):
    a = dict(packed=p, y=p, N=3, d=16, theta=p, m=p, v=p, t=1, lr=0.01, b1=0.9, b2=0.999, eps=1e-8, loss=None, ws=p, n=BIG)
    a.update(kw)
    return L.verifier_train_step8(a["packed"], a["y"], a["N"], a["d"], a["theta"], a["m"], a["v"], a["t"], a["lr"], a["b1"], a["b2"],
                                  a["eps"], a["loss"], a["ws"], a["n"], None)


def small(op, N, V, d, h=0, dt=1):
    """A little less than the call asks for (sizes are rounded up by some blocks of 256 bytes)."""
    n = spr.workspace_bytes(op, N, 1, V, d, h, dt)
    assert n > 256 and n % 256 == 0
    return n - 2048 if n > 4096 else 256


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "sprinter.h")).read()
    enum = dict((k, int(v)) for k, v in re.findall(r"\b(SPR_[A-Z0-9_]+)\s*=\s*(\d+)", text))
    for name in ("HEAD_LOSS", "HEAD_LOSS_GRAD", "VERIFIER_LABELS_HEAD", "VERIFIER_TRAIN8"):
        assert enum["SPR_OP_" + name] == getattr(binding, "OP_" + name) == getattr(spr, "OP_" + name), name
    ops = [v for k, v in enum.items() if k.startswith("SPR_OP_")]
    assert len(set(ops)) == len(ops)


@pytest.mark.parametrize("call,tensors,optional", [
    (loss, {"hidden": 16, "W": 16, "targets": 4, "loss": 4}, {"lse": 4}),
    (grad, {"hidden": 16, "W": 16, "targets": 4, "lse": 4, "g": 4}, {"dh": 16, "dW": 16}),
    (labels, {"ph": 16, "pW": 16, "qh": 16, "qW": 16, "x": 4, "labels": 1}, {"ratio": 4}),
    (step, {"packed": 16, "y": 1, "theta": 4, "m": 4, "v": 4}, {"loss": 4}),
])
def test_pointers_are_checked(mem, call, tensors, optional):
    L, (_, p, by1, by4, by8) = spr.lib(), mem
    for name, align in tensors.items():
        assert call(L, p, **{name: None}) == INVALID, name
    for name, align in {**tensors, **optional}.items():
        if align > 1:
            assert call(L, p, **{name: by1}) == INVALID, name
        if align == 16:
            assert call(L, p, **{name: by4}) == INVALID and call(L, p, **{name: by8}) == INVALID, name
    assert call(L, p, ws=None) == WORKSPACE
    assert call(L, p, ws=p + 16) == WORKSPACE
    assert call(L, p, n=16) == WORKSPACE


def test_gradients_wanted(mem):
    L, (_, p, by1, by4, by8) = spr.lib(), mem
    assert grad(L, p, dh=None, dW=None) == INVALID
    assert grad(L, p, dh=None, n=16) == WORKSPACE and grad(L, p, dW=None, n=16) == WORKSPACE


@pytest.mark.parametrize("call,dims", [(loss, ("d", "V")), (grad, ("d", "V")), (labels, ("dp", "dq", "V"))])
def test_head_sizes_are_checked(mem, call, dims):
    L, p = spr.lib(), mem[1]
    assert call(L, p, N=-1) == INVALID
    for name in dims:
        for n in (0, -5, (1 << 20) + 1 if name != "V" else (1 << 30) + 1):
            assert call(L, p, **{name: n}) == INVALID, (name, n)
    for dt in (-1, 2, 7):
        assert call(L, p, dt=dt) == UNSUPPORTED


def test_thresholds_are_checked(mem):
    L, p = spr.lib(), mem[1]
    for n in (-1, 0, 9):
        assert labels(L, p, n_lambda=n) == INVALID
    assert labels(L, p, lam=None) == INVALID


def test_step_arguments_are_checked(mem):
    L, p = spr.lib(), mem[1]
    nan, inf = float("nan"), float("inf")
    for bad in (dict(t=0), dict(t=-3), dict(N=-1), dict(d=0), dict(d=-16), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0),
                dict(b2=nan), dict(b2=inf), dict(eps=-1e-9), dict(eps=nan), dict(lr=nan)):
        assert step(L, p, **bad) == INVALID, bad
    for bad in (dict(d=8), dict(d=40), dict(d=4112), dict(N=0x7fff0001)):
        assert step(L, p, **bad) == UNSUPPORTED, bad
    # the test hook takes no flags but its own
    assert L.spr_test_verifier_train_step8(p, p, 3, 16, p, p, p, 1, 0.01, 0.9, 0.999, 1e-8, None, p, BIG, None, 64, 0) == INVALID


def test_nothing_to_do(mem):
    """Empty calls touch nothing, pointers included."""
    L, p = spr.lib(), mem[1]
    assert loss(L, p, N=0, hidden=None, W=None, targets=None, loss=None, lse=None, ws=None, n=0) == OK
    assert grad(L, p, N=0, hidden=None, W=None, targets=None, lse=None, g=None, dW=None, ws=None, n=0) == OK
    assert labels(L, p, N=0, ph=None, pW=None, qh=None, qW=None, x=None, labels=None, ratio=None, ws=None, n=0) == OK
    assert step(L, p, N=0, packed=None, y=None, theta=None, m=None, v=None, ws=None, n=0) == OK
    assert L.hidden_pack8(None, 0, 16, 1, None, None) == OK and L.hidden_unpack8(None, 0, 16, 1, None, None) == OK


def test_pack_arguments_are_checked(mem):
    L, (_, p, by1, by4, by8) = spr.lib(), mem
    # (packed is 16-byte aligned, hidden as its elements are)
    assert L.hidden_pack8(p, 3, 16, 2, p, None) == UNSUPPORTED and L.hidden_unpack8(p, 3, 16, 2, p, None) == UNSUPPORTED
    for d in (0, -1, (1 << 20) + 1):
        assert L.hidden_pack8(p, 3, d, 1, p, None) == INVALID and L.hidden_unpack8(p, 3, d, 1, p, None) == INVALID
    assert L.hidden_pack8(p, -1, 16, 1, p, None) == INVALID and L.hidden_unpack8(p, -1, 16, 1, p, None) == INVALID
    assert L.hidden_pack8(None, 3, 16, 1, p, None) == INVALID and L.hidden_pack8(p, 3, 16, 1, None, None) == INVALID
    assert L.hidden_unpack8(None, 3, 16, 1, p, None) == INVALID and L.hidden_unpack8(p, 3, 16, 1, None, None) == INVALID
    assert L.hidden_pack8(by1, 3, 16, 1, p, None) == INVALID and L.hidden_pack8(p + 2, 3, 16, 0, p, None) == INVALID
    assert L.hidden_unpack8(p, 3, 16, 1, by1, None) == INVALID
    for off in (by1, by4, by8):
        assert L.hidden_pack8(p, 3, 16, 1, off, None) == INVALID and L.hidden_unpack8(off, 3, 16, 1, p, None) == INVALID


def test_pitch_of_a_packed_row():
    for d in (1, 15, 16, 31, 32, 33, 255, 768, 1000, 2048, 4096, 1 << 20):
        blocks = -(-d // 32)
        n = spr.pack8_pitch(d)
        assert n % 16 == 0 and d + blocks <= n < d + blocks + 16
    assert [spr.pack8_pitch(d) for d in (0, -1, (1 << 20) + 1)] == [0, 0, 0]
    assert spr.pack8_pitch(2048) == 2112


def test_workspace_sizes():
    wb = spr.workspace_bytes
    for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD):
        assert wb(op, 0, 1, 100, 64, 0, 1) == wb(op, 4, 0, 100, 64, 0, 1) == wb(op, 4, 1, 0, 64, 0, 1) == wb(op, 4, 1, 100, 0, 0, 1) == 0
        assert wb(op, 4, 1, 100, 64, 0, 5) == 0 and wb(op, -1, 1, 100, 64, 0, 1) == 0
        assert wb(op, 64, 2, 1000, 64, 0, 1) == wb(op, 128, 1, 1000, 64, 0, 1)          # B K rows
    assert wb(spr.OP_VERIFIER_LABELS_HEAD, 4, 1, 100, 64, 0, 1) == 0                    # the second width is missing
    assert wb(spr.OP_VERIFIER_LABELS_HEAD, 4, 1, 100, 64, 64, 1) > 0
    assert wb(spr.OP_VERIFIER_TRAIN8, 0, 0, 0, 768, 0, 1) >= 592 * 770 * 4 and wb(spr.OP_VERIFIER_TRAIN8, 0, 0, 0, 0, 0, 1) == 0
    # no logits are kept: the loss needs two floats per row and 128 columns, the gradient one piece of the vocabulary at a time
    N, V, d = 4096, 128256, 2048
    assert wb(spr.OP_HEAD_LOSS, N, 1, V, d, 0, 1) < N * V // 8
    assert wb(spr.OP_HEAD_LOSS_GRAD, N, 1, V, d, 0, 1) < N * V
    a, b = (wb(spr.OP_HEAD_LOSS_GRAD, N, 1, V, d, 0, 1), wb(spr.OP_HEAD_LOSS_GRAD, N, 1, 4 * V, d, 0, 1))
    assert b < a + (64 << 20)


@pytest.mark.parametrize("N,d,V,dt", [(4, 256, 1000, 0), (3, 8, 16, 1), (256, 768, 50257, 1), (67, 257, 1003, 0), (300, 100, 5000, 1),
                                      (1, 2048, 32000, 1), (8, 2048, 32000, 0), (100, 512, 30000, 0)])
def test_a_short_workspace_is_refused(mem, N, d, V, dt):
    L, p = spr.lib(), mem[1]
    assert loss(L, p, N=N, d=d, V=V, dt=dt, n=small(spr.OP_HEAD_LOSS, N, V, d, 0, dt)) == WORKSPACE
    assert grad(L, p, N=N, d=d, V=V, dt=dt, n=small(spr.OP_HEAD_LOSS_GRAD, N, V, d, 0, dt)) == WORKSPACE
    assert labels(L, p, N=N, dp=d, dq=2 * d, V=V, dt=dt, n=small(spr.OP_VERIFIER_LABELS_HEAD, N, V, d, 2 * d, dt)) == WORKSPACE


@pytest.mark.parametrize("d", [16, 768, 4096])
def test_a_short_step_workspace_is_refused(mem, d):
    L, p = spr.lib(), mem[1]
    assert step(L, p, d=d, n=small(spr.OP_VERIFIER_TRAIN8, 0, 0, d)) == WORKSPACE


def test_binding_refuses_host_tensors_types_and_shapes():
    h, W, t = torch.zeros(3, 8), torch.zeros(16, 8), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="hidden must be a CUDA tensor"):
        binding._head(0, h, W, t)
    with pytest.raises(TypeError, match="element type"):
        binding._head(0, h.half(), W.half(), t)
    with pytest.raises(ValueError, match="packed must be a CUDA tensor"):
        binding._packed(0, torch.zeros(3, 32, dtype=torch.uint8), 16)
    # a host tensor has the device index -1: with it the checks behind the device check are reached
    with pytest.raises(TypeError, match="W must be"):
        binding._head(-1, h, W.bfloat16(), t)
    with pytest.raises(TypeError, match="targets must be"):
        binding._head(-1, h, W, t.long())
    with pytest.raises(ValueError, match="contiguous"):
        binding._head(-1, torch.zeros(3, 16)[:, ::2], W, t)
    with pytest.raises(ValueError, match=r"\[N,d\] and W \[V,d\]"):
        binding._head(-1, h, torch.zeros(16, 9), t)
    with pytest.raises(ValueError, match=r"\[N,d\] and W \[V,d\]"):
        binding._head(-1, torch.zeros(1, 3, 8), W, t)
    with pytest.raises(ValueError, match="one entry per hidden state"):
        binding._head(-1, h, W, t[:2])
    assert binding._head(-1, h, W, t)[:3] == (3, 8, 16)
    for bad, d in ((torch.zeros(3, 16, dtype=torch.uint8), 16), (torch.zeros(32, dtype=torch.uint8), 16),
                   (torch.zeros(3, 32, dtype=torch.uint8), 0)):
        with pytest.raises(ValueError, match="packed must be"):
            binding._packed(-1, bad, d)
    with pytest.raises(TypeError, match="packed must be"):
        binding._packed(-1, torch.zeros(3, 32, dtype=torch.int8), 16)
    out = torch.zeros(3)
    assert binding._result(-1, out, (3,), torch.float32, "loss")[0] is out
    with pytest.raises(ValueError, match=r"loss must be \(4,\)"):
        binding._result(-1, out, (4,), torch.float32, "loss")
    with pytest.raises(TypeError, match="loss must be"):
        binding._result(-1, out.double(), (3,), torch.float32, "loss")


@pytest.mark.parametrize("dt", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("d,V", [(768, 50257), (2048, 32000), (100, 5000), (64, 1003), (520, 32300), (257, 1003), (8, 9), (4104, 700),
                                 (64, 128256), (1024, 300000), (136, 1000000), (30000, 2000)])
def test_workspace_sizes_do_not_fall_as_tokens_are_added(d, V, dt):
    """A workspace for the largest batch is one for every smaller batch: what follows from sizes that never fall, as each size
    is at least what the call of that size takes."""
    counts = sorted({*range(1, 700), *(256 * m + k for m in range(1, 80) for k in (-1, 0, 1)), *(2 ** b + k for b in range(9, 19) for k in (-1, 0, 1)),
                     *(int(700 * 1.07 ** i) for i in range(90))})
    for op in (spr.OP_HEAD_LOSS, spr.OP_HEAD_LOSS_GRAD, spr.OP_VERIFIER_LABELS_HEAD):
        sizes = [spr.workspace_bytes(op, n, 1, V, d, max(8, d // 2), dt) for n in counts]
        falls = [(n, a, b) for n, a, b in zip(counts[1:], sizes, sizes[1:]) if b < a]
        assert not falls, (op, falls[:3])


def test_binding_refuses_sizes_that_do_not_fit_32_bits():
    """N, d and V travel as 32-bit integers: 2^32 + 3 rows must not be taken for three.  (Tensors without storage.)"""
    def meta(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="meta")
    big = (1 << 32) + 3
    for h, W, t in ((meta(big, 8), meta(16, 8), meta(big, dtype=torch.int32)), (meta(3, 8), meta(big, 8), meta(3, dtype=torch.int32)),
                    (meta(3, big), meta(16, big), meta(3, dtype=torch.int32)), (meta(1 << 31, 8), meta(16, 8), meta(1 << 31, dtype=torch.int32))):
        with pytest.raises(ValueError, match="below 2\\^31"):
            binding._head(-1, h, W, t)
    d = (1 << 32) + 32
    with pytest.raises(ValueError, match="at most 2\\^20"):
        binding._packed(-1, meta(2, (d + d // 32 + 15) // 16 * 16, dtype=torch.uint8), d)
    for d in (d, (1 << 20) + 1):
        with pytest.raises(ValueError, match="at most 2\\^20"):
            binding._rows(meta(2, d))
    assert binding._rows(meta(2, 1 << 20)) == (2, 1 << 20) and binding._head(-1, meta(3, 8), meta(16, 8), meta(3, dtype=torch.int32))[:3] == (3, 8, 16)
