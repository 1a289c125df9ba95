"""CPU-side checks of cache_append, tree_attention and logits_rules: sizes, types, pointers and workspaces are refused on the
host, before any device call."""
import ctypes
import math
import struct
import os
import re

import pytest
import torch

import draft_pass_reference as ref
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


def append(L, p, **kw):
    a = dict(q=p, qs=64, k=p, ks=32, v=p, vs=32, B=2, T=3, Hq=4, Hkv=2, D=16, dt=1, lens=p, counts=p, parents=p, slots=p, f=p, rot=16,
             inter=0, table=p, max_pages=4, pages=9, page=16, kc=p, vc=p, qo=p, ws=p, n=BIG)
    a.update(kw)
    return L.cache_append(*a.values(), None)


def attend(L, p, **kw):
    a = dict(q=p, kc=p, vc=p, B=2, T=3, Hq=4, Hkv=2, D=64, dt=1, lens=p, counts=p, parents=p, table=p, max_pages=4, pages=9, page=16,
             scale=0.125, out=p, ws=p, n=BIG)
    a.update(kw)
    return L.tree_attention(*a.values(), None)


def rules(L, p, **kw):
    a = dict(l=p, ldv=100, V=100, B=2, T=3, dt=1, h=p, ldh=8, hl=p, tok=p, parents=p, counts=p, pen=p, bt=p, bv=p, nb=2, masks=p, ldm=4,
             nm=3, mr=p, out=p, ldo=100, ws=p, n=BIG)
    a.update(kw)
    return L.logits_rules(*a.values(), None)


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "sprinter.h")).read()
    enum = dict((k, int(v)) for k, v in re.findall(r"\b(SPR_[A-Z0-9_]+)\s*=\s*(\d+)", text))
    for name in ("CACHE_APPEND", "TREE_ATTENTION", "LOGITS_RULES"):
        assert enum["SPR_OP_" + name] == getattr(binding, "OP_" + name) == getattr(spr, "OP_" + name), name
    for group in ("SPR_OP_", "SPR_ERR_"):
        codes = [v for k, v in enum.items() if k.startswith(group)]
        assert len(set(codes)) == len(codes)
    L = spr.lib()
    for name in ("BAD_PAGE", "BAD_TREE"):
        assert L.spr_status_string(enum["SPR_ERR_" + name]) != L.spr_status_string(99)


def test_workspaces():
    for op in (spr.OP_CACHE_APPEND, spr.OP_LOGITS_RULES):
        assert spr.workspace_bytes(op, 1000, 64, 128256, 128, 32, spr.F32) == 256
    for dt in (spr.F32, spr.BF16):
        a, b = (spr.workspace_bytes(spr.OP_TREE_ATTENTION, 1, 1, 1, d, 0, dt) for d in (64, 128))
        assert 256 < a < b and b == spr.workspace_bytes(spr.OP_TREE_ATTENTION, 500, 256, 1, 128, 64, dt)
    assert spr.workspace_bytes(spr.OP_TREE_ATTENTION, 1, 1, 1, 136, 0, spr.BF16) == 0
    assert spr.workspace_bytes(spr.OP_TREE_ATTENTION, 1, 1, 1, 0, 0, spr.BF16) == 0


@pytest.mark.parametrize("call,tensors,optional", [
    (append, {"k": 2, "v": 2, "lens": 4, "table": 4, "kc": 2, "vc": 2, "f": 4, "q": 2, "qo": 2}, {"counts": 4, "parents": 4, "slots": 4}),
    (attend, {"q": 16, "kc": 16, "vc": 16, "lens": 4, "table": 4, "out": 16}, {"counts": 4, "parents": 4}),
    (rules, {"l": 2, "out": 2, "hl": 4, "bt": 4, "bv": 4, "mr": 4}, {"h": 4, "tok": 4, "parents": 4, "counts": 4, "pen": 4, "masks": 4}),
])
def test_pointers_are_checked(mem, call, tensors, optional):
    L, (_, p, by1, by4, by8) = spr.lib(), mem
    for name in tensors:
        assert call(L, p, **{name: None}) == INVALID, name
    for name, align in {**tensors, **optional}.items():
        assert call(L, p, **{name: by1}) == INVALID, name
        if align == 16:
            assert call(L, p, **{name: by4}) == INVALID and call(L, p, **{name: by8}) == INVALID, name
    assert call(L, p, ws=None) == WORKSPACE
    assert call(L, p, ws=p + 16) == WORKSPACE
    assert call(L, p, n=255) == WORKSPACE


@pytest.mark.parametrize("call", [append, attend, rules])
def test_types_and_batches_are_checked(mem, call):
    L, p = spr.lib(), mem[1]
    for dt in (-1, 2, 7):
        assert call(L, p, dt=dt) == UNSUPPORTED
    assert call(L, p, B=-1) == INVALID and call(L, p, T=-1) == INVALID
    assert call(L, p, B=1 << 24, T=1 << 7) == INVALID
    assert call(L, p, T=257) == UNSUPPORTED                   # a tree, for cache_append


def test_append_arguments_are_checked(mem):
    L, p = spr.lib(), mem[1]
    for bad in (dict(Hkv=0), dict(Hkv=-1), dict(Hq=-1), dict(Hq=0), dict(D=0), dict(D=-16), dict(D=1026), dict(rot=-2), dict(rot=3), dict(rot=18),
                dict(max_pages=0), dict(pages=0), dict(page=0), dict(page=-16), dict(ks=31), dict(vs=31), dict(qs=63), dict(ks=-32)):
        assert append(L, p, **bad) == INVALID, bad
    assert append(L, p, q=None) == INVALID and append(L, p, qo=None) == INVALID


def test_attention_arguments_are_checked(mem):
    L, p = spr.lib(), mem[1]
    for bad in (dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(D=0), dict(D=-8), dict(max_pages=0), dict(pages=0), dict(page=0),
                dict(scale=math.inf), dict(scale=math.nan)):
        assert attend(L, p, **bad) == INVALID, bad
    for bad in (dict(D=12), dict(D=136), dict(page=4), dict(page=20), dict(pages=1 << 27)):
        assert attend(L, p, **bad) == UNSUPPORTED, bad
    # tiles of 64 keys that could pass 2^31: 2^15 sequences of 2 heads with tables of 2^17 pages
    assert attend(L, p, B=1 << 15, max_pages=1 << 17) == UNSUPPORTED
    n = spr.workspace_bytes(spr.OP_TREE_ATTENTION, 2, 3, 1, 64, 0, spr.BF16)
    assert attend(L, p, T=64, n=n // 8) == WORKSPACE


def test_rules_arguments_are_checked(mem):
    L, p = spr.lib(), mem[1]
    for bad in (dict(V=0), dict(V=-5), dict(V=(1 << 30) + 1, ldv=1 << 31, ldo=1 << 31), dict(ldv=99), dict(ldo=99), dict(ldo=101), dict(nb=-1), dict(nb=1025),
                dict(ldh=-1), dict(ldm=3), dict(nm=0), dict(nm=-1)):
        assert rules(L, p, **bad) == INVALID, bad


def test_arguments_in_an_array(mem):
    """Every argument arrives in its place: refusals and empty calls as those of the plain calls."""
    L, p = spr.lib(), mem[1]

    def call(op, f, real, **kw):
        got = []
        f(type("L", (), {"cache_append": lambda *a: got.extend(a[1:]), "tree_attention": lambda *a: got.extend(a[1:]),
                         "logits_rules": lambda *a: got.extend(a[1:])})(), p, **kw)
        fmt = "".join("d" if i == real else "q" for i in range(len(got)))
        return L.spr_draft_pass_call(op, struct.pack(fmt, *[0 if a is None else a for a in got]))

    for op, f, real, cases in (
            (spr.OP_CACHE_APPEND, append, None, (dict(Hq=0), dict(D=0), dict(rot=3), dict(page=0), dict(ks=31), dict(vs=31), dict(qs=63), dict(kc=0),
                                                 dict(vc=0), dict(table=0), dict(lens=0), dict(dt=7), dict(n=16), dict(ws=0), dict(B=0), dict(slots=p + 1))),
            (spr.OP_TREE_ATTENTION, attend, 16, (dict(Hq=3), dict(D=12), dict(page=20), dict(scale=math.nan), dict(out=0), dict(ws=0), dict(n=16),
                                                        dict(T=0), dict(table=0), dict(max_pages=0), dict(parents=p + 1))),
            (spr.OP_LOGITS_RULES, rules, None, (dict(V=0), dict(ldv=99), dict(ldo=99), dict(nb=1025), dict(ldh=-1), dict(ldm=3), dict(nm=0), dict(mr=0),
                                                dict(out=0), dict(ws=0), dict(n=16), dict(B=0), dict(pen=p + 1)))):
        for kw in cases:
            plain = f(L, p, **{k: v or None if k in ("kc", "vc", "table", "lens", "ws", "out", "mr") else v for k, v in kw.items()})
            assert call(op, f, real, **kw) == plain, (op, kw)
    assert L.spr_draft_pass_call(spr.OP_CACHE_APPEND, None) == INVALID and L.spr_draft_pass_call(3, b"\0" * 256) == INVALID


def test_nothing_to_do(mem):
    """Empty calls touch nothing, pointers included."""
    L, p = spr.lib(), mem[1]
    for empty in (dict(B=0), dict(T=0)):
        assert append(L, p, **empty, q=None, k=None, v=None, lens=None, table=None, kc=None, vc=None, qo=None, ws=None, n=0) == OK
        assert attend(L, p, **empty, q=None, kc=None, vc=None, lens=None, table=None, out=None, ws=None, n=0) == OK
        assert rules(L, p, **empty, l=None, out=None, ws=None, n=0) == OK


class _Cuda(torch.Tensor):
    """Stands for a CUDA tensor in the binding's checks, which come before anything is read."""

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return 0


def fake(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(_Cuda)


@pytest.fixture
def device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ws = object.__new__(spr.Workspace)
    ws.buf = fake(256, dtype=torch.uint8)
    return ws


I32 = torch.int32


def append_args(ws, **kw):
    a = dict(k=fake(2, 3, 2, 16), v=fake(2, 3, 2, 16), k_cache=fake(9, 2, 16, 16), v_cache=fake(9, 2, 16, 16), page_table=fake(2, 4, dtype=I32),
             lens=fake(2, dtype=I32), ws=ws, q=fake(2, 3, 4, 16), inv_freq=fake(8, dtype=torch.float32))
    a.update(kw)
    return a


@pytest.mark.parametrize("bad,why", [
    (dict(k=torch.zeros(2, 3, 2, 16, dtype=torch.bfloat16)), ValueError), (dict(v=fake(2, 3, 3, 16)), ValueError),
    (dict(v=fake(2, 3, 2, 16, dtype=torch.float32)), TypeError), (dict(k_cache=fake(9, 3, 16, 16)), ValueError),
    (dict(v_cache=fake(8, 2, 16, 16)), ValueError), (dict(page_table=fake(3, 4, dtype=I32)), ValueError),
    (dict(page_table=fake(2, 4, dtype=torch.int64)), TypeError), (dict(lens=fake(3, dtype=I32)), ValueError),
    (dict(lens=fake(2, dtype=torch.int64)), TypeError), (dict(inv_freq=fake(9, dtype=torch.float32)), ValueError),
    (dict(inv_freq=fake(8)), TypeError), (dict(counts=fake(3, dtype=I32)), ValueError), (dict(parents=fake(2, 4, dtype=I32)), ValueError),
    (dict(slots=fake(2, dtype=I32)), ValueError), (dict(q=fake(2, 3, 4, 8)), ValueError), (dict(q_out=fake(2, 3, 4, 8)), ValueError),
    (dict(q=None, q_out=fake(2, 3, 4, 16)), ValueError), (dict(k=fake(2, 3, 16, 2).transpose(2, 3)), ValueError),
    (dict(k=fake(3, 2, 2, 16).transpose(0, 1)), ValueError), (dict(k=fake(6, 2, 16)), ValueError),
    (dict(v=fake(2, 3, 4, 16, dtype=torch.float32)[:, :, :2]), TypeError), (dict(v=torch.zeros(2, 3, 4, 16, dtype=torch.bfloat16)[:, :, :2]), ValueError)])
def test_binding_refuses_append(device, bad, why):
    with pytest.raises(why):
        spr.cache_append(**append_args(device, **bad))


@pytest.mark.parametrize("bad,why", [
    (dict(q=fake(2, 3, 16)), ValueError), (dict(q=fake(2, 3, 4, 16).transpose(1, 2)), ValueError), (dict(k_cache=fake(9, 2, 16, 8)), ValueError),
    (dict(k_cache=fake(9, 2, 16, 16, dtype=torch.float32)), TypeError), (dict(out=fake(2, 3, 4, 8)), ValueError),
    (dict(out=fake(2, 3, 4, 16, dtype=torch.float32)), TypeError), (dict(counts=fake(3, dtype=I32)), ValueError),
    (dict(parents=fake(2, 3)), TypeError), (dict(lens=torch.zeros(2, dtype=I32)), ValueError)])
def test_binding_refuses_attention(device, bad, why):
    a = dict(q=fake(2, 3, 4, 16), k_cache=fake(9, 2, 16, 16), v_cache=fake(9, 2, 16, 16), page_table=fake(2, 4, dtype=I32),
             lens=fake(2, dtype=I32), ws=device)
    a.update(bad)
    with pytest.raises(why):
        spr.tree_attention(**a)


@pytest.mark.parametrize("bad,why", [
    (dict(logits=fake(6, 100)), ValueError), (dict(logits=fake(2, 3, 100, dtype=torch.float16)), TypeError),
    (dict(history_len=None), ValueError), (dict(history=None), ValueError), (dict(history=fake(3, 8, dtype=I32)), ValueError),
    (dict(history=fake(2, 8, dtype=torch.int64)), TypeError), (dict(tokens=fake(2, 4, dtype=I32)), ValueError),
    (dict(penalties=fake(2, 2, dtype=torch.float32)), ValueError), (dict(bias_values=None), ValueError),
    (dict(bias_values=fake(2, 3, dtype=torch.float32)), ValueError), (dict(mask_rows=None), ValueError),
    (dict(masks=fake(0, 4, dtype=I32)), ValueError), (dict(mask_rows=fake(2, dtype=I32)), ValueError),
    (dict(out=fake(2, 4, 100)), ValueError), (dict(out=fake(2, 3, 100, dtype=torch.float32)), TypeError), (dict(V=1 << 32), ValueError)])
def test_binding_refuses_rules(device, bad, why):
    a = dict(logits=fake(2, 3, 100), V=100, ws=device, history=fake(2, 8, dtype=I32), history_len=fake(2, dtype=I32),
             tokens=fake(2, 3, dtype=I32), penalties=fake(2, 3, dtype=torch.float32), bias_tokens=fake(2, 2, dtype=I32),
             bias_values=fake(2, 2, dtype=torch.float32), masks=fake(3, 4, dtype=I32), mask_rows=fake(2, 3, dtype=I32))
    a.update(bad)
    with pytest.raises(why):
        spr.logits_rules(**a)


def test_reference_paths():
    assert ref.path(None, 3) == [3, 2, 1, 0] and ref.path([-1, 0, 0, 1, -1], 3) == [3, 1, 0] and ref.path([-1, 0, 0, 1, -1], 4) == [4]


def test_reference_attention_is_softmax_over_what_is_seen():
    """The tests' own statement against a masked softmax written out for one sequence."""
    g = torch.Generator().manual_seed(1)
    q, k, v = torch.randn(1, 3, 2, 8, generator=g), torch.randn(2, 1, 8, 8, generator=g), torch.randn(2, 1, 8, 8, generator=g)
    parents = torch.tensor([[-1, 0, 0]], dtype=I32)
    out, _ = ref.attend(q, k, v, torch.tensor([[1, 0]], dtype=I32), torch.tensor([7], dtype=I32), None, parents, 0.5)
    keys, vals = torch.cat([k[1, 0], k[0, 0]])[:10].double(), torch.cat([v[1, 0], v[0, 0]])[:10].double()
    see = torch.ones(3, 10, dtype=torch.bool)
    see[0, 8:], see[1, 9], see[2, 8] = False, False, False
    for h in range(2):
        p = torch.softmax((0.5 * q[0, :, h].double() @ keys.T).masked_fill(~see, -math.inf), -1)
        assert torch.allclose(out[0, :, h], p @ vals)
