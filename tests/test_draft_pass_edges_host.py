"""CPU-side checks of cache_append, tree_attention and logits_rules at the edges of their arguments: refusals that come before
any device call."""
import struct

import pytest
import torch

import paper_2502_04557_b200 as spr
from paper_2502_04557_b200 import binding
from test_draft_pass_host import INVALID, WORKSPACE, append, attend, device, fake, mem, rules  # noqa: F401


def test_append_in_place_only_where_dense(mem):  # noqa: F811
    """Rotated queries over the queries' own place, but closer together, would overwrite some that are still to be read."""
    L, p = spr.lib(), mem[1]
    assert append(L, p, k=p + 512, v=p + 512, qs=65) == INVALID and append(L, p, qs=128) == INVALID
    for fine in (dict(), dict(B=1, T=1, qs=128), dict(qs=128, qo=p + 1024), dict(q=None, qo=None, qs=128)):
        assert append(L, p, n=255, **fine) == WORKSPACE, fine           # (refused, but not for that)


@pytest.mark.parametrize("op,f,real,names", [
    (spr.OP_CACHE_APPEND, append, None, ("B", "T", "Hq", "Hkv", "D", "dt", "rot", "inter", "max_pages", "pages", "page")),
    (spr.OP_TREE_ATTENTION, attend, "scale", ("B", "T", "Hq", "Hkv", "D", "dt", "max_pages", "pages", "page")),
    (spr.OP_LOGITS_RULES, rules, None, ("V", "B", "T", "dt", "nb", "nm"))])
def test_numbers_in_an_array_fit(mem, op, f, real, names):  # noqa: F811
    """What the plain calls take as 32-bit integers is not cut to 32 bits."""
    L, p = spr.lib(), mem[1]
    keep = {}

    class Recorder:
        def __getattr__(self, _):
            return lambda *a: keep.setdefault("values", a)

    def call(**kw):
        keep.clear()
        f(Recorder(), p, n=255, **kw)
        values = [0 if a is None else a for a in keep["values"]]
        return L.spr_draft_pass_call(op, struct.pack("".join("d" if isinstance(a, float) else "q" for a in values), *values))

    assert call() == WORKSPACE
    usual = dict(B=2, T=3, Hq=4, Hkv=2, D=64 if real else 16, dt=1, rot=16, inter=0, max_pages=4, pages=9, page=16, V=100, nb=2, nm=3)
    for name in names:
        assert call(**{name: usual[name]}) == WORKSPACE
        for far in (1 << 32, -1 << 32):
            assert call(**{name: usual[name] + far}) == INVALID, (name, far)
    if "B" in names:
        assert call(B=1 << 32) == INVALID          # (not an empty call)


def test_every_declared_function_is_listed():
    from test_host_api import declared_functions
    assert set(binding.EXPORTS) == set(declared_functions())


def test_heads_without_columns_are_refused(device, monkeypatch):  # noqa: F811
    """By the library, like other sizes that it does not take (there is no scale of 1 / sqrt(0) to fall over before)."""
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    with pytest.raises(spr.SprinterError) as e:
        spr.tree_attention(fake(2, 3, 4, 0), fake(9, 2, 16, 0), fake(9, 2, 16, 0), fake(2, 4, dtype=torch.int32), fake(2, dtype=torch.int32),
                           device)
    assert e.value.status == INVALID
