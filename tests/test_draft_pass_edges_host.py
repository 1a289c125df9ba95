"""CPU-side checks of cache_append, tree_attention and logits_rules at the edges of their arguments: refusals that come before
any device call."""
import paper_2502_04557_b200 as spr
from test_draft_pass_host import INVALID, WORKSPACE, append, mem  # noqa: F401


def test_append_in_place_only_where_dense(mem):  # noqa: F811
    """Rotated queries over the queries' own place, but closer together, would overwrite some that are still to be read."""
    L, p = spr.lib(), mem[1]
    assert append(L, p, k=p + 512, v=p + 512, qs=65) == INVALID and append(L, p, qs=128) == INVALID
    for fine in (dict(), dict(B=1, T=1, qs=128), dict(qs=128, qo=p + 1024), dict(q=None, qo=None, qs=128)):
        assert append(L, p, n=255, **fine) == WORKSPACE, fine           # (refused, but not for that)
