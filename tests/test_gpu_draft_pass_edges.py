"""tree_attention, cache_append and logits_rules at the edges of what they are documented for: infinities, tensors in place, long
histories, prompts in pieces.  Bounds in draft_pass_reference.py."""
import math

import pytest
import torch

import draft_pass_reference as ref
from test_gpu_draft_pass import BF16, F32, attend_case, check_attend, check_rules, ids, rules_case, run_attend, spr  # noqa: F401

pytestmark = pytest.mark.gpu


def put(cache, x, b, slot, value):
    """The entry of a sequence's slot, all heads (and columns, or as many as value has)."""
    page = cache.shape[2]
    cache[int(x["page_table"][b, slot // page]), :, slot % page] = value


@pytest.mark.parametrize("T,G,D,tiles", [(12, 2, 64, 4), (9, 4, 128, 4), (40, 1, 80, 3), (30, 5, 128, 2)])
def test_a_maximum_is_raised_beside_infinities(spr, T, G, D, tiles):  # noqa: F811
    """The last tile's keys raise the maximum of rows that have results so far, and hold a value that is infinite for some of them
    only: the others have what they have where that value is zero."""
    lens = [64 * tiles + 10, 64 * tiles + 50 - T]
    x = attend_case(2, T, 2 * G, 2, D, 16, BF16, seed=T, tree=True, lens=lens)
    x["q"] = (1 + 0.25 * x["q"].float()).to(BF16)
    for b in range(2):
        for slot in range(64 * tiles, lens[b]):
            put(x["k_cache"], x, b, slot, 256.0 / D)      # scores of some 256 / sqrt(D), 32 binary exponents and more
        x["parents"][b, 1] = 0                             # (node 1 has rows that see it and rows that do not)
        x["parents"][b, 2] = -1
    clean = dict(x, v_cache=x["v_cache"].clone())
    for b in range(2):
        put(x["v_cache"], x, b, lens[b] + 1, math.inf)
        put(clean["v_cache"], x, b, lens[b] + 1, 0.0)
    got, want = check_attend(spr, x).cpu(), check_attend(spr, clean).cpu()
    for b in range(2):
        sees = torch.tensor([1 in ref.path(x["parents"][b].tolist(), i) for i in range(T)])
        assert bool(sees.any()) and not bool(sees.all())
        assert torch.equal(got[b][~sees], want[b][~sees]) and bool(torch.isfinite(got[b][~sees]).all())
        assert bool((got[b][sees] == math.inf).all())


ROWS = [(1, 4), (2, 4), (5, 3), (8, 4), (40, 4)]            # nodes and queries per cached head: every kernel


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,G", ROWS)
def test_scores_of_minus_infinity(spr, T, G, dtype):  # noqa: F811
    """A score of -inf is a weight of zero, and a row that has no other score is NaN (not zeros: it does see keys), in items of one
    part and of many."""
    lens = [70, 70, 9000, 9000, 0]
    x = attend_case(5, T, 2 * G, 2, 64, 16, dtype, seed=91 + T, lens=lens)
    x["parents"] = torch.full((5, T), -1, dtype=torch.int32)         # all nodes follow the prefix: a row sees its own only
    x["q"][..., 0] = 1.0
    x["k_cache"][..., 0] = 0.0
    low = dict(x, k_cache=x["k_cache"].clone())
    for k, value in ((x["k_cache"], -math.inf), (low["k_cache"], -2000.0)):      # (scores of -250: weights of zero too)
        for b, n in enumerate(lens):
            own = range(n, n + T, 2)                                  # every other node
            for slot in [*range(n if b % 2 == 0 else n - 40), *own]:  # all of the prefix, or all but its last 40
                head = k[int(x["page_table"][b, slot // 16])]
                head[:, slot % 16, 0] = value
    got = run_attend(spr, x).cpu()
    args = {n: None if t is None else t.cuda() for n, t in low.items()}
    want, tol = ref.attend(args["q"], args["k_cache"], args["v_cache"], x["page_table"], x["lens"], None, x["parents"], 64 ** -0.5)
    for b, n in enumerate(lens):
        for i in range(T):
            if b % 2 == 0 and i % 2 == 0:
                assert bool(got[b, i].isnan().all()), (b, i)
            else:
                assert ref.within(got[b, i], want[b, i].cpu(), tol[b, i].cpu()), (b, i)
    # the same with signs the other way round
    y = dict(x, k_cache=x["k_cache"].clone())
    y["k_cache"].neg_()
    again = run_attend(spr, y, scale=-64 ** -0.5).cpu()
    assert torch.equal(again.isnan(), got.isnan()) and torch.equal(again.nan_to_num(), got.nan_to_num())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,G", ROWS)
def test_infinite_values_that_all_rows_see(spr, T, G, dtype):  # noqa: F811
    """Weights are positive: an infinite value makes its column infinite, with its sign, wherever it lies in the sequence."""
    lens = [130, 700, 9000]
    x = attend_case(3, T, 2 * G, 2, 64, 16, dtype, seed=95 + T, lens=lens)
    for b, n in enumerate(lens):
        for column, value, slots in ((3, math.inf, range(n)), (5, -math.inf, range(n)), (8, math.inf, (0, 77)), (9, math.nan, (n // 2,)),
                                     (10, -math.inf, (n - 1,))):
            for slot in slots:
                x["v_cache"][int(x["page_table"][b, slot // 16]), :, slot % 16, column] = value
    got = check_attend(spr, x)
    bad = [3, 5, 8, 9, 10]
    assert bool(torch.isfinite(got[..., [c for c in range(64) if c not in bad]]).all())
    for column, value in ((3, math.inf), (5, -math.inf), (8, math.inf), (10, -math.inf)):
        assert bool((got[..., column] == value).all())
    assert bool(got[..., 9].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("D", [8, 64])
@pytest.mark.parametrize("T,G", ROWS)
def test_results_over_the_queries(spr, T, G, D, dtype):  # noqa: F811
    """In place: the bits that another tensor gets, in items of one part and of many, unused nodes among them."""
    lens = [30, 9000, 0, 700, -1, 2000]
    x = attend_case(6, T, 2 * G, 2, D, 16, dtype, seed=97 + T, tree=True, lens=lens, counts=[T, T, T // 2, T, T, 1])
    want = run_attend(spr, x)
    ws = spr.Workspace(spr.workspace_bytes(spr.OP_TREE_ATTENTION, 1, 1, 1, D, 0, spr.F32 if dtype == F32 else spr.BF16))
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    for _ in range(3):
        q = c["q"].clone()
        got = spr.tree_attention(q, c["k_cache"], c["v_cache"], c["page_table"], c["lens"], ws, counts=c["counts"], parents=c["parents"], out=q)
        assert got is q and torch.equal(q, want) and ws.device_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("B,T,V,L", [(2, 5, 3001, 131072), (1, 1, 128256, 131072), (8, 1, 600007, 40000), (1, 40, 5000, 20011)])
def test_rules_over_long_histories(spr, B, T, V, L, dtype):  # noqa: F811
    """Tokens that stand hundreds of times in a history as long as a cache: both forms."""
    x, dims = rules_case(B, T, V, dtype, seed=101, L=L, masks=2)
    x["history"] = torch.randint(-1, 500, (B, L), generator=torch.Generator().manual_seed(102)).to(torch.int32)
    x["history_len"] = L - torch.arange(B, dtype=torch.int32) * 7
    check_rules(spr, x, dims)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("n,piece,Hq,Hkv,D", [(700, 256, 8, 2, 64), (513, 128, 4, 4, 128), (300, 256, 3, 1, 40)])
def test_a_prompt_in_pieces(spr, n, piece, Hq, Hkv, D, dtype):  # noqa: F811
    """A prompt goes into the cache at once and is attended to in pieces, each over those before it: causal attention."""
    x = attend_case(2, n, Hq, Hkv, D, 16, dtype, seed=103, lens=[0, 37])
    c = {k: None if t is None else t.cuda() for k, t in x.items()}
    ws = spr.Workspace(spr.workspace_bytes(spr.OP_TREE_ATTENTION, 1, 1, 1, D, 0, spr.F32 if dtype == F32 else spr.BF16))
    g = torch.Generator().manual_seed(104)
    k, v = (torch.randn((2, n, Hkv, D), generator=g).to(dtype).cuda() for _ in range(2))
    spr.cache_append(k, v, c["k_cache"], c["v_cache"], c["page_table"], c["lens"], ws)
    got = [spr.tree_attention(c["q"][:, at:at + piece].contiguous(), c["k_cache"], c["v_cache"], c["page_table"], c["lens"] + at, ws)
           for at in range(0, n, piece)]
    assert ws.device_status() == 0
    want, tol = ref.attend(c["q"], c["k_cache"], c["v_cache"], x["page_table"], x["lens"], None, None, D ** -0.5)
    # (a short last piece may be worked on with more precise weights than the bound allows for, never with less)
    got = torch.cat(got, 1)
    assert ref.within(got, want, tol), ref.worst(got, want, tol)
