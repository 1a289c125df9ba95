"""cache_append, tree_attention and logits_rules against plain float64; bounds in draft_pass_reference.py."""
import math

import pytest
import torch

import draft_pass_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
IDS = {BF16: "bf16", F32: "f32"}
OK, TIMEOUT, BAD_TOKEN, BAD_ROW, BAD_PAGE, BAD_TREE = 0, 5, 6, 7, 8, 9


@pytest.fixture(scope="module")
def spr():
    import paper_2502_04557_b200 as s
    s.lib()
    return s


def ids(x):
    return IDS.get(x, str(x))


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


def code(spr, dtype):
    return spr.F32 if dtype == F32 else spr.BF16


def workspace(spr, op, D=1, dtype=BF16):
    return spr.Workspace(spr.workspace_bytes(op, 1, 1, 1, D, 0, code(spr, dtype)))


def spread(*shape, g, dtype):
    return torch.randn(shape, generator=g).to(dtype)


# ---------------------------------------------------------------------------- cache_append


def append_case(B, T, Hq, Hkv, D, page, dtype, seed, tree=False, lens=None, ragged=False):
    g = torch.Generator().manual_seed(seed)
    lens = torch.tensor(lens, dtype=torch.int32) if lens is not None else torch.randint(0, 70, (B,), generator=g).to(torch.int32)
    most = (max(int(lens.max()), 0) + T + page - 1) // page
    table, pages = ref.make_pages(B, most, 2, g)
    x = dict(q=spread(B, T, Hq, D, g=g, dtype=dtype) if Hq else None, k=spread(B, T, Hkv, D, g=g, dtype=dtype),
             v=spread(B, T, Hkv, D, g=g, dtype=dtype), k_cache=spread(pages, Hkv, page, D, g=g, dtype=dtype),
             v_cache=spread(pages, Hkv, page, D, g=g, dtype=dtype), page_table=table, lens=lens,
             parents=ref.make_tree(B, T, g) if tree else None,
             counts=torch.randint(0, T + 1, (B,), generator=g).to(torch.int32) if ragged else None, slots=None)
    return x


def freqs(pairs, base=10000.0):
    return (base ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float()


def run_append(spr, x, inv_freq, interleaved, status=OK, inplace=False):
    ws = workspace(spr, spr.OP_CACHE_APPEND)
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    f = None if inv_freq is None else inv_freq.cuda()
    q_out = c["q"] if inplace else None
    q_out = spr.cache_append(c["k"], c["v"], c["k_cache"], c["v_cache"], c["page_table"], c["lens"], ws, q=c["q"], inv_freq=f,
                             interleaved=interleaved, counts=c["counts"], parents=c["parents"], slots=c["slots"], q_out=q_out)
    assert ws.device_status() == status
    return q_out, c["k_cache"], c["v_cache"]


def check_append(spr, x, inv_freq, interleaved=False, **kw):
    got = run_append(spr, x, inv_freq, interleaved, **kw)
    want, tol = ref.append(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], x["page_table"], x["lens"], inv_freq, interleaved,
                           x["counts"], x["parents"], x["slots"])
    for name, a, b, t in zip(("q_out", "k_cache", "v_cache"), got, want, tol):
        if b is not None:
            assert ref.within(a.cpu(), b, t), (name, ref.worst(a.cpu(), b, t))
    return got


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,page,rot", [
    (1, 1, 1, 1, 8, 1, 8), (3, 5, 4, 2, 64, 16, 64), (2, 9, 8, 2, 128, 16, 64), (2, 3, 3, 3, 80, 24, 80), (1, 4, 2, 1, 33, 5, 10),
    (2, 2, 5, 1, 96, 8, 2), (1, 2, 2, 2, 256, 16, 256), (1, 70, 2, 1, 64, 32, 0), (5, 1, 0, 4, 128, 16, 128)])
def test_append(spr, B, T, Hq, Hkv, D, page, rot, interleaved, dtype):
    x = append_case(B, T, Hq, Hkv, D, page, dtype, seed=D + T)
    check_append(spr, x, freqs(rot // 2) if rot else None, interleaved)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_append_tree_counts_and_unused_sequences(spr, dtype):
    x = append_case(5, 40, 4, 2, 64, 16, dtype, seed=3, tree=True, ragged=True, lens=[0, 17, -1, 3, 100])
    x["counts"][:] = torch.tensor([40, 0, 7, 50, 23])
    got = check_append(spr, x, freqs(32))
    assert bool((got[0][2] == 0).all()) and bool((got[0][1] == 0).all()) and bool((got[0][4, 23:] == 0).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_far_positions(spr, interleaved):
    """Angles of 2^20 radians and more."""
    x = append_case(2, 3, 2, 1, 64, 16, F32, seed=5, lens=[(1 << 20) - 5, 131071])
    table, pages = torch.full((2, (1 << 20) // 16 + 1), -1, dtype=torch.int32), 4
    table[0, ((1 << 20) - 5) // 16] = 2                 # only the pages that are written are there
    table[1, 131071 // 16:131071 // 16 + 2] = torch.tensor([0, 3])
    x["page_table"] = table
    x["k_cache"], x["v_cache"] = x["k_cache"][:pages].clone(), x["v_cache"][:pages].clone()
    if x["k_cache"].shape[0] < pages:
        x["k_cache"], x["v_cache"] = torch.zeros(pages, 1, 16, 64), torch.zeros(pages, 1, 16, 64)
    check_append(spr, x, freqs(32), interleaved)


@pytest.mark.parametrize("dtype,D,rot", [(BF16, 64, 64), (F32, 64, 32), (BF16, 20, 12)], ids=ids)
def test_append_parts_of_one_projection(spr, dtype, D, rot):
    """q, k and v side by side, as one product gives them; the same bits as from dense tensors."""
    g = torch.Generator().manual_seed(8)
    x = append_case(3, 4, 4, 2, D, 16, dtype, seed=9)
    dense = check_append(spr, x, freqs(rot // 2))
    both = torch.cat([x["q"], x["k"], x["v"]], 2).cuda()
    ws = workspace(spr, spr.OP_CACHE_APPEND)
    kc, vc, table, lens = cuda(x["k_cache"], x["v_cache"], x["page_table"], x["lens"])
    q = spr.cache_append(both[:, :, 4:6], both[:, :, 6:], kc, vc, table, lens, ws, q=both[:, :, :4], inv_freq=freqs(rot // 2).cuda())
    assert ws.device_status() == OK
    for a, b in zip((q, kc, vc), dense):
        assert torch.equal(a, b)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 36)], ids=ids)
def test_append_queries_in_place(spr, dtype, D, interleaved):
    x = append_case(2, 6, 4, 1, D, 16, dtype, seed=11)
    check_append(spr, x, freqs(D // 2), interleaved, inplace=True)


def test_append_given_slots(spr):
    """The nodes that were kept go to the slots behind the prefix, the others nowhere."""
    x = append_case(2, 8, 2, 2, 64, 8, BF16, seed=13, tree=True, lens=[5, 30])
    x["slots"] = torch.full((2, 8), -1, dtype=torch.int32)
    for b, keep in ((0, ref.path(x["parents"][0].tolist(), 7)), (1, ref.path(x["parents"][1].tolist(), 5))):
        for depth, i in enumerate(reversed(keep)):
            x["slots"][b, i] = int(x["lens"][b]) + depth
    check_append(spr, x, freqs(32))


def test_append_slots_without_a_page(spr):
    x = append_case(3, 4, 2, 1, 64, 16, BF16, seed=15, lens=[14, 14, 200])
    x["page_table"] = x["page_table"][:, :2].clone()
    x["page_table"][0, 1] = -1                    # two of sequence 0's nodes
    x["page_table"][1, 0] = x["k_cache"].shape[0]    # two of sequence 1's; sequence 2 is behind the table
    kc, vc = x["k_cache"].clone(), x["v_cache"].clone()
    _, k2, v2 = run_append(spr, x, freqs(32), False, status=BAD_PAGE)
    changed = {(p, e) for p, e in (k2.cpu() != kc).any(-1).any(1).nonzero().tolist()} | {(p, e) for p, e in (v2.cpu() != vc).any(-1).any(1).nonzero().tolist()}
    assert changed == {(int(x["page_table"][0, 0]), 14), (int(x["page_table"][0, 0]), 15), (int(x["page_table"][1, 1]), 0), (int(x["page_table"][1, 1]), 1)}


def test_append_bad_tree(spr):
    """A parent that does not come before its child counts as the prefix."""
    x = append_case(1, 5, 2, 1, 64, 16, F32, seed=17, tree=True)
    bad = torch.tensor([[0, 0, 7, 2, 3]], dtype=torch.int32)
    x["parents"] = torch.tensor([[-1, 0, -1, 2, 3]], dtype=torch.int32)
    want = run_append(spr, x, freqs(32), False)
    x["parents"] = bad
    got = run_append(spr, x, freqs(32), False, status=BAD_TREE)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------- tree_attention


def attend_case(B, T, Hq, Hkv, D, page, dtype, seed, tree=False, lens=None, counts=None, q_scale=1.0):
    g = torch.Generator().manual_seed(seed)
    lens = torch.tensor(lens, dtype=torch.int32) if lens is not None else torch.randint(0, 200, (B,), generator=g).to(torch.int32)
    most = max((max(int(lens.max()), 0) + T + page - 1) // page, 1)
    table, pages = ref.make_pages(B, most, 1, g)
    return dict(q=spread(B, T, Hq, D, g=g, dtype=dtype) * q_scale, k_cache=spread(pages, Hkv, page, D, g=g, dtype=dtype),
                v_cache=spread(pages, Hkv, page, D, g=g, dtype=dtype), page_table=table, lens=lens,
                counts=None if counts is None else torch.tensor(counts, dtype=torch.int32),
                parents=ref.make_tree(B, T, g) if tree else None)


def run_attend(spr, x, scale=None, status=OK, ws=None, **kw):
    ws = ws or workspace(spr, spr.OP_TREE_ATTENTION, x["q"].shape[-1], x["q"].dtype)
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    out = spr.tree_attention(c["q"], c["k_cache"], c["v_cache"], c["page_table"], c["lens"], ws, scale=scale, counts=c["counts"],
                             parents=c["parents"], **kw)
    assert ws.device_status() == status
    return out


def check_attend(spr, x, scale=None, **kw):
    got = run_attend(spr, x, scale, **kw)
    s = x["q"].shape[-1] ** -0.5 if scale is None else scale
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    want, tol = ref.attend(c["q"], c["k_cache"], c["v_cache"], x["page_table"], x["lens"], x["counts"], x["parents"], s)
    ok = ref.within(got, want, tol)
    assert ok, ref.worst(got, want, tol)
    return got


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,page", [
    (1, 1, 1, 1, 64, 16), (3, 1, 8, 2, 128, 16), (2, 4, 4, 2, 64, 8), (2, 5, 6, 3, 128, 64), (3, 7, 4, 4, 80, 24), (2, 9, 12, 12, 64, 16),
    (2, 17, 8, 2, 128, 32), (1, 33, 8, 1, 96, 128), (2, 64, 8, 2, 128, 16), (1, 200, 3, 1, 64, 48), (2, 3, 5, 1, 8, 16), (1, 31, 7, 1, 40, 256)])
def test_attention(spr, B, T, Hq, Hkv, D, page, tree, dtype):
    check_attend(spr, attend_case(B, T, Hq, Hkv, D, page, dtype, seed=B + T + D, tree=tree))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,G", [(1, 1), (1, 8), (5, 3), (9, 4), (17, 4), (40, 4)])
def test_attention_lengths(spr, T, G, dtype):
    """No prefix, one token, tiles and pages that end at, before and behind the sequence's end, sequences of no nodes."""
    lens = [0, 1, 15, 16, 17, 62, 63, 64, 65, 127, 128, 129, 500, -1, 1000]
    counts = [T] * len(lens)
    counts[3], counts[12] = 0, 1
    x = attend_case(len(lens), T, 2 * G, 2, 64, 16, dtype, seed=T, tree=T > 5, lens=lens, counts=counts)
    got = check_attend(spr, x)
    assert bool((got[3] == 0).all()) and bool((got[13] == 0).all()) and bool((got[12, 1:] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 8, 2, 128), (8, 8, 2, 64), (17, 8, 2, 128), (64, 8, 1, 128)])
def test_attention_long(spr, T, Hq, Hkv, D, dtype):
    """One long sequence beside short ones: its items are shared by many CTAs."""
    check_attend(spr, attend_case(3, T, Hq, Hkv, D, 16, dtype, seed=21, tree=True, lens=[20011, 3, 700]))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_attention_sharp_and_negative_scales(spr, dtype):
    """Weights that all but one key lose, growing maxima, and a scale below zero."""
    x = attend_case(2, 4, 4, 2, 64, 16, dtype, seed=23, lens=[300, 1500], q_scale=1.0)
    check_attend(spr, x, scale=2.0)
    check_attend(spr, x, scale=-0.3)
    check_attend(spr, x, scale=0.0)
    k = x["k_cache"]
    for b in range(2):                # scores that grow with the slot
        for slot in range(int(x["lens"][b])):
            k[int(x["page_table"][b, slot // 16]), :, slot % 16] = (x["q"][b, 0, ::2].float().sign() * (0.01 * slot)).to(dtype)
    check_attend(spr, x, scale=0.05)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,G,D", [(2, 1, 64), (6, 4, 128), (20, 3, 128), (48, 4, 128)])
def test_attention_nothing_from_what_is_not_seen(spr, T, G, D, dtype):
    """Infinities and NaN in entries behind the last slot, in pages of nobody and in nodes off a row's path."""
    lens = [0, 13, 64, 150]
    x = attend_case(4, T, 2 * G, 2, D, 16, dtype, seed=25, tree=True, lens=lens, counts=[T, max(T - 1, 1), T, T])
    owned = torch.zeros(x["k_cache"].shape[0], 16, dtype=torch.bool)
    for b, n in enumerate(lens):
        for slot in range(n + int(x["counts"][b])):
            owned[int(x["page_table"][b, slot // 16]), slot % 16] = True
    for c, bad in ((x["k_cache"], math.nan), (x["v_cache"], math.inf)):
        c.masked_fill_(~owned[:, None, :, None], bad)
    check_attend(spr, x)
    # node 1 of sequence 3 (and what follows it) sees infinities, the others do not
    slot = lens[3] + 1
    page = int(x["page_table"][3, slot // 16])
    x["v_cache"][page, :, slot % 16, 3] = math.inf
    x["v_cache"][page, :, slot % 16, 5] = -math.inf
    got = run_attend(spr, x).cpu()
    sees = torch.tensor([1 in ref.path(x["parents"][3].tolist(), i) for i in range(T)])
    assert bool(torch.isfinite(got[3][~sees]).all()) and bool(torch.isfinite(got[:3]).all())
    assert not bool(torch.isfinite(got[3][sees][..., [3, 5]]).any())
    y = dict(x, v_cache=x["v_cache"].clone())
    y["v_cache"][page, :, slot % 16] = 0
    clean = run_attend(spr, y).cpu()
    assert torch.equal(got[3][~sees], clean[3][~sees]) and torch.equal(got[:3], clean[:3])
    # a key that is NaN: rows that see it are NaN
    x["k_cache"][page, :, slot % 16, 0] = math.nan
    got = run_attend(spr, x).cpu()
    assert bool(torch.isfinite(got[3][~sees]).all()) and bool(got[3][sees].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_attention_without_pages(spr, dtype):
    """Slots without a page are left out and reported; a row that sees none is zeros."""
    x = attend_case(3, 2, 2, 1, 64, 16, dtype, seed=27, lens=[40, 40, 10])
    for bad in (-1, x["k_cache"].shape[0]):
        y = dict(x, page_table=x["page_table"].clone())
        y["page_table"][1, 1] = bad
        y["page_table"][2, 0] = bad
        got = run_attend(spr, y, status=BAD_PAGE)
        assert bool((got[2] == 0).all()) and bool(torch.isfinite(got).all())
        want = run_attend(spr, x)
        assert torch.equal(got[0], want[0]) and not torch.equal(got[1], want[1])
    y = dict(x, page_table=x["page_table"][:, :1].contiguous())      # the table ends before the sequences
    run_attend(spr, y, status=BAD_PAGE)


def test_attention_pages_behind_the_end_are_not_looked_at(spr):
    x = attend_case(2, 3, 4, 2, 64, 16, BF16, seed=29, lens=[20, 5])
    x["page_table"][1, 1:] = -1
    check_attend(spr, x)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_attention_bad_tree(spr, dtype):
    x = attend_case(1, 5, 2, 1, 64, 16, dtype, seed=31, lens=[9])
    x["parents"] = torch.tensor([[-1, 0, -1, 2, 3]], dtype=torch.int32)
    want = check_attend(spr, x)
    x["parents"] = torch.tensor([[0, 0, 7, 2, 3]], dtype=torch.int32)
    assert torch.equal(run_attend(spr, x, status=BAD_TREE), want)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_attention_runs_alike(spr, dtype):
    """Bit for bit the same again, whatever the workspace held, and beside another call on another stream."""
    x = attend_case(4, 9, 8, 2, 128, 16, dtype, seed=33, tree=True, lens=[5000, 40, 900, 17])
    ws = workspace(spr, spr.OP_TREE_ATTENTION, 128, dtype)
    a = run_attend(spr, x, ws=ws)
    y = attend_case(2, 1, 8, 2, 128, 16, dtype, seed=34, lens=[9000, 70])
    run_attend(spr, y, ws=ws)
    assert torch.equal(run_attend(spr, x, ws=ws), a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = run_attend(spr, x)
    b = run_attend(spr, x, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(b, a) and torch.equal(c, a)


def test_attention_timeout(spr):
    """No tile is ever loaded: every wait runs out, results are NaN, and the workspace stays usable."""
    x = attend_case(2, 3, 8, 2, 64, 16, BF16, seed=35, lens=[3000, 20])
    ws = workspace(spr, spr.OP_TREE_ATTENTION, 64)
    want = run_attend(spr, x, ws=ws)
    for T, G in ((5, 4), (40, 4)):
        y = attend_case(2, T, 2 * G, 2, 64, 16, BF16, seed=36, lens=[3000, 20])
        spr.lib().spr_test_tree_attention(1, 2000)
        try:
            got = run_attend(spr, y, status=TIMEOUT, ws=ws)
        finally:
            spr.lib().spr_test_tree_attention(0, 0)
        assert bool(got.isnan().all())
    assert torch.equal(run_attend(spr, x, ws=ws), want)


# ---------------------------------------------------------------------------- logits_rules


def rules_case(B, T, V, dtype, seed, ldv=None, L=30, n_bias=5, masks=3, tree=False, lead=0):
    g = torch.Generator().manual_seed(seed)
    ldv = ldv or V
    words = (V + 31) // 32 + 1
    flat = (torch.randn((lead + B * T * ldv,), generator=g) * 3).to(dtype)
    few = max(V // 4, 1)
    x = dict(logits=flat, history=torch.randint(-1, few, (B, L), generator=g).to(torch.int32),
             history_len=torch.randint(0, L + 1, (B,), generator=g).to(torch.int32),
             tokens=torch.randint(0, few, (B, T), generator=g).to(torch.int32), parents=ref.make_tree(B, T, g) if tree else None,
             counts=torch.randint(0, T + 1, (B,), generator=g).to(torch.int32) if tree else None,
             penalties=torch.rand((B, 3), generator=g) + torch.tensor([0.7, -0.2, -0.2]), bias_tokens=None, bias_values=None,
             masks=None, mask_rows=None)
    if n_bias:
        x["bias_tokens"] = torch.randint(-1, few, (B, n_bias), generator=g).to(torch.int32)
        x["bias_values"] = torch.randn((B, n_bias), generator=g) * 3
    if masks:
        x["masks"] = torch.randint(-2 ** 31, 2 ** 31, (masks, words), generator=g).to(torch.int32)
        x["masks"][0] = 0                                   # nothing is allowed
        x["mask_rows"] = torch.randint(-1, masks, (B, T), generator=g).to(torch.int32)
    return x, (B, T, V, ldv, lead)


def run_rules(spr, x, dims, status=OK, inplace=False, out=None):
    B, T, V, ldv, lead = dims
    ws = workspace(spr, spr.OP_LOGITS_RULES)
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    logits = c.pop("logits")[lead:].view(B, T, ldv)
    got = spr.logits_rules(logits, V, ws, out=logits if inplace else out, **c)
    assert ws.device_status() == status
    return got


def check_rules(spr, x, dims, **kw):
    B, T, V, ldv, lead = dims
    got = run_rules(spr, x, dims, **kw)[..., :V].cpu()
    rest = {n: t for n, t in x.items() if n != "logits"}
    want, tol = ref.rules(x["logits"][lead:].view(B, T, ldv), V, **rest)
    assert ref.within(got, want, tol), ref.worst(got, want, tol)
    return got


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("B,T,V,ldv", [(1, 1, 1, 1), (1, 1, 3, 3), (2, 3, 31, 40), (2, 5, 1000, 1000), (3, 4, 1001, 1001), (1, 2, 8197, 8200),
                                       (2, 9, 50257, 50257), (1, 40, 2049, 2055)])
def test_rules(spr, B, T, V, ldv, tree, dtype):
    x, dims = rules_case(B, T, V, dtype, seed=V + T, ldv=ldv, tree=tree)
    check_rules(spr, x, dims)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("lead", [0, 1, 3])
def test_rules_in_place_and_off_alignment(spr, lead, dtype):
    x, dims = rules_case(3, 4, 5003, dtype, seed=41, ldv=5009, lead=lead)
    a = check_rules(spr, x, dims, inplace=True)
    assert torch.equal(check_rules(spr, x, dims), a)
    out = torch.full((3, 4, 5014), 7.0, dtype=dtype, device="cuda")          # rows of another length
    run_rules(spr, x, dims, out=out)
    assert torch.equal(out[..., :5003].cpu(), a) and bool((out[..., 5003:] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_rules_many_sequences(spr, dtype):
    """The form for many sequences: longer stretches of the vocabulary."""
    x, dims = rules_case(80, 2, 33001, dtype, seed=43, L=700, n_bias=40, masks=4)
    check_rules(spr, x, dims)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("B,T,V,L,few", [(600, 1, 4000, 30, 1000), (40, 3, 70001, 900, 30000), (150, 2, 17001, 6000, 4250), (8, 1, 600007, 3000, 2900)])
def test_rules_few_rows(spr, B, T, V, L, few, dtype):
    """The form for few rows: long pieces of a row, in place and apart, off alignment, more touched tokens than its table holds."""
    x, dims = rules_case(B, T, V, dtype, seed=44, ldv=V + 2, L=L, n_bias=300, masks=3, lead=1, tree=T > 1)
    x["history"] = torch.randint(-1, few, (B, L), generator=torch.Generator().manual_seed(45)).to(torch.int32)
    a = check_rules(spr, x, dims, inplace=True)
    assert torch.equal(check_rules(spr, x, dims), a)
    out = torch.full((B, T, V + 5), 7.0, dtype=dtype, device="cuda")          # rows that lie otherwise: one by one
    run_rules(spr, x, dims, out=out)
    assert torch.equal(out[..., :V].cpu(), a) and bool((out[..., V:] == 7.0).all())


@pytest.mark.parametrize("without", ["penalties", "bias", "masks", "history", "tokens", "all"])
def test_rules_each_is_optional(spr, without):
    x, dims = rules_case(2, 6, 3001, BF16, seed=45, tree=True)
    gone = {"bias": ("bias_tokens", "bias_values"), "masks": ("masks", "mask_rows"), "history": ("history", "history_len"),
            "all": ("penalties", "bias_tokens", "bias_values", "masks", "mask_rows", "history", "history_len", "tokens")}.get(without, (without,))
    x.update({n: None for n in gone})
    got = check_rules(spr, x, dims)
    if without == "all":
        assert torch.equal(got, x["logits"].view(2, 6, 3001))


def test_rules_same_token_again(spr):
    """Repeated in the history, on the path and in the biases: counts add up, the last bias counts."""
    x, dims = rules_case(1, 6, 700, F32, seed=47, n_bias=0, masks=0)
    x["history"][:] = 5
    x["history_len"][:] = 30
    x["tokens"][:] = 5
    x["bias_tokens"], x["bias_values"] = torch.tensor([[9, 5, 9, 5]], dtype=torch.int32), torch.tensor([[1.0, 2.0, -3.0, 0.5]])
    got = check_rules(spr, x, dims)
    r, f, s = x["penalties"][0].double().tolist()
    l = x["logits"].view(6, 700)[3, 5].double().item()
    assert got[0, 3, 5].item() == pytest.approx((l / r if l > 0 else l * r) - 34 * f - s + 0.5, rel=1e-5)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_rules_infinities(spr, dtype):
    """-inf stays -inf under penalties; what a mask forbids is -inf whatever stood there; other bits go by."""
    x, dims = rules_case(1, 2, 300, dtype, seed=49, n_bias=0, masks=0)
    l = x["logits"].view(2, 300)
    l[:, 5], l[:, 6], l[:, 7], l[:, 8] = -math.inf, math.nan, math.inf, -0.0
    x["history"][:] = 5
    x["history_len"][:] = 3
    x["tokens"][:] = -1
    x["masks"] = torch.full((1, 10), -1, dtype=torch.int32)
    x["masks"][0, 0] = ~(1 << 6)
    x["mask_rows"] = torch.tensor([[0, -1]], dtype=torch.int32)
    got = run_rules(spr, x, dims).cpu()
    assert bool((got[0, :, 5] == -math.inf).all()) and got[0, 0, 6] == -math.inf and got[0, 1, 6].isnan() and bool((got[0, :, 7] == math.inf).all())
    assert math.copysign(1.0, float(got[0, 0, 8])) == -1.0


def test_rules_bad_tokens_and_rows(spr):
    for what, status in (("history", BAD_TOKEN), ("tokens", BAD_TOKEN), ("bias_tokens", BAD_TOKEN), ("mask_rows", BAD_ROW)):
        x, dims = rules_case(2, 3, 900, F32, seed=51)
        x["history_len"][:] = 30
        good, bad = dict(x), dict(x)
        good[what], bad[what] = x[what].clone(), x[what].clone()
        good[what][1, 2], bad[what][1, 2] = -1, 900
        want = run_rules(spr, good, dims)
        assert torch.equal(run_rules(spr, bad, dims, status=status), want), what


def test_rules_bad_tree(spr):
    x, dims = rules_case(1, 5, 400, F32, seed=53)
    x["parents"] = torch.tensor([[-1, 0, -1, 2, 3]], dtype=torch.int32)
    want = check_rules(spr, x, dims)
    x["parents"] = torch.tensor([[0, 0, 7, 2, 3]], dtype=torch.int32)
    x["tokens"][:] = torch.tensor([3, 3, 8, 3, 8])
    x["parents"][0, 0] = -1
    y = dict(x, parents=torch.tensor([[-1, 0, -1, 2, 3]], dtype=torch.int32))
    assert torch.equal(run_rules(spr, x, dims, status=BAD_TREE), run_rules(spr, y, dims))
    assert want.shape == (1, 5, 400)
