"""cache_append, tree_attention and logits_rules as a decoding loop uses them: one behind the other with the verification,
in captured graphs, and over the largest sizes.  Bounds in draft_pass_reference.py."""
import pytest
import torch

import draft_pass_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
I32 = torch.int32


@pytest.fixture(scope="module")
def spr():
    import paper_2502_04557_b200 as s
    s.lib()
    return s


def ids(x):
    return {BF16: "bf16", F32: "f32"}.get(x, str(x))


def workspace(spr, dtype, B=1, K=1, V=1, D=128):
    """One for all the calls of a pass."""
    from paper_2502_04557_b200 import binding
    dt = spr.F32 if dtype == F32 else spr.BF16
    ops = [(spr.OP_CACHE_APPEND, 1, 1, 1, D), (spr.OP_TREE_ATTENTION, 1, 1, 1, D), (spr.OP_LOGITS_RULES, 1, 1, 1, 1)]
    if V > 1:
        ops += [(binding.OP_SD_VERIFY, B, K, V, 1), (binding.OP_REPLACE_SAMPLE, B * (K + 1), K, V, 1)]
    return spr.Workspace(max(spr.workspace_bytes(op, b, k, v, d, 0, dt) for op, b, k, v, d in ops))


def freqs(pairs):
    return (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()


class Cache:
    """Pages of one layer and what a pass needs beside them."""

    def __init__(self, B, most, Hkv, D, page, dtype, g):
        table, pages = ref.make_pages(B, (most + page - 1) // page, 3, g)
        self.table = table.cuda()
        self.k = torch.randn((pages, Hkv, page, D), generator=g).to(dtype).cuda()
        self.v = torch.randn((pages, Hkv, page, D), generator=g).to(dtype).cuda()

    def rows(self, b, n):
        slot = torch.arange(n, device="cuda")
        page = self.k.shape[2]
        at = self.table[b].long()[slot // page]
        return self.k[at, :, slot % page], self.v[at, :, slot % page]


def attend_checked(spr, q, cache, lens, ws, counts=None, parents=None):
    out = spr.tree_attention(q, cache.k, cache.v, cache.table, lens, ws, counts=counts, parents=parents)
    want, tol = ref.attend(q, cache.k, cache.v, cache.table, lens.cpu(), None if counts is None else counts.cpu(),
                           None if parents is None else parents.cpu(), q.shape[-1] ** -0.5)
    assert ref.within(out, want, tol), ref.worst(out, want, tol)
    return out


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_a_pass_over_drafted_chains(spr, dtype):
    """The last token and K drafted ones go through the cache, the attention, a head, the rules and the verification; what
    was accepted is then the prefix of the next pass."""
    import oracle
    B, K, Hq, Hkv, D, V, page = 4, 5, 8, 2, 64, 3001, 16
    T, g = K + 1, torch.Generator().manual_seed(71)
    lens = torch.tensor([0, 15, 200, 61], dtype=I32).cuda()
    cache, f = Cache(B, 300, Hkv, D, page, dtype, g), freqs(D // 2).cuda()
    ws = workspace(spr, dtype, B, K, V)
    head = (torch.randn((Hq * D, V), generator=g) / 8).to(dtype).cuda()
    for step in range(3):
        both = torch.randn((B, T, Hq + 2 * Hkv, D), generator=g).to(dtype).cuda()
        tokens = torch.randint(0, V, (B, T), generator=g).to(I32).cuda()
        kv = cache.k.cpu(), cache.v.cpu()
        q = spr.cache_append(both[:, :, Hq:Hq + Hkv], both[:, :, Hq + Hkv:], cache.k, cache.v, cache.table, lens, ws, q=both[:, :, :Hq],
                             inv_freq=f)
        host = both.cpu()
        want, tol = ref.append(host[:, :, :Hq], host[:, :, Hq:Hq + Hkv], host[:, :, Hq + Hkv:], *kv, cache.table.cpu(), lens.cpu(), f.cpu(),
                               False, None, None, None)
        for a, b, t in zip((q, cache.k, cache.v), want, tol):
            assert ref.within(a.cpu(), b, t)
        o = attend_checked(spr, q, cache, lens, ws)
        logits = (o.reshape(B, T, Hq * D) @ head).contiguous()
        raw = logits.cpu()
        history = torch.randint(0, V, (B, 40), generator=g).to(I32).cuda()
        few = torch.tensor([40, 0, 17, 3], dtype=I32).cuda()
        pen = torch.tensor([[1.2, 0.1, 0.2], [1.0, 0.0, 0.0], [0.8, -0.1, 0.3], [1.5, 0.5, 0.0]]).cuda()
        masks = torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), generator=g).to(I32).cuda()
        rows = torch.randint(-1, 3, (B, T), generator=g).to(I32).cuda()
        p = spr.logits_rules(logits, V, ws, history=history, history_len=few, tokens=tokens, penalties=pen, masks=masks, mask_rows=rows,
                             out=logits)
        want, tol = ref.rules(raw, V, history.cpu(), few.cpu(), tokens.cpu(), None, None, pen.cpu(), None, None, masks.cpu(), rows.cpu())
        assert ref.within(p.cpu(), want, tol)
        draft = tokens[:, 1:].contiguous()
        q_logits = (p[:, :K].float() + torch.randn((B, K, V), generator=g).cuda()).nan_to_num(neginf=-30.0).to(dtype).contiguous()
        u = torch.rand((B, K + 1), generator=g)
        got = spr.sd_verify(p, q_logits, V, draft, u.cuda(), ws)
        as_np = (lambda t: t.cpu().view(torch.int16).numpy().view("uint16")) if dtype == BF16 else (lambda t: t.cpu().numpy())
        want = oracle.sd_verify(as_np(p), as_np(q_logits), V, draft.cpu().numpy(), u.numpy())
        assert got["accepted_len"].tolist() == want["accepted_len"].tolist()
        assert got["correction_token"].tolist() == want["correction_token"].tolist()
        lens = lens + 1 + got["accepted_len"]
    assert ws.device_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_a_tree_is_cut_back_to_one_path(spr, dtype):
    """Nodes of a tree are put behind the prefix and attended to; a path is taken and moved together by `slots`; the cache and
    the next attention are those of a sequence that only ever had that path."""
    B, T, Hq, Hkv, D, V, page = 3, 21, 4, 2, 64, 1500, 8
    g = torch.Generator().manual_seed(73)
    lens, f = torch.tensor([7, 0, 130], dtype=I32).cuda(), freqs(D // 2).cuda()
    cache, ws = Cache(B, 200, Hkv, D, page, dtype, g), workspace(spr, dtype, B, T - 1, V)
    counts, parents = torch.tensor([21, 9, 16], dtype=I32).cuda(), ref.make_tree(B, T, g, roots=0.05).cuda()
    q, k, v = (torch.randn((B, T, h, D), generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
    alone = [cache.k.clone(), cache.v.clone()]
    qr = spr.cache_append(k, v, cache.k, cache.v, cache.table, lens, ws, q=q, inv_freq=f, counts=counts, parents=parents)
    o = attend_checked(spr, qr, cache, lens, ws, counts, parents)
    logits = torch.randn((B, T, V), generator=g).to(dtype).cuda()
    tokens = torch.randint(0, V, (B, T), generator=g).to(I32).cuda()
    pen = torch.tensor([[1.3, 0.2, 0.1]]).repeat(B, 1).cuda()
    p = spr.logits_rules(logits, V, ws, tokens=tokens, parents=parents, counts=counts, penalties=pen)
    want, tol = ref.rules(logits.cpu(), V, None, None, tokens.cpu(), parents.cpu(), counts.cpu(), pen.cpu(), None, None, None, None)
    assert ref.within(p.cpu(), want, tol)
    drawn = spr.replace_sample(p, V, torch.rand(B * T, generator=g).cuda(), ws)
    assert bool(((drawn >= 0) & (drawn < V)).all())
    # the deepest node's path is taken
    slots, deep = torch.full((B, T), -1, dtype=I32), []
    for b in range(B):
        paths = [ref.path(parents[b].tolist(), i)[::-1] for i in range(int(counts[b]))]
        deep.append(max(paths, key=len))
        for at, node in enumerate(deep[b]):
            slots[b, node] = int(lens[b]) + at
    spr.cache_append(k, v, cache.k, cache.v, cache.table, lens, ws, inv_freq=f, counts=counts, parents=parents, slots=slots.cuda())
    # the same sequences, path by path
    other = Cache.__new__(Cache)
    other.k, other.v, other.table = alone[0], alone[1], cache.table
    for b in range(B):
        one = slice(b, b + 1)
        at = torch.tensor(deep[b], device="cuda")
        qb = spr.cache_append(k[one, at], v[one, at], other.k, other.v, other.table[one], lens[one], ws, q=q[one, at], inv_freq=f)
        n = int(lens[b]) + len(deep[b])
        for x, y in zip(cache.rows(b, n), other.rows(b, n)):
            assert torch.equal(x, y)
        # a node's queries are those of its position in the chain
        assert torch.equal(qb[0], qr[b, at])
    lens = lens + torch.tensor([len(d) for d in deep], dtype=I32).cuda()
    nxt = [torch.randn((B, 1, h, D), generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv)]
    res = []
    for c in (cache, other):
        qn = spr.cache_append(nxt[1], nxt[2], c.k, c.v, c.table, lens, ws, q=nxt[0], inv_freq=f)
        res.append(attend_checked(spr, qn, c, lens, ws))
    assert torch.equal(*res) and ws.device_status() == 0
    assert bool((o[1, 9:] == 0).all()) and bool((o[2, 16:] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("T,G", [(1, 4), (3, 4), (9, 4)])
def test_captured_passes_share_a_workspace(spr, dtype, T, G):
    """Two graphs, of two layers, over one workspace; lengths, counts and pages change between replays, and each replay gives
    what calls from the host give."""
    B, Hkv, D, V, page = 5, 2, 128, 777, 16
    g = torch.Generator().manual_seed(75 + T)
    ws, f = workspace(spr, dtype), freqs(D // 2).cuda()
    lens, counts = torch.zeros(B, dtype=I32).cuda(), torch.full((B,), T, dtype=I32).cuda()
    parents = torch.full((B, T), -1, dtype=I32).cuda()
    tokens = torch.randint(0, V, (B, T), generator=g).to(I32).cuda()
    pen = torch.tensor([[1.3, 0.2, 0.1]]).repeat(B, 1).cuda()
    layers = []
    for _ in range(2):
        c = Cache(B, 4000, Hkv, D, page, dtype, g)
        x = [torch.randn((B, T, h, D), generator=g).to(dtype).cuda() for h in (Hkv * G, Hkv, Hkv)]
        logits = torch.randn((B, T, V), generator=g).to(dtype).cuda()
        layers.append((c, x, logits))

    def run(c, x, logits, w):
        q = spr.cache_append(x[1], x[2], c.k, c.v, c.table, lens, w, q=x[0], inv_freq=f, counts=counts, parents=parents)
        o = spr.tree_attention(q, c.k, c.v, c.table, lens, w, counts=counts, parents=parents)
        return o, spr.logits_rules(logits, V, w, tokens=tokens, parents=parents, counts=counts, penalties=pen)

    graphs, outs = [], []
    for layer in layers:
        run(*layer, ws)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(run(*layer, ws))
        graphs.append(gr)
    own = workspace(spr, dtype)
    for at, (ll, cc) in enumerate([([0, 1, 64, 3990, 17], [T] * 5), ([3000, -1, 63, 2, 900], [T, T, 0, 1, T]), ([5] * 5, [T] * 5)]):
        lens.copy_(torch.tensor(ll, dtype=I32))
        counts.copy_(torch.tensor(cc, dtype=I32))
        parents.copy_(ref.make_tree(B, T, g))
        for c, x, logits in layers:
            c.table.copy_(c.table[:, torch.randperm(c.table.shape[1], generator=g).cuda()])
            for t in (*x, logits):
                t.copy_(torch.randn(t.shape, generator=g).to(dtype))
        for i in (0, 1, 1, 0) if at else (1, 0):
            graphs[i].replay()
            got = [t.clone() for t in outs[i]]
            kv = layers[i][0].k.clone(), layers[i][0].v.clone()
            want = run(*layers[i], own)
            for a, b in zip((*got, *kv), (*want, layers[i][0].k, layers[i][0].v)):
                assert torch.equal(a, b)
    c, x, _ = layers[0]
    q = spr.cache_append(x[1], x[2], c.k, c.v, c.table, lens, ws, q=x[0], inv_freq=f, counts=counts, parents=parents)
    attend_checked(spr, q, c, lens, ws, counts, parents)
    assert ws.device_status() == 0 and own.device_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_two_passes_at_once(spr, dtype):
    """Two streams with a workspace each, many calls in flight: as one after the other."""
    g = torch.Generator().manual_seed(79)
    cases = []
    for B, T, n in ((3, 2, 9000), (2, 12, 3000)):
        c = Cache(B, n + T, 2, 128, 16, dtype, g)
        q = torch.randn((B, T, 8, 128), generator=g).to(dtype).cuda()
        lens = torch.tensor([n] + [n // 7] * (B - 1), dtype=I32).cuda()
        cases.append((q, c, lens, workspace(spr, dtype)))
    want = [spr.tree_attention(q, c.k, c.v, c.table, l, w) for q, c, l, w in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(10):
        for i, (q, c, l, w) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(spr.tree_attention(q, c.k, c.v, c.table, l, w))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, want[i]) for o in got[i]) and cases[i][3].device_status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
@pytest.mark.parametrize("B,T,lens", [(700, 1, 40), (400, 3, 9), (333, 20, 3), (2, 256, 70), (1, 256, 2500)])
def test_many_sequences_and_nodes(spr, dtype, B, T, lens):
    g = torch.Generator().manual_seed(B + T)
    Hq, Hkv, D = 4, 2, 64
    c, ws = Cache(B, lens + T + 1, Hkv, D, 16, dtype, g), workspace(spr, dtype)
    n = torch.randint(-1, lens + 1, (B,), generator=g).to(I32).cuda()
    counts, parents = torch.randint(0, T + 1, (B,), generator=g).to(I32).cuda(), ref.make_tree(B, T, g).cuda()
    q, k, v = (torch.randn((B, T, h, D), generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
    kv, f = (c.k.cpu(), c.v.cpu()), freqs(D // 2).cuda()
    qr = spr.cache_append(k, v, c.k, c.v, c.table, n, ws, q=q, inv_freq=f, counts=counts, parents=parents)
    want, tol = ref.append(q.cpu(), k.cpu(), v.cpu(), *kv, c.table.cpu(), n.cpu(), f.cpu(), False, counts.cpu(), parents.cpu(), None)
    for a, b, t in zip((qr, c.k, c.v), want, tol):
        assert ref.within(a.cpu(), b, t)
    attend_checked(spr, qr, c, n, ws, counts, parents)
    logits = torch.randn((B, T, 300), generator=g).to(dtype)
    tokens, pen = torch.randint(0, 40, (B, T), generator=g).to(I32), torch.rand((B, 3), generator=g) + 0.5
    got = spr.logits_rules(logits.cuda(), 300, ws, tokens=tokens.cuda(), parents=parents, counts=counts, penalties=pen.cuda())
    want, tol = ref.rules(logits, 300, None, None, tokens, parents.cpu(), counts.cpu(), pen, None, None, None, None)
    assert ref.within(got.cpu(), want, tol) and ws.device_status() == 0


@pytest.mark.parametrize("T", [1, 20])
def test_cache_of_more_than_2_31_entries(spr, T):
    """Pages whose first entries lie behind 2^31."""
    B, Hq, Hkv, D, page = 2, 8, 2, 128, 64
    pages, g = (1 << 31) // (Hkv * page * D) + 40, torch.Generator().manual_seed(81)
    c = Cache.__new__(Cache)
    c.k = torch.empty((pages, Hkv, page, D), dtype=BF16, device="cuda")
    c.v = torch.empty((pages, Hkv, page, D), dtype=BF16, device="cuda")
    c.table = torch.stack([torch.arange(pages - 16, pages), torch.cat([torch.arange(8), torch.arange(pages - 24, pages - 16)])]).to(I32).cuda()
    for at in (slice(0, 8), slice(pages - 24, pages)):
        c.k[at], c.v[at] = (torch.randn(c.k[at].shape, generator=g).to(BF16).cuda() for _ in range(2))
    lens, ws = torch.tensor([900, 700], dtype=I32).cuda(), workspace(spr, BF16)
    q, k, v = (torch.randn((B, T, h, D), generator=g).to(BF16).cuda() for h in (Hq, Hkv, Hkv))
    spr.cache_append(k, v, c.k, c.v, c.table, lens, ws)
    for b in range(B):
        n = int(lens[b])
        kr, vr = c.rows(b, n + T)
        assert torch.equal(kr[n:], k[b]) and torch.equal(vr[n:], v[b])
    attend_checked(spr, q, c, lens, ws)
    assert ws.device_status() == 0


def test_logits_of_more_than_2_31_entries(spr):
    B, T, V, g = 130, 127, 131072, torch.Generator().manual_seed(83)
    logits, ws = torch.zeros((B, T, V), dtype=BF16, device="cuda"), workspace(spr, BF16)
    tokens = torch.full((B, T), V - 1, dtype=I32).cuda()
    pen = torch.tensor([[1.0, 0.5, 2.0]]).repeat(B, 1).cuda()
    spr.logits_rules(logits, V, ws, tokens=tokens, penalties=pen, out=logits)
    want = -(0.5 * torch.arange(1, T + 1) + 2.0).to(BF16)
    assert torch.equal(logits[:, :, -1].cpu(), want[None].expand(B, T))
    assert not bool(logits[-1, :, :-1].any()) and not bool(logits[0, :, :-1].any()) and ws.device_status() == 0
