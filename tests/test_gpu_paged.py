"""The paged key/value cache on the GPU against plain 64-bit forms: storing, attention over the pages with the weights that
cached tokens receive, eviction, and the decoder block that uses them.  Slots that hold no token hold NaN."""
import numpy as np
import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2512_16843_amd import llmc
    assert torch.cuda.is_available(), "these tests need the GPU"
    llmc.lib()
    return llmc


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def starts_of(news):
    s = [0]
    for q in news:
        s.append(s[-1] + q)
    return s


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Inputs of one attention call, made on the CPU, and the call."""

    def __init__(self, L, dtype, H, kv, dh, page, lens, news, seed=0, softcap=0.0, window=0, slopes=False, weights=False,
                 moved=False, spread=1.5, max_len=None, behind=0):
        g = torch.Generator().manual_seed(seed)
        self.L, self.lens, self.news = L, lens, news
        self.k, self.v, self.table = R.make_cache(g, DT[dtype], kv, dh, page, lens)
        self.starts = starts_of(news)
        rows = self.starts[-1] + behind
        self.q = (spread * torch.randn((rows, H, dh), generator=g)).to(DT[dtype])
        self.slots = self.table.shape[1] * page
        self.pos = None
        if moved:       # as after evictions: positions with gaps, the older tokens in no order
            p = torch.randint(1, 4, (len(lens), self.slots), generator=g).cumsum(1) - 1
            for b, n in enumerate(lens):
                old = max(0, n - news[b])
                p[b, :old] = p[b, :old][torch.randperm(old, generator=g)]
            self.pos = p.to(torch.int32)
        self.slopes = (2.0 ** (-8.0 * torch.arange(1, H + 1) / H)).float() if slopes else None
        self.weight = torch.rand((len(lens), self.slots), generator=g) if weights else None
        self.opt = dict(softcap=softcap, window=window)
        self.max_len = max(max(lens), 1) if max_len is None else max_len
        self.max_new = max(max(news), 1)

    def gpu(self, decode=False, stream=None, ws=None, out=None):
        c = lambda t: None if t is None else t.cuda()
        self.w_gpu = c(self.weight)
        q = c(self.q)
        if out is None:
            out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        tab, kp, vp = c(self.table), c(self.k), c(self.v)
        n = self.L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=self.max_new, max_len=self.max_len,
                                                        weights=self.weight is not None)
        if ws is None:
            ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        self.L.llmc_attention_paged(q, kp, vp, tab, i32(self.lens), out, ws,
                                    new_start=None if decode else i32(self.starts), max_new=self.max_new,
                                    max_len=self.max_len, pos=c(self.pos), weight=self.w_gpu, slopes=c(self.slopes),
                                    **self.opt)
        torch.cuda.synchronize()
        return out.cpu()

    def check(self, got, **more):
        want, tol, ws, wt = R.attention(self.q, self.k, self.v, self.table, self.lens, self.starts, pos=self.pos,
                                        slopes=self.slopes, **self.opt, **more)
        end = self.starts[-1]
        bad = (got[:end].double() - want[:end]).abs() - tol[:end]
        assert torch.isfinite(got[:end].double()).all()
        assert bad.numel() == 0 or bad.max() <= 0, (bad.max(), (bad > 0).sum(), np.unravel_index(int(bad.argmax()), bad.shape))
        assert (got[end:] == 7.0).all()                       # rows of no sequence are left as they were
        if self.weight is not None:
            w = self.w_gpu.cpu().double()
            for b, n in enumerate(self.lens):
                add = w[b] - self.weight[b].double()
                slack = wt[b] + 2.0 ** -23 * (self.weight[b, :n].double() + ws[b])
                assert ((add[:n] - ws[b]).abs() <= slack).all(), (b, ((add[:n] - ws[b]).abs() / slack).max())
                assert (add[n:] == 0).all()


DECODE_LENS = [
    [1],
    [16, 17, 31, 32, 33],
    [777, 1, 128, 129, 300, 255, 257],
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh,page", [(12, 12, 64, 16), (8, 2, 128, 64), (6, 2, 64, 32), (16, 1, 128, 16), (1, 1, 64, 1024)])
@pytest.mark.parametrize("lens", DECODE_LENS, ids=lambda l: "n%d" % max(l))
def test_single_tokens(L, dtype, heads, kv, dh, page, lens):
    c = Case(L, dtype, heads, kv, dh, page, lens, [1] * len(lens), seed=len(lens) + heads, weights=True)
    c.check(c.gpu(decode=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("opts", [
    dict(softcap=5.0), dict(slopes=True), dict(window=1), dict(window=50), dict(window=100000), dict(window=2 ** 31 - 1),
    dict(softcap=30.0, slopes=True, window=70), dict(slopes=True, moved=True), dict(window=90, moved=True),
], ids=lambda o: "-".join("%s%s" % kv for kv in o.items()))
@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
def test_single_tokens_score_options(L, dtype, opts, weights):
    lens = [333, 64, 1, 200]
    c = Case(L, dtype, 8, 4, 64, 16, lens, [1] * 4, seed=5, weights=weights, **opts)
    c.check(c.gpu(decode=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh", [(4, 1, 64), (8, 8, 128)])
def test_single_tokens_over_a_long_cache_in_pieces(L, dtype, heads, kv, dh):
    lens = [5000, 4095, 256, 257, 513]
    c = Case(L, dtype, heads, kv, dh, 128, lens, [1] * 5, seed=2, weights=True)
    c.check(c.gpu(decode=True))


CHUNKS = [
    ([1, 1], [1, 1]),
    ([2, 9, 5], [2, 3, 5]),                     # up to 16 rows a head
    ([40, 17, 128], [17, 17, 16]),
    ([300, 64, 65, 1], [130, 64, 1, 1]),
    ([129, 0, 500, 7], [129, 0, 33, 0]),        # a sequence without tokens, one without new ones
    ([1100], [257]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh,page", [(2, 2, 64, 16), (6, 2, 128, 32)])
@pytest.mark.parametrize("lens,news", CHUNKS, ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
def test_chunks(L, dtype, heads, kv, dh, page, lens, news, weights):
    c = Case(L, dtype, heads, kv, dh, page, lens, news, seed=sum(lens), weights=weights, behind=3)
    c.check(c.gpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("opts", [
    dict(softcap=5.0), dict(slopes=True), dict(window=1), dict(window=37), dict(window=2 ** 31 - 1),
    dict(softcap=30.0, slopes=True, window=150), dict(slopes=True, moved=True), dict(window=90, moved=True),
], ids=lambda o: "-".join("%s%s" % kv for kv in o.items()))
def test_chunks_score_options(L, dtype, dh, opts):
    c = Case(L, dtype, 4, 2, dh, 16, [700, 65, 200, 31], [200, 65, 3, 20], seed=9, weights=True, **opts)
    c.check(c.gpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_short_chunk_over_a_long_cache_in_pieces(L, dtype):
    c = Case(L, dtype, 4, 2, 128, 64, [6000, 100], [70, 30], seed=3, weights=True, window=5500)
    c.check(c.gpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_cross_a_wavefront_of_starts(L, dtype):
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 50, 150)]
    news = [int(rng.integers(0, n + 1)) for n in lens]
    c = Case(L, dtype, 3, 1, 64, 16, lens, news, seed=4, weights=True)
    c.check(c.gpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [40, 25]])
def test_tokens_that_see_nothing_give_zeros(L, dtype, news):
    """Fewer tokens in the cache than are said to be new: the rows in front stand before the first slot."""
    c = Case(L, dtype, 2, 2, 64, 16, [20, 0], news, seed=1, weights=True, max_len=48)
    got = c.gpu()
    assert torch.isfinite(got.double()).all()
    want, tol, _, _ = R.attention(c.q, c.k, c.v, c.table, c.lens, c.starts)
    assert ((got.double() - want).abs() <= tol).all()
    assert (got[c.starts[1]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [30, 3, 40]])
def test_scores_at_the_ends_of_the_range(L, dtype, news):
    """Large scores: one key takes everything; equal scores: the mean of the values."""
    c = Case(L, dtype, 2, 1, 64, 16, [100, 33, 64], news, seed=6, spread=200.0, weights=True)
    c.check(c.gpu())
    c.q.zero_()
    c.check(c.gpu())


@pytest.mark.parametrize("dtype,weights", [("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("softcap", [1.0, 50.0, 2000.0, 1e6])
@pytest.mark.parametrize("news", [[1, 1], [200, 40]])
def test_capping_is_exact_however_far_the_cap(L, dtype, weights, softcap, news):
    """Roundings of tanh(z), z = x / cap, in half steps f = 2^-24 relative to the result, |z| >= 0.45, E = e^(-2 |z|) <= 0.41:
    z itself 2 (its factor t' z / t is below one), the exponent 1 + 1 more of 2 |z| and the exponential 2 on E, all of them scaled by
    2 E / (1 - E^2) <= 1 and |z| E small; 1 - E, 1 + E, the product 1 each, the reciprocal 2: below 12.  Below 0.45 the series: z 2,
    six fmas whose errors shrink with z^2, the last one whole, the first term left out 2 * 10^-8 = 0.34 f: fewer.  Back to a score in base 2:
    two more.  Only bf16 chunks round more coarsely, 2^-23 of the cap: up to a cap of 1024, where they leave no weights, or 64."""
    fast = dtype == "bf16" and sum(news) > 32 and softcap <= (64 if weights else 1024)
    c = Case(L, dtype, 4, 2, 64, 16, [333, 64], news, seed=8, weights=weights, softcap=softcap)
    c.check(c.gpu(), cap_rel=None if fast else 16 * 2.0 ** -24)


def test_more_blocks_of_a_chunk_than_lanes(L):
    c = Case(L, "bf16", 6, 1, 64, 64, [1500, 1400], [1400, 3], seed=10)     # 8400 rows a head: 66 blocks of 128
    c.check(c.gpu())


@pytest.mark.parametrize("news", [1, 20])
def test_lengths_outside_their_bounds_are_cut(L, news):
    """Many sequences, some of whose lengths are negative or beyond max_len."""
    g = torch.Generator().manual_seed(12)
    lens = [int(x) for x in torch.randint(news, 49, (70,), generator=g)]
    c = Case(L, "bf16", 4, 4, 64, 16, lens, [news] * 70, seed=11, max_len=48)
    wrong = list(lens)
    for b in (0, 3, 69):
        lens[b], wrong[b] = 0, -5 - b
    full = lens.index(48)
    wrong[full] = 10 ** 6
    c.lens = wrong
    got = c.gpu(decode=news == 1)
    c.lens = lens
    c.check(got)
    for b in (0, 3, 69):
        assert (got[c.starts[b]:c.starts[b + 1]] == 0).all()


def test_starts_that_fall_store_nothing_before_a_sequence(L):
    g = torch.Generator().manual_seed(13)
    k, v, table = R.make_cache(g, torch.float32, 2, 64, 16, [20, 20], fill=0.0)
    new = torch.randn((6, 2, 64), generator=g)
    kg, vg = k.cuda(), v.cuda()
    L.llmc_kv_append(new.cuda(), new.cuda(), kg, vg, table.cuda(), i32([20, 20]), new_start=i32([3, 0, 6]), max_new=6)
    torch.cuda.synchronize()
    for got, was in ((kg, k), (vg, v)):
        assert torch.equal(R.tokens(got.cpu(), table, 0, 20), R.tokens(was, table, 0, 20))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,lens", [(40, [300, 1, 64]), (130, [int(n) for n in range(1, 71)])])
def test_single_tokens_of_many_heads_on_one_key(L, dtype, heads, lens):
    c = Case(L, dtype, heads, 1, 64, 16, lens, [1] * len(lens), seed=heads, weights=True)
    c.check(c.gpu(decode=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,decode", [(1, True), (1, False), (5, False)])
def test_more_sequences_than_lanes_in_pieces(L, dtype, new, decode):
    """70 sequences that share one key/value head, two of them long: their axis is cut."""
    lens = [40 + 3 * i for i in range(70)]
    lens[7], lens[66] = 3000, 1999
    c = Case(L, dtype, 4, 1, 64, 16, lens, [new] * 70, seed=15, weights=True)
    c.check(c.gpu(decode=decode))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 3, 100]])
def test_a_pool_beyond_32_bits(L, dtype, news):
    """The same pages at the end of a pool of more than 2^32 elements, and at its start: the same bits."""
    g = torch.Generator().manual_seed(14)
    lens, kv, dh, page = [120, 33, 200], 4, 64, 64
    k, v, table = R.make_cache(g, DT[dtype], kv, dh, page, lens)
    far = 2 ** 32 // (kv * dh * page) + 5
    starts = starts_of(news)
    q = torch.randn((starts[-1], kv, dh), generator=g).to(DT[dtype]).cuda()
    slots = table.shape[1] * page
    pos0 = torch.arange(slots, dtype=torch.int32).repeat(3, 1)
    res = []
    for shift in (0, far):
        kp = torch.empty((k.shape[0] + shift, kv, page, dh), dtype=k.dtype, device="cuda")
        vp = torch.empty_like(kp)
        kp[shift:], vp[shift:] = k.cuda(), v.cuda()
        tab = (table + shift).cuda()
        pos, w = pos0.cuda(), torch.zeros((3, slots), device="cuda")
        kw = dict(new_start=i32(starts), max_new=max(news))
        L.llmc_kv_append(q, q, kp, vp, tab, i32(lens), pos=pos, weight=w, **kw)
        ws = torch.empty((L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=max(news), max_len=200, weights=True),),
                         dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        L.llmc_attention_paged(q, kp, vp, tab, i32(lens), out, ws, max_len=200, weight=w, **kw)
        left = i32([0, 0, 0])
        ws = torch.empty((L.llmc_kv_evict_workspace_bytes(tab, 200),), dtype=torch.uint8, device="cuda")
        L.llmc_kv_evict(kp, vp, tab, i32(lens), pos, w, i32([50, 30, 20]), left, ws, max_len=200, recent=10)
        torch.cuda.synchronize()
        res.append([out.cpu(), w.cpu(), pos.cpu(), left.cpu()] + [R.tokens(p[shift:].cpu(), table, b, n)
                                                                  for p in (kp, vp) for b, n in enumerate([50, 30, 20])])
        del kp, vp
    assert torch.isfinite(res[0][0].double()).all()
    assert all(torch.equal(x, y) for x, y in zip(*res))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,vpr", [(1, 1), (7, 2), (64, 12)])
@pytest.mark.parametrize("dh,page", [(64, 16), (128, 64)])
def test_append(L, dtype, new, vpr, dh, page):
    kv = vpr
    g = torch.Generator().manual_seed(new)
    lens = [new, 3 * new + 5, 100 + new, 16 + new]
    news = [new, max(1, new - 2), new, 0 if new > 1 else 1]
    k, v, table = R.make_cache(g, DT[dtype], kv, dh, page, lens, fill=0.5)
    starts = starts_of(news)
    rows = starts[-1] + (2 if new > 1 else 0)
    qkv = torch.randn((rows, 3 * kv, dh), generator=g).to(DT[dtype])
    slots = table.shape[1] * page
    pos = torch.full((4, slots), -5, dtype=torch.int32)
    weight = torch.rand((4, slots), generator=g)
    pn = torch.arange(rows, dtype=torch.int32) * 3
    kg, vg, tg, pg, wg, qg = (t.cuda() for t in (k, v, table, pos, weight, qkv))
    for given in (pn, None):
        L.llmc_kv_append(qg[:, kv:2 * kv], qg[:, 2 * kv:], kg, vg, tg, i32(lens), new_start=None if new == 1 else i32(starts),
                         max_new=new, pos_new=None if given is None else given.cuda(), pos=pg, weight=wg)
        torch.cuda.synchronize()
        for b in range(4):
            for i in range(news[b]):
                s, r = lens[b] - news[b] + i, starts[b] + i
                p = int(table[b, s // page])
                k[p, :, s % page], v[p, :, s % page] = qkv[r, kv:2 * kv], qkv[r, 2 * kv:]
                pos[b, s], weight[b, s] = (s if given is None else int(given[r])), 0.0
        for got, want in ((kg, k), (vg, v), (pg, pos), (wg, weight)):
            assert torch.equal(got.cpu(), want)


EVICT = [
    # lens, keep, sink, recent
    ([5, 1, 9], [3, 1, 0], 0, 0),
    ([100, 40, 64, 0], [99, 50, 32, 4], 4, 8),
    ([1030, 2049, 17], [1024, 100, 16], 4, 32),
    ([1500, 1500], [700, 701], 0, 2000),          # everything is protected
    ([3000], [1], 1, 0),
    ([64, 64], [-3, 0], 2, 2),
    ([65, 128, 5000], [64, 64, 4999], 0, 0),
    ([8192, 8193, 66], [2000, 8192, 1], 4, 100),
    ([20000, 33000], [15000, 16000], 16, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "same"])
@pytest.mark.parametrize("lens,keep,sink,recent", EVICT, ids=lambda x: "-".join(map(str, x)) if isinstance(x, list) else str(x))
def test_evict(L, dtype, kind, lens, keep, sink, recent):
    kv, dh, page = 3, 64 if dtype == "bf16" else 128, 16
    g = torch.Generator().manual_seed(sum(lens))
    k, v, table = R.make_cache(g, DT[dtype], kv, dh, page, lens, fill=0.25)
    slots = table.shape[1] * page
    B = len(lens)
    pos = torch.stack([torch.randperm(3 * slots, generator=g)[:slots] for _ in range(B)]).to(torch.int32)
    weight = torch.exp(2 * torch.randn((B, slots), generator=g))
    if kind == "ties":
        weight = torch.randint(0, 3, (B, slots), generator=g).float()
    if kind == "same":           # positions that repeat are not promised to be sensible, but the order is: by slot
        weight.fill_(0.5)
        pos //= 1000
    if kind == "odd":
        for x, every in ((float("nan"), 7), (float("inf"), 5), (-1.0, 3), (-0.0, 4), (0.0, 11)):
            weight[:, ::every] = x
    kg, vg, tg, pg, wg = (t.cuda() for t in (k, v, table, pos, weight))
    out = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ml = max(max(lens), 1)
    ws = torch.full((L.llmc_kv_evict_workspace_bytes(tg, ml),), 255, dtype=torch.uint8, device="cuda")
    L.llmc_kv_evict(kg, vg, tg, i32(lens), pg, wg, i32(keep), out, ws, max_len=ml, sink=sink, recent=recent)
    torch.cuda.synchronize()
    want_len = []
    for b, n in enumerate(lens):
        moves, left = R.evict(pos[b].tolist(), weight[b].tolist(), n, keep[b], sink, recent)
        want_len.append(left)
        for s, d in moves:
            ps, pd = int(table[b, s // page]), int(table[b, d // page])
            k[pd, :, d % page], v[pd, :, d % page] = k[ps, :, s % page], v[ps, :, s % page]
            pos[b, d], weight[b, d] = pos[b, s], weight[b, s]
    assert out.tolist() == want_len
    assert torch.equal(pg.cpu(), pos)
    assert torch.equal(wg.cpu().view(torch.int32), weight.view(torch.int32))
    assert torch.equal(kg.cpu(), k) and torch.equal(vg.cpu(), v)


# ---- together, as a decoder uses them ------------------------------------------------------------------------------

TOL = {"f32": 1e-4, "bf16": 2e-2}          # the bars of the dense block's parity tests, relative to the row's largest value


def small_decoder(dtype, n_layers=2, S=96):
    from paper_2512_16843_amd import workloads as W
    cfg = W.scaled(W.TINY_ENCODER, arch=1, n_layers=n_layers, S=S, dtype=dtype)
    return W, cfg, W.make_layer_weights(cfg, seed=0)


def oracle_outputs(cfg, ws, h):
    from oracle import llmc_oracle as O
    x = h.double().numpy()
    for w in ws:
        wn = {k: v.float().numpy() for k, v in w.items()}
        x = O.layer_forward(x, wn, 1, cfg.n_heads, cfg.ln_eps, cfg.gelu)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_in_chunks_equals_the_whole(L, dtype):
    """Prompts, chunks and single tokens of three sequences through the stack: each token's output is that of the oracle's
    decoder on the whole sequence."""
    from paper_2512_16843_amd.engine import PagedStack
    W, cfg, ws = small_decoder(dtype)
    g = torch.Generator().manual_seed(0)
    seqs = [torch.randn((n, cfg.d), generator=g).to(cfg.torch_dtype) for n in (96, 50, 1)]
    st = PagedStack(cfg, ws, 3, 96, page_size=16, n_pages=6 + 4 + 1)
    plan = [[40, 0, 1], [1, 30, 0], [33, 20, 0], [1, 0, 0], [21, 0, 0]]
    at, got = [0, 0, 0], [[], [], []]
    for new in plan:
        rows = torch.cat([s[a:a + q] for s, a, q in zip(seqs, at, new)]).cuda()
        out = st.extend(rows, new).cpu()
        r = 0
        for b, q in enumerate(new):
            got[b].append(out[r:r + q])
            r += q
            at[b] += q
    assert st.lengths == [96, 50, 1] and not st.free
    for s, o in zip(seqs, got):
        want = oracle_outputs(cfg, ws, s)
        o = torch.cat(o).double().numpy()
        err = np.abs(o - want).max(axis=1) / np.abs(want).max(axis=1)
        assert err.max() < TOL[dtype], err.max()
    with pytest.raises(ValueError):
        st.extend(torch.zeros((1, cfg.d), dtype=cfg.torch_dtype, device="cuda"), [1, 0, 0])      # beyond max_len
    with pytest.raises(ValueError):
        st.extend(torch.zeros((20, cfg.d), dtype=cfg.torch_dtype, device="cuda"), [0, 0, 20])    # no pages left
    st.release(0)
    assert st.extend(torch.zeros((20, cfg.d), dtype=cfg.torch_dtype, device="cuda"), [0, 0, 20]).shape == (20, cfg.d)


def test_a_budget_keeps_what_was_attended_to(L):
    """One layer in fp32: after each step the cache holds the tokens that plain 64-bit bookkeeping keeps."""
    from paper_2512_16843_amd.engine import PagedStack
    from oracle import llmc_oracle as O
    W, cfg, ws = small_decoder("f32", n_layers=1)
    g = torch.Generator().manual_seed(3)
    budget, sink, recent = 24, 2, 6
    st = PagedStack(cfg, ws, 2, 64, page_size=16, budget=budget, sink=sink, recent=recent)
    w = {k: v.double() for k, v in ws[0].items()}
    H, dh = cfg.n_heads, 64
    cache = [[], []]                                    # per sequence: [position, weight, k [H, dh], v [H, dh]] in slot order
    seen = [0, 0]
    for new in ([30, 20], [1, 1], [1, 9], [3, 0], [1, 1]):
        h = torch.randn((sum(new), cfg.d), generator=g)
        st.extend(h.cuda(), new)
        x = h.double()
        mu = x.mean(1, keepdim=True)
        y = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + cfg.ln_eps) * w["ln1_g"] + w["ln1_b"]
        q, k, v = (y @ w["wqkv"].t() + w["bqkv"]).reshape(-1, 3, H, dh).unbind(1)
        r = 0
        for b, n in enumerate(new):
            for i in range(n):
                cache[b].append([seen[b] + i, 0.0, k[r + i], v[r + i]])
            seen[b] += n
            K = torch.stack([c[2] for c in cache[b]])
            for i in range(n):
                upto = len(cache[b]) - n + i + 1
                s = torch.einsum("hd,khd->hk", q[r + i], K[:upto]) * dh ** -0.5
                p = torch.softmax(s, 1).sum(0)
                for j in range(upto):
                    cache[b][j][1] += float(p[j])
            r += n
            moves, left = R.evict([c[0] for c in cache[b]], [c[1] for c in cache[b]], len(cache[b]), budget, sink, recent)
            for s_, d_ in moves:
                cache[b][d_] = list(cache[b][s_])
            cache[b] = cache[b][:left]
        assert st.lengths == [len(c) for c in cache]
        for b in range(2):
            n = len(cache[b])
            assert st.pos[0][b, :n].tolist() == [c[0] for c in cache[b]]
            assert np.allclose(st.weight[0][b, :n].cpu().numpy(), [c[1] for c in cache[b]], rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("heads,kv,dh", [(4, 4, 64), (8, 2, 128)])
def test_a_recorded_step_is_replayed(L, heads, kv, dh):
    """Append, attention with weights, and eviction of one decoding step recorded once; each replay, on other inputs and with
    eager work and synchronisation between, equals the eager step."""
    g = torch.Generator().manual_seed(1)
    lens = [300, 17, 1, 280]
    k, v, table = R.make_cache(g, torch.bfloat16, kv, dh, 16, [n + 40 for n in lens], fill=0.0)
    slots = table.shape[1] * 16

    def state():
        return dict(k=k.cuda(), v=v.cuda(), table=table.cuda(), length=i32(lens), pos=torch.arange(slots).repeat(4, 1).int().cuda(),
                    weight=torch.zeros((4, slots), device="cuda"), keep=i32([290, 100, 100, 290]), new_len=i32([0] * 4),
                    qkv=torch.zeros((4, heads + 2 * kv, dh), dtype=torch.bfloat16, device="cuda"), pos_new=i32(lens),
                    out=torch.zeros((4, heads, dh), dtype=torch.bfloat16, device="cuda"))

    def step(s, ws, ws2):
        s["length"] += 1
        q, kn, vn = s["qkv"].split([heads, kv, kv], 1)
        L.llmc_kv_append(kn, vn, s["k"], s["v"], s["table"], s["length"], pos_new=s["pos_new"], pos=s["pos"], weight=s["weight"])
        L.llmc_attention_paged(q, s["k"], s["v"], s["table"], s["length"], s["out"], ws, max_len=320, pos=s["pos"],
                               weight=s["weight"], window=250)
        L.llmc_kv_evict(s["k"], s["v"], s["table"], s["length"], s["pos"], s["weight"], s["keep"], s["new_len"], ws2,
                        max_len=320, sink=2, recent=8)
        s["length"].copy_(s["new_len"])
        s["pos_new"] += 1

    a, b = state(), state()
    q0 = a["qkv"][:, :heads]
    nb = L.llmc_attention_paged_workspace_bytes(q0, a["k"], a["table"], max_len=320, weights=True)
    wss = [(torch.empty((nb,), dtype=torch.uint8, device="cuda"),
            torch.empty((L.llmc_kv_evict_workspace_bytes(a["table"], 320),), dtype=torch.uint8, device="cuda")) for _ in range(2)]
    warm = state()
    step(warm, *wss[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, *wss[0])
    for i in range(20):
        x = torch.randn((4, heads + 2 * kv, dh), generator=g).to(torch.bfloat16).cuda()
        a["qkv"].copy_(x)
        b["qkv"].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        step(b, *wss[1])
        torch.cuda.synchronize()
        for key in a:
            assert torch.equal(a[key], b[key]), (i, key)
    assert a["length"].tolist() == [290, 37, 21, 290]


def test_another_stream_and_odd_strides(L):
    """Queries and outputs that are slices of wider rows, on a stream of their own."""
    c = Case(L, "bf16", 4, 2, 64, 16, [90, 200, 33], [20, 40, 33], seed=8)
    want = c.gpu()
    st = torch.cuda.Stream()
    wide = torch.full((c.q.shape[0], 7, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:5] = c.q.cuda()
    res = torch.full((c.q.shape[0], 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    n = L.llmc_attention_paged_workspace_bytes(c.q.cuda(), c.k.cuda(), c.table.cuda(), max_new=c.max_new, max_len=c.max_len)
    kp, vp, tab, ln, sr = c.k.cuda(), c.v.cuda(), c.table.cuda(), i32(c.lens), i32(c.starts)
    ws = torch.empty((n,), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    L.llmc_attention_paged(wide[:, 1:5], kp, vp, tab, ln, res[:, 4:8], ws, new_start=sr, max_new=c.max_new,
                           max_len=c.max_len, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(res[:, 4:8].cpu(), want)
    assert (res[:, :4] == 5).all() and (res[:, 8:] == 5).all()


def test_pages_outside_the_pool_are_no_pages(L):
    """A table entry beyond the pool: its tokens are not stored, not seen and not moved, and nothing else is touched."""
    g = torch.Generator().manual_seed(2)
    k, v, table = R.make_cache(g, torch.bfloat16, 2, 64, 16, [40, 40], fill=0.0)
    bad = table.clone()
    bad[0, 1] = k.shape[0]
    bad[1, 2] = -7
    q = torch.randn((2, 2, 64), generator=g).to(torch.bfloat16)
    out = torch.zeros_like(q).cuda()
    ws = torch.empty((1 << 20,), dtype=torch.uint8, device="cuda")
    kg, vg = k.cuda(), v.cuda()
    L.llmc_attention_paged(q.cuda(), kg, vg, bad.cuda(), i32([40, 40]), out, ws, max_len=48)
    torch.cuda.synchronize()
    for b, idx in ((0, [*range(16), *range(32, 40)]), (1, range(32))):
        kk, vv = R.tokens(k, table, b, 40)[:, list(idx)], R.tokens(v, table, b, 40)[:, list(idx)]
        p = torch.softmax(torch.einsum("hd,hkd->hk", q[b].double(), kk) / 8, 1)
        want = torch.einsum("hk,hkd->hd", p, vv)
        size = torch.einsum("hk,hkd->hd", p, vv.abs())
        assert ((out[b].cpu().double() - want).abs() <= 2.0 ** -8 * (size + want.abs()) + 1e-4).all()
    pos, w = torch.arange(64).repeat(2, 1).int().cuda(), torch.zeros((2, 64), device="cuda")
    L.llmc_kv_append(q.cuda(), q.cuda(), kg, vg, bad.cuda(), i32([20, 40]), pos=pos, weight=w)
    torch.cuda.synchronize()
    assert torch.equal(kg.cpu(), k) and torch.equal(vg.cpu(), v)


MIXED = [                                                # (dtype, heads, kv, dh, page, lens, news, options)
    ("bf16", 4, 2, 64, 16, [900, 33, 200], [200, 33, 7], dict(window=150, weights=True)),
    ("f32", 4, 4, 64, 32, [600, 5], [100, 1], dict(slopes=True, weights=True)),
    ("bf16", 8, 2, 128, 64, [3000, 1, 700], [1, 1, 1], dict(weights=True)),
]


def test_calls_on_two_streams_at_once(L):
    """Calls of different shapes on two streams, each with its own workspace, in flight together: the bits of calls alone."""
    cases = [Case(L, *m[:7], seed=20 + i, **m[7]) for i, m in enumerate(MIXED)]
    alone = [(c.gpu(), c.w_gpu.cpu()) for c in cases]
    args = []
    for c in cases:
        q, kp, tab = c.q.cuda(), c.k.cuda(), c.table.cuda()
        n = L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=c.max_new, max_len=c.max_len, weights=True)
        args.append((q, kp, c.v.cuda(), tab, i32(c.lens), n, i32(c.starts), None if c.slopes is None else c.slopes.cuda()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    runs = []
    torch.cuda.synchronize()
    for rep in range(6):
        for i, (c, a) in enumerate(zip(cases, args)):
            q, kp, vp, tab, length, n, start, slopes = a
            with torch.cuda.stream(streams[(rep + i) & 1]):
                out, w = torch.zeros_like(q), c.weight.cuda()
                ws = torch.empty((n,), dtype=torch.uint8, device="cuda")
                L.llmc_attention_paged(q, kp, vp, tab, length, out, ws, new_start=start, max_new=c.max_new, max_len=c.max_len,
                                       weight=w, slopes=slopes, **c.opt)
                runs.append((i, out, w, ws))
    torch.cuda.synchronize()
    for i, out, w, _ in runs:
        assert torch.equal(out.cpu(), alone[i][0]) and torch.equal(w.cpu(), alone[i][1]), i


def test_recorded_calls_share_a_workspace(L):
    """Two graphs recorded with one workspace, replayed in turn with an eager call in it between: no call needs what another left."""
    cases = [Case(L, *m[:7], seed=20 + i, **m[7]) for i, m in enumerate(MIXED)]
    alone = [(c.gpu(), c.w_gpu.cpu()) for c in cases]
    args, need = [], 0
    for c in cases:
        q, kp, tab = c.q.cuda(), c.k.cuda(), c.table.cuda()
        need = max(need, L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=c.max_new, max_len=c.max_len, weights=True))
        args.append([q, kp, c.v.cuda(), tab, i32(c.lens), torch.zeros_like(q)])
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    extra = [(i32(c.starts), c.weight.cuda(), None if c.slopes is None else c.slopes.cuda()) for c in cases]

    def call(i):
        c, (start, w, slopes) = cases[i], extra[i]
        L.llmc_attention_paged(*args[i], ws, new_start=start, max_new=c.max_new, max_len=c.max_len, weight=w, slopes=slopes, **c.opt)

    graphs = []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for rep in range(4):
        for i in range(3):
            extra[i][1].copy_(cases[i].weight)
            args[i][5].fill_(7.0)
            if i < 2:
                graphs[i].replay()
            else:
                call(i)
        torch.cuda.synchronize()
        for i in range(3):
            assert torch.equal(args[i][5].cpu(), alone[i][0]) and torch.equal(extra[i][1].cpu(), alone[i][1]), (rep, i)
        ws.fill_(rep)
