"""The paged key/value cache on the GPU where it can go wrong besides its sizes: how exactly few rows are weighted."""
import pytest
import torch

import paged_ref as R
from test_gpu_paged import DT, L, Case, i32, starts_of  # noqa: F401 (L is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,dh,lens,news", [
    (12, 12, 64, [777], [1]),
    (8, 2, 128, [300, 1, 64, 17], [1, 1, 1, 1]),
    (16, 1, 64, [500, 33], [1, 1]),
    (4, 2, 64, [90, 8, 1500], [8, 5, 1]),
    (8, 8, 64, [6000, 4095], [1, 1]),              # in pieces
])
@pytest.mark.parametrize("opts", [dict(), dict(softcap=20.0, slopes=True), dict(weights=True)],
                         ids=lambda o: "-".join(o) or "plain")
def test_few_rows_are_weighted_to_sixteen_bits(L, heads, kv, dh, lens, news, opts):
    """Up to 16 rows a key/value head in bf16: a weight p enters the value product as two bf16 numbers, p rounded (off by at most
    half a step, 2^-8 p) and what that left, rounded (2^-8 of it): 2^-16 p in all, where one number would be off by 2^-8 p.  The
    bound of the plain form has that one rounding in it; here it is exchanged, and the fp32 sum has twice as many terms."""
    c = Case(L, "bf16", heads, kv, dh, 16, lens, news, seed=31 + heads, **opts)
    got = c.gpu(decode=news == [1] * len(news))
    form = dict(pos=c.pos, slopes=c.slopes, **c.opt)
    want, tol, _, _ = R.attention(c.q, c.k, c.v, c.table, c.lens, c.starts, **form)
    size, _, _, _ = R.attention(c.q, c.k, c.v.abs(), c.table, c.lens, c.starts, **form)
    tol = tol + size * (2.0 ** -16 - 2.0 ** -8 + (max(lens) + 64) * 2.0 ** -24)
    over = ((got.double() - want).abs() - tol).max()
    assert over <= 0, over


def evicted(L, lens, keep, sink, recent, table, k, v, pos, weight):
    """(k, v, pos, weight, new lengths) after the call, on the CPU."""
    kg, vg, tg, pg, wg = (t.cuda() for t in (k, v, table, pos, weight))
    out = torch.full((len(lens),), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((L.llmc_kv_evict_workspace_bytes(tg, max(lens)),), 255, dtype=torch.uint8, device="cuda")
    L.llmc_kv_evict(kg, vg, tg, i32(lens), pg, wg, i32(keep), out, ws, max_len=max(lens), sink=sink, recent=recent)
    torch.cuda.synchronize()
    return kg.cpu(), vg.cpu(), pg.cpu(), wg.cpu(), out.tolist()


@pytest.mark.parametrize("lens,keep,sink,recent", [
    ([100, 60], [70, 33], 4, 8),
    ([64, 64], [16, 0], 20, 16),                   # more protected tokens than are kept
    ([3000, 900], [1500, 899], 0, 64),
    ([5000, 8000], [4000, 100], 16, 0),
    ([33000, 40], [20000, 20], 0, 0),
])
@pytest.mark.parametrize("weights", ["spread", "ends"])
def test_eviction_leaves_slots_without_a_page_alone(L, lens, keep, sink, recent, weights):
    """Entries of the table outside the pool, under holes, movers and protected tokens: such slots neither give nor take a token,
    and what the others hold is chosen among the tokens that have pages."""
    page, B = 16, len(lens)
    g = torch.Generator().manual_seed(sum(lens))
    k, v, table = R.make_cache(g, torch.bfloat16, 2, 64, page, lens, fill=0.25)
    slots = table.shape[1] * page
    pos = torch.stack([torch.randperm(2 * slots, generator=g)[:slots] for _ in range(B)]).to(torch.int32)
    w = torch.exp(2 * torch.randn((B, slots), generator=g))
    if weights == "ends":                          # the ends of the weights' order, and of the positions'
        for x, every in ((float("nan"), 3), (float("inf"), 5), (-float("inf"), 4), (0.0, 7)):
            w[:, ::every] = x
        pos[:, 1] = 2 ** 31 - 1
        w[:, 1] = float("nan")
    for b, n in enumerate(lens):
        cols = (n + page - 1) // page
        for i, c in enumerate({0, cols // 2, cols - 1, max(0, keep[b] // page - 1), min(cols - 1, keep[b] // page)}):
            table[b, c] = (k.shape[0], -7, 2 ** 30)[i % 3]
    got = evicted(L, lens, keep, sink, recent, table, k, v, pos, w)
    has = lambda b, j: 0 <= int(table[b, j // page]) < k.shape[0]
    for b, n in enumerate(lens):
        m = max(0, min(keep[b], n))
        on = [j for j in range(n) if has(b, j)]
        below = sum(j < m for j in on)
        last = max(pos[b, :n].tolist())
        p, ww = pos[b].tolist(), w[b].tolist()

        def order(j):
            x = ww[j]
            return (p[j] < sink or p[j] > last - recent, (1, 0.0) if x != x else (0, x), p[j], j)

        gone = set(sorted(on, key=order)[:len(on) - below])
        holes = [j for j in on if j < m and j in gone]
        movers = [j for j in on if j >= m and j not in gone]
        assert len(holes) == len(movers)
        for s, d in zip(movers, holes):
            ps, pd = int(table[b, s // page]), int(table[b, d // page])
            k[pd, :, d % page], v[pd, :, d % page] = k[ps, :, s % page], v[ps, :, s % page]
            pos[b, d], w[b, d] = pos[b, s], w[b, s]
        assert got[4][b] == m
    assert torch.equal(got[2], pos) and torch.equal(got[3].view(torch.int32), w.view(torch.int32))
    assert torch.equal(got[0], k) and torch.equal(got[1], v)


def spoil(c, pages, b, slot, head, dims, value):
    page = c.k.shape[2]
    pages[int(c.table[b, slot // page]), head, slot % page, dims] = value


def who_sees(c, b):
    """[new tokens, slots] of sequence b: which new token sees which slot."""
    n, q = c.lens[b], c.starts[b + 1] - c.starts[b]
    slot = torch.arange(n - q, n)
    p = c.pos[b, :n].long() if c.pos is not None else torch.arange(n)
    away = p[slot][:, None] - p[None, :]
    seen = torch.arange(n)[None, :] <= slot[:, None]
    return seen & (away < c.opt["window"]) if c.opt["window"] else seen


HIDDEN = [
    # heads, kv, head_dim, lens, news
    (4, 2, 64, [90, 33, 200], [1, 1, 1]),          # single tokens: hidden by a window alone
    (4, 2, 64, [90, 12, 8], [4, 8, 2]),            # up to 16 rows a head
    (3, 3, 64, [200, 300], [200, 70]),
    (4, 1, 128, [150, 700], [150, 100]),
    (6, 2, 128, [5000, 100], [30, 40]),            # in pieces
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh,lens,news", HIDDEN)
@pytest.mark.parametrize("opts", [dict(), dict(window=20), dict(window=150, moved=True), dict(softcap=20.0, window=40),
                                  dict(slopes=True, weights=True), dict(weights=True, window=64)],
                         ids=lambda o: "-".join(o) or "plain")
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(L, dtype, heads, kv, dh, lens, news, opts):
    """Infinities and NaN among the values of new tokens, and of tokens at the edge of the window: a row that sees none of them is
    what it is without them; where a row sees them, those dims alone are +infinity, -infinity or NaN.  A weight below 2^-149 is
    zero in 32 bits, and zero times an infinity NaN: with a slope of 2^-2 the first of 700 tokens has exp(-0.25 * 699) = 2^-252.
    Below 2^-100 (what follows is 2^-126 and the normaliser, at most 700) either will do."""
    c = Case(L, dtype, heads, kv, dh, 16, lens, news, seed=41, spread=0.5, **opts)
    form = dict(pos=c.pos, slopes=c.slopes, **c.opt)
    want, tol, ws, wt = R.attention(c.q, c.k, c.v, c.table, c.lens, c.starts, **form)
    up = torch.zeros(want.shape, dtype=torch.bool)
    down = torch.zeros_like(up)
    clean, mark = c.v.clone(), torch.nan_to_num(c.v) * 0
    for b, (n, q) in enumerate(zip(lens, news)):
        first = max(0, n - q)
        spots = {0, n - 1, n - q // 2 - 1, first, max(0, first - 19), max(0, first - 20), max(0, first - 63), max(0, first - 64)}
        for i, slot in enumerate(sorted(spots)):
            h, dim, value = i % kv, (7 * i + 3) % dh, (float("inf"), -float("inf"), float("nan"))[i % 3]
            spoil(c, c.v, b, slot, h, dim, value)
            spoil(c, clean, b, slot, h, dim, 0.0)
            spoil(c, mark, b, slot, h, dim, 1.0)
            rows = torch.nonzero(who_sees(c, b)[:, slot])[:, 0] + c.starts[b]
            for head in range(h * heads // kv, (h + 1) * heads // kv):
                up[rows, head, dim] |= not value < 0
                down[rows, head, dim] |= not value > 0
    want, tol, ws, wt = R.attention(c.q, c.k, clean, c.table, c.lens, c.starts, **form)
    got = c.gpu(decode=news == [1] * len(news)).double()
    inf = float("inf")
    faint = R.attention(c.q, c.k, mark, c.table, c.lens, c.starts, **form)[0] < 2.0 ** -100
    assert not torch.isfinite(got[(up | down) & faint]).any()
    got = torch.where((up ^ down) & faint, torch.where(up, inf, -inf).double(), got)
    assert (got[up & ~down] == inf).all() and (got[down & ~up] == -inf).all() and torch.isnan(got[up & down]).all()
    rest = ~(up | down)
    assert torch.isfinite(got[rest]).all()
    over = ((got - want).abs() - tol)[rest].max()
    assert over <= 0, over
    if c.weight is not None:
        for b, n in enumerate(lens):
            add = c.w_gpu.cpu()[b].double() - c.weight[b].double()
            assert ((add[:n] - ws[b]).abs() <= wt[b] + 2.0 ** -23 * (c.weight[b, :n].double() + ws[b])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dh,lens,news", HIDDEN[:4] + [(4, 1, 64, [900, 40], [400, 40])])
@pytest.mark.parametrize("opts", [dict(), dict(window=20), dict(window=150, moved=True), dict(softcap=20.0, window=40),
                                  dict(slopes=True)], ids=lambda o: "-".join(o) or "plain")
def test_rows_of_nan_give_weight_to_what_they_see_alone(L, dtype, heads, kv, dh, lens, news, opts):
    """A query that is NaN, a key that is: the rows they concern are NaN, and so is the weight of the slots that these rows see.
    Every other row, and the weight of every other slot, is what it is without them."""
    c = Case(L, dtype, heads, kv, dh, 16, lens, news, seed=43, weights=True, **opts)
    q, k = c.q.clone(), c.k.clone()
    nan = float("nan")
    odd = torch.zeros((c.starts[-1], heads), dtype=torch.bool)
    for b, (n, m) in enumerate(zip(lens, news)):
        row = c.starts[b] + m // 3
        if b == 0:
            c.q[row, heads - 1, 3], q[row, heads - 1] = nan, 0.0
            odd[row, heads - 1] = True
        else:
            slot = max(0, n - m) + m // 3
            spoil(c, c.k, b, slot, 0, 5, nan)
            spoil(c, k, b, slot, 0, slice(None), 0.0)
            rows = torch.nonzero(who_sees(c, b)[:, slot])[:, 0] + c.starts[b]
            odd[rows, :heads // kv] = True
    got = c.gpu(decode=news == [1] * len(news)).double()
    want, tol, ws, wt = R.attention(q, k, c.v, c.table, c.lens, c.starts, pos=c.pos, slopes=c.slopes, **c.opt)
    assert torch.isnan(got[odd]).all()
    over = ((got - want).abs() - tol)[~odd].max() if (~odd).any() else 0.0
    assert over <= 0, over
    for b, n in enumerate(lens):
        add = c.w_gpu.cpu()[b].double() - c.weight[b].double()
        touched = who_sees(c, b)[odd[c.starts[b]:c.starts[b + 1]].any(1)].any(0)
        assert torch.isnan(add[:n][touched]).all()
        off = (add[:n] - ws[b]).abs() - wt[b] - 2.0 ** -23 * (c.weight[b, :n].double() + ws[b])
        assert (off[~touched] <= 0).all(), off[~touched].max()
        assert (add[n:] == 0).all()


# ---- launches of more workgroups than one dimension takes ------------------------------------------------------------

def test_append_of_rows_beyond_one_dimension(L):
    """2^26 rows and a few, a wavefront each: 2^32 threads.  All but the last eight belong to no sequence."""
    n = 2 ** 26 + 5
    g = torch.Generator().manual_seed(50)
    k, v, table = R.make_cache(g, torch.bfloat16, 1, 64, 16, [20], fill=0.5)
    new = torch.zeros((n, 1, 64), dtype=torch.bfloat16, device="cuda")
    last = torch.randn((8, 1, 64), generator=g).to(torch.bfloat16)
    new[n - 8:] = last.cuda()
    kg, vg = k.cuda(), v.cuda()
    L.llmc_kv_append(new, new, kg, vg, table.cuda(), i32([20]), new_start=i32([n - 8, n]), max_new=8)
    torch.cuda.synchronize()
    for got, was in ((kg, k), (vg, v)):
        assert torch.equal(R.tokens(got.cpu(), table, 0, 20)[:, 12:], last.transpose(0, 1).double())
        assert torch.equal(R.tokens(got.cpu(), table, 0, 12), R.tokens(was, table, 0, 12))


def test_pieces_of_rows_beyond_one_dimension(L):
    """The last 40 of 2^26 and a few rows attend over a cut axis: the outputs are those of the 40 rows alone."""
    n = 2 ** 26 + 5
    c = Case(L, "bf16", 1, 1, 64, 16, [500], [40], seed=51)
    alone = c.gpu()
    c.check(alone)
    q = torch.zeros((n, 1, 64), dtype=torch.bfloat16, device="cuda")
    q[n - 40:] = c.q.cuda()
    out = torch.full_like(q, 7.0)
    kp, vp, tab = c.k.cuda(), c.v.cuda(), c.table.cuda()
    need = L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=40, max_len=512)
    assert need >= n * 2 * 64 * 4                                  # two pieces, or more
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    L.llmc_attention_paged(q, kp, vp, tab, i32([500]), out, ws, new_start=i32([n - 40, n]), max_new=40, max_len=512)
    torch.cuda.synchronize()
    got = out[n - 40:].cpu()
    c.check(got)
    assert (out[:n - 40] == 7.0).all()


def test_weights_of_slots_beyond_one_dimension(L):
    """65535 sequences of up to 16400 tokens, a wavefront each 16 slots: 2^32 threads.  Three of them have new tokens."""
    at, B, max_len = [0, 40000, 65534], 65535, 16400
    c = Case(L, "f32", 1, 1, 128, 16, [30, 16400, 200], [17, 17, 5], seed=52, weights=True)
    mp = c.table.shape[1]
    table = torch.full((B, mp), -1, dtype=torch.int32, device="cuda")
    length, start = torch.zeros((B,), dtype=torch.int32), torch.zeros((B + 1,), dtype=torch.int32)
    weight = torch.full((B, mp * 16), 3.0, device="cuda")
    for i, b in enumerate(at):
        table[b], length[b], weight[b] = c.table[i].cuda(), c.lens[i], c.weight[i].cuda()
        start[b + 1:] += c.news[i]
    q, kp = c.q.cuda(), c.k.cuda()
    out = torch.zeros_like(q)
    ws = torch.empty((L.llmc_attention_paged_workspace_bytes(q, kp, table, max_new=17, max_len=max_len, weights=True),),
                     dtype=torch.uint8, device="cuda")
    L.llmc_attention_paged(q, kp, c.v.cuda(), table, length.cuda(), out, ws, new_start=start.cuda(), max_new=17, max_len=max_len,
                           weight=weight)
    torch.cuda.synchronize()
    c.w_gpu = weight[at]
    c.check(out.cpu())
    weight[at] = 3.0
    assert (weight == 3.0).all()


@pytest.mark.parametrize("first,second,ld", [(0, 4, 9), (5, 0, 9), (1, 5, 16), (0, 4, 8), (4, 0, 8)])
def test_queries_and_outputs_between_each_other_in_one_buffer(L, first, second, ld):
    """Rows of outputs that lie between the rows of queries overlap nothing."""
    c = Case(L, "bf16", 4, 2, 64, 16, [90, 200, 33], [20, 40, 33], seed=8)
    want = c.gpu()
    wide = torch.full((c.q.shape[0] + 1, ld, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    n = c.q.shape[0]
    q, out = wide[:n, first:first + 4], wide[1:, second:second + 4] if second < first else wide[:n, second:second + 4]
    q.copy_(c.q.cuda())
    kp, vp, tab = c.k.cuda(), c.v.cuda(), c.table.cuda()
    ws = torch.empty((L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_new=c.max_new, max_len=c.max_len),), dtype=torch.uint8,
                     device="cuda")
    L.llmc_attention_paged(q, kp, vp, tab, i32(c.lens), out, ws, new_start=i32(c.starts), max_new=c.max_new, max_len=c.max_len)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want) and torch.equal(q.cpu(), c.q)
    with pytest.raises(L.LlmcError, match="overlap"):
        L.llmc_attention_paged(q, kp, vp, tab, i32(c.lens), wide[:n, first + 1:first + 5] if first + 5 <= ld else wide[:n, first - 1:first + 3],
                               ws, new_start=i32(c.starts), max_new=c.max_new, max_len=c.max_len)


def test_queries_and_outputs_of_other_strides_in_one_buffer(L):
    """Two rows of queries 1024 elements apart, two of outputs 512 apart, the first behind the first: next to each other, not over."""
    c = Case(L, "bf16", 4, 2, 64, 16, [90, 20], [1, 1], seed=9)
    want = c.gpu(decode=True)
    flat = torch.full((2400,), 3.0, dtype=torch.bfloat16, device="cuda")
    q, out = flat.as_strided((2, 4, 64), (1024, 64, 1), 0), flat.as_strided((2, 4, 64), (512, 64, 1), 256)
    q.copy_(c.q.cuda())
    kp, vp, tab = c.k.cuda(), c.v.cuda(), c.table.cuda()
    ws = torch.empty((L.llmc_attention_paged_workspace_bytes(q, kp, tab, max_len=c.max_len),), dtype=torch.uint8, device="cuda")
    L.llmc_attention_paged(q, kp, vp, tab, i32(c.lens), out, ws, max_len=c.max_len)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want) and torch.equal(q.cpu(), c.q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 100, 7])
def test_windows_of_all_there_is_over_chunks_longer_than_their_sequence(L, dtype, window):
    """The slots of the rows in front are negative, and so far below the window's end that the difference leaves 32 bits."""
    c = Case(L, dtype, 2, 2, 64, 16, [20, 0, 150], [170, 40, 150], seed=60, weights=True, window=window, max_len=176)
    got = c.gpu()
    want, tol, ws, wt = R.attention(c.q, c.k, c.v, c.table, c.lens, c.starts, window=window)
    assert ((got.double() - want).abs() <= tol).all()
    assert (got[:150] == 0).all() and (got[170:210] == 0).all()
    for b, n in enumerate(c.lens):
        add = c.w_gpu.cpu()[b].double() - c.weight[b].double()
        assert ((add[:n] - ws[b]).abs() <= wt[b] + 2.0 ** -23 * (c.weight[b, :n].double() + ws[b])).all()
