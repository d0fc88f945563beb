"""The decoder block over the paged cache and the stack of it, with windows, budgets, capped scores and biases, against a 64-bit
decoder that keeps every token's key and value in a list."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
from oracle import llmc_oracle as O
from test_gpu_paged import TOL, L, i32, small_decoder  # noqa: F401 (L is a fixture)


def strong(ws, by=4.0):
    """Weights whose attention is not nearly uniform and not a small part of the output: scores of a standard deviation near one."""
    out = []
    for w in ws:
        w = dict(w)
        for name in ("wqkv", "wo"):
            w[name] = (w[name].float() * by).to(w[name].dtype)
        out.append(w)
    return out


class Plain:
    """The cache of one layer and sequence, [position, weight, key, value] in the order of the slots, and the block on new tokens."""

    def __init__(self, cfg, w, window=0, softcap=0.0, slopes=None):
        self.cfg, self.w = cfg, {k: v.double().numpy() for k, v in w.items()}
        self.window, self.softcap, self.slopes = window, softcap, slopes
        self.cache = []

    def block(self, x, first):
        """x [n, d]; positions from first on."""
        cfg, w, H = self.cfg, self.w, self.cfg.n_heads
        n, d = x.shape
        dh = d // H
        y = O.layer_norm(x, w["ln1_g"], w["ln1_b"], cfg.ln_eps)
        q, k, v = np.moveaxis((y @ w["wqkv"].T + w["bqkv"]).reshape(n, 3, H, dh), 1, 0)
        self.cache += [[first + i, 0.0, k[i], v[i]] for i in range(n)]
        K, V = np.stack([c[2] for c in self.cache]), np.stack([c[3] for c in self.cache])
        pos = np.array([c[0] for c in self.cache])
        ctx = np.zeros((n, H, dh))
        for i in range(n):
            away = first + i - pos
            seen = np.arange(len(pos)) <= len(pos) - n + i
            if self.window:
                seen &= away < self.window
            s = np.einsum("hd,khd->hk", q[i], K) / math.sqrt(dh)
            if self.softcap:
                s = self.softcap * np.tanh(s / self.softcap)
            if self.slopes is not None:
                s = s - self.slopes[:, None] * away
            e = np.where(seen, np.exp(s - s[:, seen].max(1, keepdims=True)), 0.0)
            p = e / e.sum(1, keepdims=True)
            ctx[i] = np.einsum("hk,khd->hd", p, V)
            for c, a in zip(self.cache, p.sum(0)):
                c[1] += float(a)
        x1 = x + ctx.reshape(n, d) @ w["wo"].T + w["bo"]
        y = O.layer_norm(x1, w["ln2_g"], w["ln2_b"], cfg.ln_eps)
        return x1 + O.gelu(y @ w["w1"].T + w["b1"], cfg.gelu) @ w["w2"].T + w["b2"]

    def protected(self, sink, recent):
        last = max(c[0] for c in self.cache)
        return [c[0] < sink or c[0] > last - recent for c in self.cache]

    def evict(self, keep, sink, recent):
        """Returns how far apart the last one that goes and the first one that stays are, relative to the weight."""
        if len(self.cache) <= keep:
            return math.inf
        free = sorted(c[1] for c, safe in zip(self.cache, self.protected(sink, recent)) if not safe)
        gone = len(self.cache) - keep
        gap = (free[gone] - free[gone - 1]) / free[gone] if gone < len(free) else math.inf
        moves, left = R.evict([c[0] for c in self.cache], [c[1] for c in self.cache], len(self.cache), keep, sink, recent)
        for s, d in moves:
            self.cache[d] = self.cache[s]
        self.cache = self.cache[:left]
        return gap

    def take(self, positions):
        """The cache holds these positions from now on, in this order."""
        by = {c[0]: c for c in self.cache}
        self.cache = [by[p] for p in positions]


def close(got, want, dtype):
    got = got.double().cpu().numpy()
    return (np.abs(got - want).max(axis=1) / np.abs(want).max(axis=1)).max() < TOL[dtype]


def test_the_plain_block_is_the_oracles():
    _, cfg, ws = small_decoder("f32")
    x = np.random.default_rng(0).standard_normal((30, cfg.d))
    p = Plain(cfg, strong(ws)[0])
    got = np.concatenate([p.block(x[:11], 0), p.block(x[11:12], 11), p.block(x[12:], 12)])
    want = O.layer_forward(x, {k: v.double().numpy() for k, v in strong(ws)[0].items()}, 1, cfg.n_heads, cfg.ln_eps, cfg.gelu)
    assert np.abs(got - want).max() < 1e-10


PLAN = [[40, 3], [1, 1], [33, 25], [5, 0], [1, 1], [1, 30]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 20, 64])
def test_a_stack_in_a_window(L, dtype, window):
    """Chunks longer and shorter than the window, three layers."""
    from paper_2512_16843_amd.engine import PagedStack
    _, cfg, ws = small_decoder(dtype, n_layers=3)
    ws = strong(ws)
    st = PagedStack(cfg, ws, 2, 96, page_size=16, window=window)
    plain = [[Plain(cfg, w, window=window) for w in ws] for _ in range(2)]
    whole = [[Plain(cfg, w) for w in ws] for _ in range(2)]
    g = torch.Generator().manual_seed(window)
    at, apart = [0, 0], 0.0
    for new in PLAN:
        h = torch.randn((sum(new), cfg.d), generator=g).to(cfg.torch_dtype)
        got = st.extend(h.cuda(), new)
        r = 0
        for b, n in enumerate(new):
            if n == 0:
                continue
            x = y = h[r:r + n].double().numpy()
            for l in range(3):
                x, y = plain[b][l].block(x, at[b]), whole[b][l].block(y, at[b])
            assert close(got[r:r + n], x, dtype)
            apart = max(apart, np.abs(x - y).max() / np.abs(x).max())
            r += n
            at[b] += n
    assert apart > 5 * TOL[dtype]                                  # without the window the outputs are others


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 30])
def test_two_layers_keep_what_each_attended_to(L, window):
    """fp32: each layer keeps other tokens, over one table and one length, and the window goes by positions."""
    from paper_2512_16843_amd.engine import PagedStack
    _, cfg, ws = small_decoder("f32", n_layers=2)
    ws = strong(ws)
    budget, sink, recent = 24, 2, 6
    st = PagedStack(cfg, ws, 2, 96, page_size=16, budget=budget, sink=sink, recent=recent, window=window)
    plain = [[Plain(cfg, w, window=window) for w in ws] for _ in range(2)]
    g = torch.Generator().manual_seed(40 if window else 5)       # choices by a per cent and more
    at, others = [0, 0], 0
    for new in PLAN:
        h = torch.randn((sum(new), cfg.d), generator=g)
        got = st.extend(h.cuda(), new)
        r = 0
        for b, n in enumerate(new):
            x = h[r:r + n].double().numpy()
            for l in range(2):
                if n:
                    x = plain[b][l].block(x, at[b])
                assert plain[b][l].evict(budget, sink, recent) > 1e-3         # no choice that fp32 could make otherwise
                kept = [c[0] for c in plain[b][l].cache]
                assert st.lengths[b] == len(kept)
                assert st.pos[l][b, :len(kept)].tolist() == kept
                assert np.allclose(st.weight[l][b, :len(kept)].cpu().numpy(), [c[1] for c in plain[b][l].cache], rtol=1e-4, atol=1e-5)
            assert n == 0 or close(got[r:r + n], x, "f32")
            others += [c[0] for c in plain[b][0].cache] != [c[0] for c in plain[b][1].cache]
            r += n
            at[b] += n
    assert others


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 30])
def test_a_budget_in_bf16(L, window):
    """The plain form follows the choices made on the GPU, which its own weights have to allow.  Scores here are within 4, from
    queries and keys rounded three times (the LayerNorm, the product, the layer before: 2^-8 each), so a score is off by up to
    4 * 6 * 2^-8 = 0.094, a weight by a tenth of itself, and two weights that are compared by a quarter."""
    from paper_2512_16843_amd.engine import PagedStack
    _, cfg, ws = small_decoder("bf16", n_layers=2)
    ws = strong(ws, 3.0)
    budget, sink, recent = 24, 2, 6
    st = PagedStack(cfg, ws, 2, 96, page_size=16, budget=budget, sink=sink, recent=recent, window=window)
    plain = [[Plain(cfg, w, window=window) for w in ws] for _ in range(2)]
    g = torch.Generator().manual_seed(7 + window)
    at = [0, 0]
    for new in PLAN:
        h = torch.randn((sum(new), cfg.d), generator=g).to(torch.bfloat16)
        got = st.extend(h.cuda(), new)
        r = 0
        for b, n in enumerate(new):
            x = h[r:r + n].double().numpy()
            for l in range(2):
                p = plain[b][l]
                if n:
                    x = p.block(x, at[b])
                kept = st.pos[l][b, :st.lengths[b]].tolist()
                assert len(kept) == len(set(kept)) == min(len(p.cache), budget)
                safe = p.protected(sink, recent)
                gone = [c[1] for c, s in zip(p.cache, safe) if c[0] not in kept and not s]
                stay = [c[1] for c, s in zip(p.cache, safe) if c[0] in kept and not s]
                assert all(c[0] in kept for c, s in zip(p.cache, safe) if s)
                assert not gone or not stay or max(gone) <= 1.25 * min(stay)
                p.take(kept)
                assert np.allclose(st.weight[l][b, :len(kept)].cpu().numpy(), [c[1] for c in p.cache], rtol=0.1, atol=0)
            assert n == 0 or close(got[r:r + n], x, "bf16")
            r += n
            at[b] += n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("opts", [dict(softcap=2.0), dict(slopes=True), dict(window=25), dict(softcap=3.0, slopes=True, window=40)],
                         ids=lambda o: "-".join(o))
@pytest.mark.parametrize("news", [[1, 1], [3, 8], [50, 21]])
def test_the_block_with_scores_that_are_not_plain(L, dtype, opts, news):
    """Three calls of one block: what is there, a chunk and a token; the weights that the cached tokens have gathered too."""
    _, cfg, ws = small_decoder(dtype, n_layers=1)
    w = strong(ws)[0]
    slopes = torch.tensor([0.25, 0.0625][:cfg.n_heads]) if "slopes" in opts else None
    o = dict(opts, slopes=None if slopes is None else slopes.cuda())
    layer = L.layer_from_weights(cfg, w, "cuda")
    plain = [Plain(cfg, w, window=opts.get("window", 0), softcap=opts.get("softcap", 0.0),
                   slopes=None if slopes is None else slopes.double().numpy()) for _ in range(2)]
    bare = [Plain(cfg, w) for _ in range(2)]
    k = torch.full((16, cfg.n_heads, 16, 64), float("nan"), dtype=cfg.torch_dtype, device="cuda")
    v = k.clone()
    table = torch.randperm(16, generator=torch.Generator().manual_seed(1)).reshape(2, 8).int().cuda()
    weight = torch.zeros((2, 128), device="cuda")
    g = torch.Generator().manual_seed(11)
    at, apart = [0, 0], 0.0
    for new in ([30, 40], news, [1, 1]):
        h = torch.randn((sum(new), cfg.d), generator=g).to(cfg.torch_dtype)
        out = torch.empty_like(h, device="cuda")
        lens = [a + n for a, n in zip(at, new)]
        ws_ = torch.empty((L.llmc_layer_paged_workspace_bytes(layer, sum(new), 2, max(new), 128, True),), dtype=torch.uint8, device="cuda")
        L.llmc_layer_forward_paged(layer, h.cuda(), out, k, v, table, i32(lens), ws_, new_start=i32([0, new[0], sum(new)]),
                                   max_new=max(new), weight=weight, accumulate=True, **o)
        r = 0
        for b, n in enumerate(new):
            x = h[r:r + n].double().numpy()
            want = plain[b].block(x, at[b])
            assert close(out[r:r + n], want, dtype)
            apart = max(apart, np.abs(want - bare[b].block(x, at[b])).max() / np.abs(want).max())
            r += n
            at[b] += n
    assert apart > 2 * TOL[dtype]                                  # plain scores would not do
    for b in range(2):
        rtol = 1e-4 if dtype == "f32" else 0.1
        assert np.allclose(weight[b, :at[b]].cpu().numpy(), [c[1] for c in plain[b].cache], rtol=rtol, atol=1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["wqkv", "ln2_b"])
def test_a_layer_whose_weights_lie_elsewhere_is_refused(L, name):
    _, cfg, ws = small_decoder("f32", n_layers=1)
    layer = L.layer_from_weights(cfg, ws[0], "cuda")
    layer.w[name] = layer.w[name].cpu()
    k = torch.zeros((2, cfg.n_heads, 16, 64), device="cuda")
    h = torch.zeros((1, cfg.d), device="cuda")
    ws_ = torch.empty((L.llmc_layer_paged_workspace_bytes(layer, 1, 1, 1, 16),), dtype=torch.uint8, device="cuda")
    with pytest.raises(L.LlmcError, match=name) as e:
        L.llmc_layer_forward_paged(layer, h, torch.empty_like(h), k, k.clone(), i32([[0]]), i32([1]), ws_)
    assert e.value.status == L.ERR_INVALID_ARG


@pytest.mark.gpu
def test_a_stack_stays_on_the_device_it_was_made_on(L):
    from paper_2512_16843_amd.engine import PagedStack
    _, cfg, ws = small_decoder("f32", n_layers=1)
    st = PagedStack(cfg, ws, 1, 32)
    assert st.device == torch.device("cuda", torch.cuda.current_device()) == st.k[0].device
