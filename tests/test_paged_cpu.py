"""Host-only checks of the paged key/value cache: refusals come before any GPU call, sizes are told, and the plain forms that
the GPU tests compare with hold up by themselves."""
import ctypes as C
import os

import pytest
import torch

import paged_ref as R
from paper_2512_16843_amd import llmc


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(llmc.LIB_PATH):
        from paper_2512_16843_amd.build import build_library
        build_library()
    return llmc.lib()


P = 4096            # never dereferenced: validation fails first


def kv(**o):
    d = dict(n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, dtype=llmc.BF16, d_k=P, d_v=P)
    d.update(o)
    return llmc.KvDesc(*d.values())


def batch(**o):
    d = dict(n_seqs=3, max_pages=4, d_table=P, d_length=P, d_new_start=None, n_rows=3, max_new=1, max_len=64, d_pos=P, d_weight=P)
    d.update(o)
    return llmc.KvBatch(*d.values())


def attn(**o):
    d = dict(n_heads=4, scale=0.125, softcap=0.0, window=0, d_slopes=None, accumulate=0)
    d.update(o)
    return llmc.AttnDesc(*d.values())


def ref(x):
    return None if x is None else C.byref(x)


BAD_KV = [
    (None, llmc.ERR_INVALID_ARG), (kv(dtype=5), llmc.ERR_DTYPE), (kv(n_pages=0), llmc.ERR_INVALID_ARG),
    (kv(n_kv_heads=0), llmc.ERR_INVALID_ARG), (kv(page_size=8), llmc.ERR_SHAPE), (kv(page_size=48), llmc.ERR_SHAPE),
    (kv(page_size=2048), llmc.ERR_SHAPE), (kv(head_dim=96), llmc.ERR_SHAPE), (kv(d_k=None), llmc.ERR_INVALID_ARG),
    (kv(d_v=P + 4), llmc.ERR_SHAPE),
]
BAD_BATCH = [
    (None, llmc.ERR_INVALID_ARG), (batch(n_seqs=0), llmc.ERR_INVALID_ARG), (batch(n_seqs=70000), llmc.ERR_SHAPE),
    (batch(max_len=0), llmc.ERR_INVALID_ARG), (batch(max_len=65), llmc.ERR_SHAPE), (batch(max_pages=0), llmc.ERR_SHAPE),
    (batch(max_pages=1 << 28, max_len=1 << 29), llmc.ERR_SHAPE), (batch(d_table=None), llmc.ERR_INVALID_ARG),
    (batch(d_length=None), llmc.ERR_INVALID_ARG), (batch(d_pos=P + 4), llmc.ERR_SHAPE), (batch(d_weight=P + 8), llmc.ERR_SHAPE),
]
BAD_ROWS = [
    (batch(n_rows=-1), llmc.ERR_INVALID_ARG), (batch(max_new=0), llmc.ERR_INVALID_ARG), (batch(max_new=2), llmc.ERR_SHAPE),
    (batch(n_rows=4), llmc.ERR_SHAPE), (batch(d_new_start=P, max_new=65), llmc.ERR_SHAPE),
]
BAD_ATTN = [
    (None, llmc.ERR_INVALID_ARG), (attn(n_heads=0), llmc.ERR_INVALID_ARG), (attn(n_heads=3), llmc.ERR_SHAPE),
    (attn(scale=0.0), llmc.ERR_INVALID_ARG), (attn(scale=float("nan")), llmc.ERR_INVALID_ARG),
    (attn(scale=float("inf")), llmc.ERR_INVALID_ARG), (attn(softcap=-1.0), llmc.ERR_INVALID_ARG),
    (attn(softcap=float("nan")), llmc.ERR_INVALID_ARG), (attn(window=-1), llmc.ERR_INVALID_ARG),
    (attn(accumulate=2), llmc.ERR_INVALID_ARG),
]


def test_refusals_of_scales_and_caps_that_overflow(lib):
    def call(a):
        return lib.llmc_attention_paged(ref(kv()), ref(batch()), ref(a), P, 256, P + 16, 256, P, 1 << 30, None)
    for a in (attn(scale=3e38), attn(softcap=2e38), attn(scale=1e3, softcap=1e-38)):
        assert call(a) == llmc.ERR_INVALID_ARG, lib.llmc_last_error()


def test_refusals_of_append(lib):
    def call(k=kv(), b=batch(), kn=P, ldk=128, vn=P, ldv=128):
        return lib.llmc_kv_append(ref(k), ref(b), kn, ldk, vn, ldv, None, None)
    for k, st in BAD_KV:
        assert call(k=k) == st, lib.llmc_last_error()
    for b, st in BAD_BATCH + BAD_ROWS:
        assert call(b=b) == st, lib.llmc_last_error()
    assert call(kn=None) == llmc.ERR_INVALID_ARG and call(vn=None) == llmc.ERR_INVALID_ARG
    assert call(ldk=120) == llmc.ERR_SHAPE and call(ldv=132) == llmc.ERR_SHAPE
    assert call(kn=P + 2) == llmc.ERR_SHAPE
    # nothing to store: no GPU call is made
    assert call(b=batch(n_rows=0, d_new_start=P), kn=None, vn=None) == llmc.LLMC_OK


def test_refusals_of_attention(lib):
    big = 1 << 30
    def call(k=kv(), b=batch(), a=attn(), q=P, ldq=256, out=2 * P, ldo=256, ws=P, n=big):
        return lib.llmc_attention_paged(ref(k), ref(b), ref(a), q, ldq, out, ldo, ws, n, None)
    for k, st in BAD_KV:
        assert call(k=k) == st, lib.llmc_last_error()
    for b, st in BAD_BATCH + BAD_ROWS:
        assert call(b=b) == st, lib.llmc_last_error()
    for a, st in BAD_ATTN:
        assert call(a=a) == st, lib.llmc_last_error()
    assert call(a=attn(accumulate=1), b=batch(d_weight=None)) == llmc.ERR_INVALID_ARG
    assert call(q=None) == llmc.ERR_INVALID_ARG and call(out=None) == llmc.ERR_INVALID_ARG and call(out=P) == llmc.ERR_INVALID_ARG
    assert call(ldq=248) == llmc.ERR_SHAPE and call(ldo=260) == llmc.ERR_SHAPE
    assert call(q=P + 8) == llmc.ERR_SHAPE and call(ws=P + 8) == llmc.ERR_SHAPE
    assert call(ws=None) == llmc.ERR_WORKSPACE and call(n=8) == llmc.ERR_WORKSPACE
    assert call(b=batch(n_rows=0, d_new_start=P), q=None, out=None) == llmc.LLMC_OK
    # too large for one launch
    huge = batch(n_seqs=65535, max_pages=1 << 20, max_len=1 << 24, d_new_start=P, n_rows=1 << 30, max_new=1 << 15)
    assert call(b=huge, a=attn(n_heads=64, accumulate=1)) == llmc.ERR_SHAPE


def test_refusals_of_eviction(lib):
    def call(k=kv(), b=batch(), keep=P, sink=0, recent=0, out=P, ws=P, n=1 << 30):
        return lib.llmc_kv_evict(ref(k), ref(b), keep, sink, recent, out, ws, n, None)
    for k, st in BAD_KV:
        assert call(k=k) == st, lib.llmc_last_error()
    for b, st in BAD_BATCH + [(batch(d_pos=None), llmc.ERR_INVALID_ARG), (batch(d_weight=None), llmc.ERR_INVALID_ARG)]:
        assert call(b=b) == st, lib.llmc_last_error()
    assert call(keep=None) == llmc.ERR_INVALID_ARG and call(out=None) == llmc.ERR_INVALID_ARG
    assert call(sink=-1) == llmc.ERR_INVALID_ARG and call(recent=-1) == llmc.ERR_INVALID_ARG
    assert call(ws=None) == llmc.ERR_WORKSPACE and call(n=16) == llmc.ERR_WORKSPACE and call(ws=P + 1) == llmc.ERR_SHAPE


def layer(**o):
    d = dict(arch=1, d=128, n_heads=2, d_ff=256, gelu=1, ln_eps=1e-5, dtype=llmc.BF16)
    d.update(o)
    return llmc.LayerDesc(*d.values(), *([P] * 12))


def test_refusals_of_the_block(lib):
    def call(l=layer(), k=kv(), b=batch(), a=attn(n_heads=2), x=P, y=2 * P, ws=P, n=1 << 30):
        return lib.llmc_layer_forward_paged(ref(l), ref(k), ref(b), ref(a), None, x, y, ws, n, None)
    assert call(l=None) == llmc.ERR_INVALID_ARG and call(l=layer(arch=0)) == llmc.ERR_INVALID_ARG
    for k, st in BAD_KV:
        assert call(k=k) == st, lib.llmc_last_error()
    for b, st in BAD_BATCH + BAD_ROWS:
        assert call(b=b) == st, lib.llmc_last_error()
    assert call(k=kv(dtype=llmc.F32)) == llmc.ERR_DTYPE
    assert call(k=kv(n_kv_heads=1)) == llmc.ERR_SHAPE and call(a=attn(n_heads=4)) == llmc.ERR_SHAPE
    assert call(k=kv(head_dim=128)) == llmc.ERR_SHAPE
    assert call(x=None) == llmc.ERR_INVALID_ARG and call(y=P) == llmc.ERR_INVALID_ARG
    assert call(ws=P + 16) == llmc.ERR_SHAPE and call(n=100) == llmc.ERR_WORKSPACE
    assert call(b=batch(n_rows=0, d_new_start=P)) == llmc.LLMC_OK


def test_the_binding_refuses_what_it_cannot_express(lib):
    k = torch.zeros((8, 2, 16, 64), dtype=torch.bfloat16)
    table = torch.zeros((3, 4), dtype=torch.int32)
    length = torch.ones((3,), dtype=torch.int32)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    ws = torch.zeros((1 << 20,), dtype=torch.uint8)
    n = llmc.llmc_attention_paged_workspace_bytes(q, k, table, max_len=64)
    assert 0 < n <= ws.numel()
    def refused(status, **o):
        a = dict(q=q, k_pages=k, v_pages=k, table=table, length=length, out=q.clone(), workspace=ws)
        a.update(o)
        with pytest.raises(llmc.LlmcError) as e:
            llmc.llmc_attention_paged(**a)
        assert e.value.status == status, e.value
    refused(llmc.ERR_DTYPE, q=q.float())
    refused(llmc.ERR_DTYPE, table=table.long())
    refused(llmc.ERR_DTYPE, v_pages=k.float())
    refused(llmc.ERR_DTYPE, k_pages=k.half(), v_pages=k.half())
    refused(llmc.ERR_SHAPE, length=length[:2])
    refused(llmc.ERR_SHAPE, out=q[:2])
    refused(llmc.ERR_SHAPE, q=q[:, :, :32], out=q[:, :, :32])
    refused(llmc.ERR_SHAPE, q=q.transpose(0, 1).contiguous().transpose(0, 1))
    refused(llmc.ERR_SHAPE, k_pages=k.transpose(1, 2), v_pages=k.transpose(1, 2))
    refused(llmc.ERR_SHAPE, weight=torch.zeros((3, 60)))
    refused(llmc.ERR_DTYPE, pos=torch.zeros((3, 64)))
    refused(llmc.ERR_DTYPE, slopes=torch.zeros((4,), dtype=torch.float64))
    refused(llmc.ERR_INVALID_ARG)                       # all is well, but for the tensors being on the host
    with pytest.raises(llmc.LlmcError):
        llmc.llmc_attention_paged_workspace_bytes(q, k, table, max_len=0)


def test_workspace_sizes(lib):
    assert lib.llmc_kv_evict_workspace_bytes(0, 5) == 0 and lib.llmc_kv_evict_workspace_bytes(2, 0) == 0
    assert lib.llmc_kv_evict_workspace_bytes(3, 100) >= 3 * 50 * 8
    a = lib.llmc_attention_paged_workspace_bytes(ref(kv()), ref(batch()), ref(attn()))
    b = lib.llmc_attention_paged_workspace_bytes(ref(kv()), ref(batch()), ref(attn(accumulate=1)))
    assert 0 < a < b
    assert lib.llmc_attention_paged_workspace_bytes(ref(kv(head_dim=32)), ref(batch()), ref(attn())) == 0
    assert lib.llmc_layer_paged_workspace_bytes(ref(layer()), ref(batch()), ref(attn(n_heads=2))) > a
    assert lib.llmc_layer_paged_workspace_bytes(ref(layer(d=100)), ref(batch()), ref(attn(n_heads=2))) == 0


def test_plain_eviction_by_hand():
    # slots 0..5, budget 3: weights 5 1 4 2 9 3 -> 1, 2, 3 go; kept 5 (slot 0), 4 (slot 2), 9 (slot 4); hole 1 takes slot 4
    assert R.evict([0, 1, 2, 3, 4, 5], [5, 1, 4, 2, 9, 3], 6, 3, 0, 0) == ([(4, 1)], 3)
    # the last two positions are protected (2 and 3 of weight stay), the first too
    assert R.evict([0, 1, 2, 3, 4, 5], [0, 1, 4, 2, 9, 3], 6, 4, 1, 2) == ([(4, 1), (5, 3)], 4)
    # ties go to the lower position, wherever it stands
    assert R.evict([3, 0, 2, 1], [1, 1, 1, 1], 4, 2, 0, 0) == ([(2, 1)], 2)
    assert R.evict([0, 1], [1, 1], 2, 5, 0, 0) == ([], 2)


def test_plain_attention_against_torch():
    g = torch.Generator().manual_seed(0)
    k, v, table = R.make_cache(g, torch.float32, 2, 64, 16, [40, 19])
    q = torch.randn((5, 4, 64), generator=g)
    out, tol, w, _ = R.attention(q, k, v, table, [40, 19], [0, 3, 5])
    for b, n, lo, hi in ((0, 40, 0, 3), (1, 19, 3, 5)):
        kk, vv = R.tokens(k, table, b, n).repeat_interleave(2, 0), R.tokens(v, table, b, n).repeat_interleave(2, 0)
        mask = torch.arange(n)[None] <= torch.arange(n - (hi - lo), n)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(q[lo:hi].double().transpose(0, 1), kk, vv, attn_mask=mask)
        assert torch.allclose(out[lo:hi], want.transpose(0, 1), rtol=1e-12, atol=1e-12)
        assert abs(float(w[b].sum()) - 4 * (hi - lo)) < 1e-9
    assert (tol > 0).all()
