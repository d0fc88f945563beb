"""Refusals of the paged key/value cache that look at where arrays lie.  Only calls that have to be refused are made: an accepted one
would go on to the GPU with addresses of nothing."""
import random

import pytest

from paper_2512_16843_amd import llmc
from test_paged_cpu import attn, batch, kv, layer, lib, ref  # noqa: F401 (lib is a fixture)

PAGES = 1 << 30                     # the pools lie apart from the rows
POOL = 8 * 2 * 16 * 64 * 2          # bytes of one


def chunks(at, n, row, ld):
    return {at + i * ld + j for i in range(n) for j in range(0, row, 16)}


def refused(lib, st):
    assert st == llmc.ERR_INVALID_ARG and b"overlap" in lib.llmc_last_error(), (st, lib.llmc_last_error())


def test_outputs_that_overlap_their_queries(lib):
    rng = random.Random(0)
    heads, row = 4, 4 * 64 * 2
    seen = 0
    while seen < 300:
        n = rng.choice([1, 2, 3, 7, 40])
        ldq = row + 16 * rng.randrange(0, 80)
        ldo = ldq if rng.random() < 0.5 else row + 16 * rng.randrange(0, 80)
        q = 1 << 20
        out = q + 16 * rng.randrange(-2 * n * ldq // 16, 2 * n * ldq // 16)
        if not chunks(q, n, row, ldq) & chunks(out, n, row, ldo):
            continue
        seen += 1
        b = batch(n_rows=n, max_new=min(n, 64), d_new_start=4096)
        refused(lib, lib.llmc_attention_paged(ref(kv(d_k=PAGES, d_v=PAGES + POOL)), ref(b), ref(attn(n_heads=heads)), q, ldq // 2, out,
                                              ldo // 2, 4096, 1 << 30, None))


@pytest.mark.parametrize("pool", ["d_k", "d_v"])
def test_outputs_that_overlap_the_pages(lib, pool):
    row, ld = 4 * 64 * 2, 3 * POOL // 2                           # the pool may lie between two rows, but for its ends
    for at in (PAGES, PAGES + POOL - 16, PAGES - row + 16, PAGES - ld, PAGES - ld + POOL - 16, PAGES - 2 * ld - row + 16):
        k = kv(**{"d_k": 1 << 40, "d_v": 1 << 41, pool: PAGES})
        refused(lib, lib.llmc_attention_paged(ref(k), ref(batch(d_new_start=4096)), ref(attn()), 1 << 35, 256, at, ld // 2, 4096,
                                              1 << 30, None))


def test_outputs_of_the_block_that_overlap(lib):
    bytes_ = 3 * 128 * 2                                          # three rows
    def call(x, y, **o):
        return lib.llmc_layer_forward_paged(ref(layer()), ref(kv(**dict(dict(d_k=PAGES, d_v=PAGES + POOL), **o))), ref(batch()),
                                            ref(attn(n_heads=2)), None, x, y, 4096, 1 << 30, None)
    for d in (-bytes_ + 16, -16, 0, 16, bytes_ - 16):
        refused(lib, call(1 << 20, (1 << 20) + d))
    for at in (PAGES - bytes_ + 16, PAGES, PAGES + 2 * POOL - 16):
        refused(lib, call(1 << 20, at))
