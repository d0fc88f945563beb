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
