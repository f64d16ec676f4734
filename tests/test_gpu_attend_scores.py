"""Attention where scores are not finite, or nearly not: what lse and the results are then, in
one piece and joined from several."""
import math

import pytest
import torch

from tests import _cache as R
from tests.test_gpu_attend import Case, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,dim", [(2, 64), (40, 64), (3, 200)])
@pytest.mark.parametrize("length", [60, 3000, 20000])
def test_a_query_that_is_nan(kind, n_q, dim, length):
    """All of its scores are NaN, in every piece: out and lse are, and those of no other row."""
    c = Case([length, 50], [2, 1], n_q=n_q, n_kv=1, dim=dim, kind=kind)
    q = c.q.clone()
    q[1, n_q - 1, 3] = math.nan
    out, lse = c.run(q=q.cuda())
    assert bool(out[1, n_q - 1].isnan().all()) and bool(lse[1, n_q - 1].isnan())
    assert int(out.isnan().any(2).sum()) == 1 and int(lse.isnan().sum()) == 1
    good = c.run()
    out[1, n_q - 1], lse[1, n_q - 1] = good[0][1, n_q - 1], good[1][1, n_q - 1]
    c.check(out, lse)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("where", ["first", "last"])
def test_a_piece_of_nan_keys(kind, where):
    """Keys that are NaN for the length of whole pieces, beside finite ones."""
    c = Case([3000], [1], n_q=2, n_kv=1, dim=64, kind=kind)
    c.k[0][slice(0, 600) if where == "first" else slice(2400, 3000), 0, 5] = math.nan
    put(c)
    out, lse = c.run()
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,dim", [(2, 64), (40, 64), (3, 200), (1, 1)])
@pytest.mark.parametrize("length", [60, 3000])
def test_scores_of_infinity(kind, n_q, dim, length):
    """lse, the logarithm of the sum, is infinity, out NaN (infinity less infinity), for the rows
    that see the key; with a NaN score as well, lse is NaN."""
    c = Case([length, 50], [3, 1], n_q=n_q, n_kv=1, dim=dim, kind=kind)
    c.q = c.q.abs() + 1
    good = c.run()
    c.check(*good)
    k = c.k[0].clone()
    at = length - 2                  # the first of the three new tokens does not see it
    c.k[0][at, 0, 0] = math.inf
    if length > 60:
        c.k[0][700, 0, 0] = -math.inf
    put(c)
    out, lse = c.run()
    assert bool((lse[1:3] == math.inf).all()) and bool(out[1:3].isnan().all())
    assert bool(lse[0].isfinite().all()) and bool(out[0].isfinite().all())
    assert torch.equal(lse[3], good[1][3]) or bool((lse[3] - good[1][3]).abs().max() < 1e-4)
    for nan in (at, 0, length - 1):
        c.k[0] = k.clone()
        c.k[0][at, 0, 0] = math.inf
        c.k[0][nan, 0, -1] = math.nan
        put(c)
        out, lse = c.run()
        seen = 2 if nan == length - 1 else 1     # the rows from here on see both
        assert bool(lse[seen:3].isnan().all()) and bool(out[1:3].isnan().all())
        assert bool((lse[1:seen] == math.inf).all())
    # And in every row, of a negative scale.
    c.k[0] = k.clone()
    c.k[0][0, 0, 0] = -math.inf
    put(c)
    out, lse = c.run(scale=-0.25)
    assert bool((lse[:3] == math.inf).all()) and bool(out[:3].isnan().all())


def test_products_past_the_largest_float():
    """Scores of finite queries and keys that float32 has as infinity."""
    c = Case([300], [1], n_q=2, n_kv=1, dim=8)
    c.q[0, 0, :] = 3e38
    c.k[0].fill_(1.0)
    c.k[0][17] = 100.0
    c.k[0][18] = -100.0
    c.q[0, 1, :] = 1.0
    put(c)
    out, lse = c.run(scale=1.0)
    assert float(lse[0, 0]) == math.inf and bool(out[0, 0].isnan().all())
    assert abs(float(lse[0, 1]) - 800.0) < 1e-3
    assert torch.equal(out[0, 1], c.v[0][17, 0])
