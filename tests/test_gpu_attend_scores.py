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


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("x", [1e6, 3e9, 1e11, 1e20, 3.0e38, 3.1e38, 3.25e38, 3.35e38])
@pytest.mark.parametrize("tokens", [1, 2, 300, 3000])
def test_scores_as_large_as_floats(kind, n_q, sign, x, tokens):
    """Finite scores up to nearly 2^128 (in log2) of either sign: equal ones weigh the same."""
    c = Case([tokens], [1], n_q=n_q, n_kv=1, dim=1, kind=kind)
    c.q.fill_(1.0)
    c.k[0].fill_(sign * 1.5)
    c.v[0].fill_(2.0)
    c.v[0][::2] = 4.0
    put(c)
    scale = math.log(2.0) * x / 1.5
    out, lse = c.run(scale=scale)
    assert bool((out == (4.0 if tokens == 1 else 3.0)).all())
    # (The factor to log2 and back, the product, the logarithm of the count: a few roundings.)
    want = sign * x * math.log(2.0) + math.log(tokens)
    assert bool(((lse.double() / want - 1).abs() < 2.0 ** -20).all())
    # Twice the score (half of it, where that overflows): one key alone, or all others.
    if tokens > 2:
        c.k[0][tokens - 2] = sign * 0.75
        put(c)
        out, lse = c.run(scale=scale)
        if sign < 0:
            assert bool((out == c.v[0][tokens - 2]).all())
            want = -0.5 * x * math.log(2.0)
        else:
            rest = torch.cat([c.v[0][:tokens - 2], c.v[0][tokens - 1:]]).double().mean()
            assert bool(((out.double() - rest).abs() <= R.ROUND[kind] * rest + 2.0 ** -13).all())
            want = x * math.log(2.0) + math.log(tokens - 1)
        assert bool(((lse.double() / want - 1).abs() < 2.0 ** -20).all())
