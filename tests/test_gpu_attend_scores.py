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
