"""The weights that enter attention's second product: what is left of them where values cancel."""
import math

import pytest
import torch

from tests import _cache as R
from tests.test_gpu_attend import Case, put

pytestmark = pytest.mark.gpu

# What a weight loses on its way into the product, of itself: two parts of 8 or 11 bits, each
# rounded to nearest.  (tests/_cache.py allows float16 one part of 11.)
CUT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22}


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,dim", [(16, 32), (40, 64), (64, 128), (16, 200), (32, 256)])
def test_values_that_cancel(monkeypatch, kind, n_q, dim):
    """Two tokens; head h weighs them 1 to exp(s_h), and element h of their values is
    (exp(s_h), -1), rounded: what is left of the sum is as small as that rounding, and
    the result's own rounding with it.  A weight that is off by 2^-11 shows there."""
    monkeypatch.setitem(R.CUT, kind, CUT[kind])
    c = Case([2], [1], n_q=n_q, n_kv=1, dim=dim, kind=kind)
    t = R.TYPES[kind]
    # A score is one product, exact in 32 bits.
    s = torch.linspace(0.01, 0.5, n_q).to(t)
    c.q = torch.zeros(1, n_q, dim, dtype=t)
    c.q[0, :, 0] = s
    c.k = [torch.zeros(2, 1, dim, dtype=t)]
    c.k[0][1, 0, 0] = 1.0
    c.v = [torch.zeros(2, 1, dim, dtype=t)]
    m = min(n_q, dim)
    c.v[0][0, 0, :m] = torch.exp(s[:m].double()).to(t)
    c.v[0][1, 0, :m] = -1.0
    put(c)
    out, lse = c.run(scale=1.0)
    c.check(out, lse, scale=1.0)
    # The bound is under a weight's last of 11 bits where values cancel.
    o, tol, _, _ = R.attend(c.q, c.k[0], c.v[0], 1, 1.0, kind)
    d = torch.arange(m)
    assert float(tol[0, d, d].max()) < 2.0 ** -13


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("lengths,counts,n_q,n_kv,dim", [
    ([700, 3, 130, 41], [3, 1, 3, 2], 2, 1, 36), ([400, 1200, 70], [5, 5, 5], 16, 2, 128),
    ([300, 129], [4, 1], 12, 1, 192), ([3000], [1], 8, 2, 64)])
def test_bounds_of_two_parts(monkeypatch, kind, lengths, counts, n_q, n_kv, dim):
    """The ordinary bounds, with what two parts lose in place of one."""
    monkeypatch.setitem(R.CUT, kind, CUT[kind])
    c = Case(lengths, counts, n_q=n_q, n_kv=n_kv, dim=dim, kind=kind, seed=5)
    c.check(*c.run())


def test_small_weights_of_two_parts(monkeypatch):
    """Float16's second part ends at 2^-32 of the largest weight: many weights of 2^-13 of it,
    whose values cancel but for their rounding."""
    monkeypatch.setitem(R.CUT, "f16", CUT["f16"])
    n, dim = 401, 64
    c = Case([n], [1], n_q=1, n_kv=1, dim=dim, kind="f16", seed=2)
    c.q = torch.zeros(1, 1, dim).half()
    c.q[0, 0, 0] = 1.0
    c.k[0] = torch.zeros(n, 1, dim).half()
    c.k[0][1:, 0, 0] = -9.0 - torch.rand(n - 1, generator=torch.Generator().manual_seed(1)).half()
    w = torch.exp(c.k[0][:, 0, 0].double())
    v = torch.randn(n, dim, generator=torch.Generator().manual_seed(3)).double()
    v[0] = 0
    v[1:] -= (w[1:] @ v[1:]) / w[1:].sum()
    c.v[0] = v.half()[:, None]
    put(c)
    out, lse = c.run(scale=1.0)
    c.check(out, lse, scale=1.0)
    assert math.isfinite(float(lse[0, 0]))
