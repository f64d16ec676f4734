"""The products at the ends of the number range: sums that pass it on the way and
come back, and infinite weights."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("w_exp,x_exp", [(-30, 126), (-100, 127), (-20, 120), (110, -20), (120, -60), (-60, -30)])
def test_matvec_large_tokens_small_scales(w_exp, x_exp, group):
    """Tokens or scales near bfloat16's largest, whose products are far from it:
    no sum on the way may overflow that the result does not."""
    gen = torch.Generator().manual_seed(group)
    rows, cols = 40, 300
    w = (torch.randn(rows, cols, generator=gen).clamp(-3, 3) * 2.0 ** w_exp).bfloat16()
    w[3] = 1.5 * 2.0 ** w_exp           # codes of one sign
    x = ((1 + torch.rand(5, cols, generator=gen) * 0.9) * 2.0 ** x_exp).bfloat16()
    x[1] *= torch.randn(cols, generator=gen).sign()
    q = rr.Quantized(rows, cols, group)
    rr.rr_quantize(q, w.cuda())
    vals = P.values(*P.quantize(w, group), group)
    out = torch.empty(5, rows, device="cuda")
    rr.rr_matvec(q, x.cuda(), out)
    want, tol = P.matvec(vals, x, False, "f32")
    assert bool((want.abs() < 2.0 ** 126).all())
    P.check(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("inter", [48, 43])
@pytest.mark.parametrize("tokens", [1, 3, 20])
def test_moe_infinite_weights(tokens, inter, kind):
    """An infinite weight of the second product: its row is infinite, by the sign of
    its h, or NaN where h is zero or two infinities meet; other rows are as without it."""
    gen = torch.Generator().manual_seed(inter + tokens)
    hidden = 64
    w13 = (torch.randn(1, 2 * inter, hidden, generator=gen) * 0.1).to(P.TYPES[kind])
    w2 = (torch.randn(1, hidden, inter, generator=gen) * 0.1).to(P.TYPES[kind])
    w13[0, 9] = 0                         # gate 9 is 0, so is h
    x = P.grid_tokens(gen, tokens, hidden, kind)
    router = torch.zeros(1, hidden, dtype=P.TYPES[kind])
    w2[0, 5, 20] = math.inf
    w2[0, 17, 31] = -math.inf
    w2[0, 30, 9] = math.inf
    w2[0, 41, 2] = w2[0, 41, 3] = math.inf
    layer = rr.MoeLayer(router.cuda(), w13.cuda(), w2.cuda(), 1)
    ws = rr.MoeWorkspace(layer, tokens)
    out = torch.empty(tokens, hidden, dtype=P.TYPES[kind], device="cuda")
    rr.rr_moe(layer, x.cuda(), out, ws)
    g = x.double() @ w13[0, :inter].double().T
    h = P.silu(g) * (x.double() @ w13[0, inter:].double().T)
    spoiled = (h.unsqueeze(1) * w2[0].double()).sum(2)
    zero, one = torch.zeros(tokens, 1, dtype=torch.int64), torch.ones(tokens, 1, dtype=torch.float64)
    _, tol = P.moe(x, zero, one, w13.double(), w2.double().nan_to_num(0.0, 0.0, 0.0), 0, kind)
    assert bool(torch.isinf(spoiled[:, [5, 17]]).all()) and bool(torch.isnan(spoiled[:, 30]).all())
    P.check(out, spoiled, tol)
