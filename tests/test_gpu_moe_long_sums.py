"""Long sums of a layer's products, to what float32 additions that round to nearest
give.  A matrix instruction cuts its sum off instead, always towards zero, so a
long chain of them would drift.

A row's weights are positive, of 8 bits each over 11 binades, and its last three are
minus the sum of the others in three 16-bit parts, so that the result is what the
sum's errors leave.  Bound, for n columns with sums P_b of the first b blocks of 64
and S of all: an addition per block, at most 2^-24 of the sum so far, which is at most
P_b (a row cut between warps has smaller ones); 16 more where warps and the last
step join them; within a block four instructions that cut off at most 2^-23 of the
block's sum, four more times of S for the block of the last three columns and as much
for where the row's parts straddle two blocks."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


def rows_of(rows, cols, kind, gen):
    """(weights [rows, cols], the exact sum of each row, the bound on its error)."""
    t = P.TYPES[kind]
    bits = torch.randint(128, 256, (rows, cols), device="cuda", generator=gen) / 128.0
    w = (bits * 2.0 ** -torch.randint(0, 11, (rows, cols), device="cuda", generator=gen)).to(t)
    w[:, -3:] = 0
    whole = w.double()
    prefix = whole.cumsum(1)
    total = prefix[:, -1]
    rest = total.clone()
    for i in (3, 2, 1):
        w[:, -i] = -rest.to(t)
        rest += w[:, -i].double()
    bound = prefix[:, 63::64].sum(1) * 2.0 ** -24 + total * (17 * 2.0 ** -24 + 12 * 2.0 ** -23)
    return w, w.double().sum(1), bound


def run(w13, w2, experts):
    """One token of ones through `experts` copies of an expert, with equal weights."""
    hidden, inter = w2.shape
    a = w13.unsqueeze(0).expand(experts, -1, -1).contiguous()
    b = w2.unsqueeze(0).expand(experts, -1, -1).contiguous()
    layer = rr.MoeLayer(torch.zeros(experts, hidden, dtype=w2.dtype, device="cuda"), a, b, experts)
    x, ws = torch.ones(1, hidden, dtype=w2.dtype, device="cuda"), rr.MoeWorkspace(layer, 1)
    out = torch.empty_like(x)
    rr.rr_moe(layer, x, out, ws)
    rr.rr_moe_check(layer, ws)
    return out[0].double()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("hidden", [16384, 16381])
def test_first_product(hidden, kind):
    """gate is 28 (and silu leaves it: exp(-28) is under 2^-24), up the row's sum."""
    gen = torch.Generator("cuda").manual_seed(hidden)
    inter, experts = 2048, 12          # more strips than warps: most rows are one warp's
    w, exact, bound = rows_of(inter, hidden, kind, gen)
    w13 = torch.zeros(2 * inter, hidden, dtype=P.TYPES[kind], device="cuda")
    w13[:inter, 0] = 28
    w13[inter:] = w
    w2 = torch.zeros(hidden, inter, dtype=P.TYPES[kind], device="cuda")
    pick = torch.arange(hidden, device="cuda") % inter
    w2[torch.arange(hidden, device="cuda"), pick] = 1
    got = run(w13, w2, experts)
    want = 28 * exact[pick]
    tol = 28 * bound[pick]
    assert bool(((got - want).abs() <= tol + P.rounding(want.abs() + tol, kind)).all()), \
        ((got - want).abs() / tol).max().item()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("inter", [8192, 8187])
def test_second_product(inter, kind):
    """Every h is 28."""
    gen = torch.Generator("cuda").manual_seed(inter)
    hidden, experts = 4096, 12
    w2, exact, bound = rows_of(hidden, inter, kind, gen)
    w13 = torch.zeros(2 * inter, hidden, dtype=P.TYPES[kind], device="cuda")
    w13[:inter, 0] = 28
    w13[inter:, 0] = 1
    got = run(w13, w2, experts)
    want, tol = 28 * exact, 28 * bound
    assert bool(((got - want).abs() <= tol + P.rounding(want.abs() + tol, kind)).all()), \
        ((got - want).abs() / tol).max().item()
