"""The order in which the products add up."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


def shifted(x, offset, extra):
    """The same rows elsewhere: `offset` elements past an aligned address, a longer stride."""
    n, cols = x.shape
    store = torch.zeros(offset + n * (cols + extra), dtype=x.dtype, device="cuda")
    view = store[offset:].view(n, cols + extra)[:, :cols]
    view.copy_(x)
    return view


@pytest.mark.parametrize("rows,cols,tokens,pair", [
    (6144, 4096, 16, False), (4096, 4096, 16, False), (4096, 12288, 4, False), (24576, 4096, 12, True),
    (1000, 30000, 13, False), (2500, 640, 9, False)])
def test_matvec_alignment_leaves_the_bits(rows, cols, tokens, pair):
    """Where the tokens lie does not enter the order of a product's sums."""
    gen = torch.Generator("cuda").manual_seed(rows + cols)
    w = (torch.randn(rows, cols, device="cuda", generator=gen) * 0.05).bfloat16()
    q = rr.Quantized(rows, cols, 128, "bf16", pair)
    rr.rr_quantize(q, w)
    x = torch.randn(tokens, cols, device="cuda", generator=gen).bfloat16()
    want = torch.empty(tokens, q.n_out, device="cuda")
    rr.rr_matvec(q, x, want)
    for offset, extra in ((1, 0), (3, 5), (8, 0), (0, 8)):
        got = torch.full_like(want, 9.0)
        rr.rr_matvec(q, shifted(x, offset, extra), got)
        assert torch.equal(got, want), (offset, extra)
    stored = torch.full((tokens, q.n_out + 3), 9.0, device="cuda")
    rr.rr_matvec(q, x, stored[:, 1:-2])
    assert torch.equal(stored[:, 1:-2], want)


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("tokens", [1, 8, 16, 40])
def test_moe_alignment_leaves_the_bits(tokens, group):
    """Nor into that of a layer's; nor does a workspace's history."""
    gen = torch.Generator().manual_seed(tokens)
    hidden, inter = 1000, 520
    w13 = (torch.randn(8, 2 * inter, hidden, generator=gen) * 0.05).bfloat16().cuda()
    w2 = (torch.randn(8, hidden, inter, generator=gen) * 0.05).bfloat16().cuda()
    if group:
        a, b = rr.Quantized(2 * inter, hidden, group, "bf16", True, 8), rr.Quantized(hidden, inter, group, "bf16", False, 8)
        rr.rr_quantize(a, w13)
        rr.rr_quantize(b, w2)
    else:
        a, b = w13, w2
    layer = rr.MoeLayer(P.grid_router(gen, 8, hidden, "bf16").cuda(), a, b, 3)
    x = P.grid_tokens(gen, tokens, hidden, "bf16").cuda()
    ws = rr.MoeWorkspace(layer, 64)
    want = torch.empty_like(x)
    rr.rr_moe(layer, x, want, ws)
    other = P.grid_tokens(gen, 64, hidden, "bf16").cuda()
    rr.rr_moe(layer, other, torch.empty_like(other), ws)
    for offset, extra in ((1, 0), (3, 5), (8, 0)):
        got = torch.full_like(want, 9.0)
        rr.rr_moe(layer, shifted(x, offset, extra), got, ws)
        assert torch.equal(got, want), (offset, extra)
    rr.rr_moe_check(layer, ws)
