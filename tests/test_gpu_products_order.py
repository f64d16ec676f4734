"""The order in which the products add up."""
import pytest
import torch

import paper_2512_22492_gb300 as rr

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
