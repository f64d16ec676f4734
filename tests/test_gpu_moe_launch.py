"""How a mixture-of-experts layer is launched: the mark that a wait which ran out
leaves, and workspaces."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


def layer_of(seed, experts, hidden, inter, top_k, first=0, local=None):
    gen = torch.Generator().manual_seed(seed)
    local = experts if local is None else local
    router = P.grid_router(gen, experts, hidden, "bf16")
    w13 = (torch.randn(local, 2 * inter, hidden, generator=gen) * 0.05).bfloat16()
    w2 = (torch.randn(local, hidden, inter, generator=gen) * 0.05).bfloat16()
    return rr.MoeLayer(router.cuda(), w13.cuda(), w2.cuda(), top_k, first), router, w13, w2


def tokens_of(seed, n, hidden):
    return P.grid_tokens(torch.Generator().manual_seed(seed), n, hidden, "bf16").cuda()


@pytest.mark.parametrize("experts,hidden,inter,tokens", [(8, 128, 96, 1), (8, 128, 96, 20), (16, 512, 512, 20)])
def test_a_marked_workspace_runs_nothing(experts, hidden, inter, tokens):
    """After a wait that ran out, calls of every size leave their outputs alone until
    rr_moe_check has reported it."""
    layer, _, _, _ = layer_of(5, experts, hidden, inter, 2)
    x = tokens_of(5, tokens, hidden)
    ws, want = rr.MoeWorkspace(layer, tokens), torch.empty_like(x)
    rr.rr_moe(layer, x, want, ws)
    rr.rr_moe_check(layer, ws)
    ws.data[0] = 1                 # the mark of an earlier call
    out = torch.full_like(x, 5.0)
    ids = torch.full((tokens, 2), -7, dtype=torch.int32, device="cuda")
    for _ in range(2):
        rr.rr_moe(layer, x, out, ws, ids=ids)
    with pytest.raises(rr.RRError, match="RR_ECUDA"):
        rr.rr_moe_check(layer, ws)
    assert bool((out == 5).all()) and bool((ids == -7).all())
    rr.rr_moe(layer, x, out, ws)
    rr.rr_moe_check(layer, ws)
    assert torch.equal(out, want)


def test_a_workspace_is_ready_when_it_is_there():
    """Its zeros have been written when the constructor returns, so that the first call
    may be on any stream."""
    layer, _, _, _ = layer_of(7, 8, 128, 96, 2)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)             # about a tenth of a second
    ws = rr.MoeWorkspace(layer, 4)
    assert torch.cuda.current_stream().query()
    x, side = tokens_of(7, 4, 128), torch.cuda.Stream()
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    rr.rr_moe(layer, x, out, ws, stream=side)
    rr.rr_moe_check(layer, ws, side)
