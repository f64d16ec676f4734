"""Verification of drafted tokens where a block has next to nothing to do before it sends its
sums to the others of its cluster: small vocabularies, few or no drafts, many sequences."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _cache as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 300])
@pytest.mark.parametrize("n", [1, 2, 16, 17, 150, 3000])
def test_sampling_from_small_vocabularies(n, vocab):
    gen = torch.Generator().manual_seed(n + vocab)
    p = torch.softmax(2 * torch.randn(n, vocab, generator=gen), 1)
    v = torch.rand(n, generator=gen)
    want = [R.accept(p[i:i + 1], None, [], [], v[i])[1] for i in range(n)]
    p, v = p.cuda(), v.cuda()
    outs = [torch.full((2, n), 77, dtype=torch.int32, device="cuda") for _ in range(20)]
    for o in outs:
        rr.rr_accept(p, None, None, v, o[0], o[1])
    for o in outs:
        assert o[0].tolist() == [0] * n and o[1].tolist() == want


@pytest.mark.parametrize("sure", [False, True])
@pytest.mark.parametrize("n", [1, 16, 17, 700])
def test_a_refused_draft_whose_rest_is_zero(n, sure):
    """The second pass over p, right behind the first: q is p, or all of p is the draft."""
    p = torch.zeros(2 * n, 5, device="cuda")
    p[:, 3] = 0.5
    drafts = torch.full((2 * n,), 3, dtype=torch.int32, device="cuda")
    u, v = torch.ones(2 * n, device="cuda"), torch.full((n,), 0.25, device="cuda")
    starts = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    for _ in range(20):
        acc = torch.full((n,), 77, dtype=torch.int32, device="cuda")
        tok = torch.full((2 * n,), 77, dtype=torch.int32, device="cuda")
        rr.rr_accept(p, drafts, u, v, acc, tok, q=None if sure else p, starts=starts)
        assert acc.tolist() == [0] * n
        assert tok.tolist() == [3, -1] * n
