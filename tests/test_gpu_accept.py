"""Verification of drafted tokens on the GPU, against a plain restatement in whole numbers."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _cache as R

pytestmark = pytest.mark.gpu


def run(p, q, drafts, u, v, starts, rejected=True):
    n = len(starts) - 1
    out = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
    tokens = torch.full((p.shape[0],), 77, dtype=torch.int32, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    rr.rr_accept(p, ints(drafts), u, v, out[0], tokens, q=q, starts=ints(starts),
                 rejected=out[1] if rejected else None)
    return out[0].tolist(), tokens.tolist(), out[1].tolist()


def want(p, q, drafts, u, v, starts):
    p, u, v = p.cpu(), u.cpu(), v.cpu()
    q = None if q is None else q.cpu()
    acc, tok, rej = [], [], []
    for i, (lo, hi) in enumerate(zip(starts, starts[1:])):
        a, t = R.accept(p[lo:hi], None if q is None else q[lo:hi], drafts[lo:hi], u[lo:hi], v[i])
        acc.append(a)
        rej.append(hi - lo - 1 - a)
        tok += drafts[lo:lo + a] + [t] + [-1] * (hi - lo - 1 - a)
    return acc, tok, rej


def probabilities(gen, rows, vocab, sharp=2.0):
    return torch.softmax(sharp * torch.randn(rows, vocab, generator=gen), 1).cuda()


@pytest.mark.parametrize("vocab", [1, 2, 31, 512, 1027, 5000])
@pytest.mark.parametrize("sure", [False, True])
@pytest.mark.parametrize("counts", [[1], [4], [1, 3, 9, 2], [2] * 40])
def test_against_whole_numbers(vocab, sure, counts):
    gen = torch.Generator().manual_seed(vocab + len(counts))
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    p, q = probabilities(gen, rows, vocab), None
    if not sure:
        q = torch.softmax(torch.log(p).cpu() + 0.5 * torch.randn(rows, vocab, generator=gen), 1).cuda()
    drafts = torch.multinomial((p if sure else q).cpu(), 1, generator=gen).flatten().tolist()
    u, v = torch.rand(rows, generator=gen).cuda(), torch.rand(len(counts), generator=gen).cuda()
    assert run(p, q, drafts, u, v, starts) == want(p, q, drafts, u, v, starts)
    # Rows at odd places.
    store = torch.zeros(rows, vocab + 3, device="cuda")
    store[:, 1:-2] = p
    assert run(store[:, 1:-2], q, drafts, u, v, starts) == want(p, q, drafts, u, v, starts)


def test_special_values():
    """NaN, negative and large values, ends of the number range, drafts out of the vocabulary."""
    nan, inf = math.nan, math.inf
    p = torch.tensor([[0.5, 0.25, 0.25, 0.0], [nan, 0.5, nan, 0.25], [-1.0, 0.0, -0.0, 0.0], [inf, 2.0, 1.0, 0.5],
                      [2.0 ** -43, 2.0 ** -42, 1.5 * 2.0 ** -42, 2.5 * 2.0 ** -42], [1e-45, 1.0, 1e-38, 2.0 ** -18],
                      [0.25, 0.25, 0.25, 0.25], [0.5, 0.5, 0.0, 0.0]], device="cuda")
    rows = p.shape[0]
    for starts in ([0, 1, 2, 3, 4, 5, 6, 7, 8], [0, 3, 5, 8], [0, 8]):
        n = len(starts) - 1
        for drafts in ([1] * rows, [0, 4, -1, 3, 1 << 30, 2, 0, 1], [3] * rows):
            for uu in (0.0, 0.3, 1.0, nan):
                for vv in (0.0, 0.5, 1.0 - 2.0 ** -24, 1.0, -3.0, 9.0, 2.0 ** -31):
                    u, v = torch.full((rows,), uu, device="cuda"), torch.full((n,), vv, device="cuda")
                    for q in (None, p, p.flip(1).contiguous()):
                        assert run(p, q, drafts, u, v, starts) == want(p, q, drafts, u, v, starts)


def test_long_vocabulary():
    gen = torch.Generator().manual_seed(5)
    for rows, starts in ((3, [0, 3]), (40, list(range(41)))):
        p = probabilities(gen, rows, 151936, 3.0)
        q = probabilities(gen, rows, 151936, 3.0)
        drafts = torch.multinomial(q.cpu(), 1, generator=gen).flatten().tolist()
        u = torch.rand(rows, generator=gen).cuda()
        for x in (0.0, 0.999999, None):
            v = torch.rand(len(starts) - 1, generator=gen).cuda() if x is None else torch.full((len(starts) - 1,), x, device="cuda")
            got = run(p, q, drafts, u, v, starts)
            if len(starts) == 2:
                assert got == want(p, q, drafts, u, v, starts)
            else:
                # One row each: the sums by numpy's integers.
                units = torch.round(p.double() * 2.0 ** 42).long()
                sums = units.cumsum(1)
                t = [int(sums[i, -1]) * min(int(float(v[i]) * 2 ** 31), 2 ** 31 - 1) >> 31 for i in range(rows)]
                assert got[1] == [int((sums[i] <= t[i]).sum()) for i in range(rows)]


def test_sampling_without_drafts():
    gen = torch.Generator().manual_seed(2)
    p, v = probabilities(gen, 9, 300), torch.rand(9, generator=gen).cuda()
    accepted = torch.empty(9, dtype=torch.int32, device="cuda")
    tokens = torch.empty_like(accepted)
    rr.rr_accept(p, None, None, v, accepted, tokens)
    assert accepted.tolist() == [0] * 9
    assert tokens.tolist() == [R.accept(p[i:i + 1].cpu(), None, [], [], v[i])[1] for i in range(9)]


def test_starts_that_do_not_fit():
    p = torch.full((4, 8), 0.125, device="cuda")
    u, v = torch.zeros(4, device="cuda"), torch.zeros(3, device="cuda")
    acc, tok, rej = run(p, None, [1] * 4, u, v, [0, 0, 2, 5])
    assert acc == [-1, 1, -1] and rej == [0, 0, 0] and tok == [1, 0, 77, 77]
    acc, tok, rej = run(p, None, [1] * 4, u, v, [-1, 2, 1, 3])
    assert acc == [-1, -1, 1] and tok == [77, 1, 0, 77]


def test_distribution():
    """Accepted or drawn again, a token is one of p: over 20000 sequences each token's share
    is within 5 standard deviations."""
    gen = torch.Generator().manual_seed(11)
    n, vocab = 20000, 6
    p1, q1 = probabilities(gen, 1, vocab, 1.0), probabilities(gen, 1, vocab, 1.0)
    p, q = p1.repeat(2 * n, 1), q1.repeat(2 * n, 1)
    drafts = torch.multinomial(q1.cpu().expand(2 * n, vocab), 1, generator=gen).flatten().int().cuda()
    u, v = torch.rand(2 * n, generator=gen).cuda(), torch.rand(n, generator=gen).cuda()
    starts = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    acc = torch.empty(n, dtype=torch.int32, device="cuda")
    tok = torch.empty(2 * n, dtype=torch.int32, device="cuda")
    rr.rr_accept(p, drafts, u, v, acc, tok, q=q, starts=starts)
    share = torch.bincount(tok[::2].long(), minlength=vocab).double().cpu() / n
    want = p1[0].double().cpu()
    assert bool(((share - want).abs() < 5 * (want * (1 - want) / n).sqrt()).all())
