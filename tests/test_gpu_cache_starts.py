"""Lists of starts that do not fit: what append, extend and attend make of them."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests.test_gpu_cache import Both, ints, same, state

pytestmark = pytest.mark.gpu

LEAST, MOST = -(1 << 31), (1 << 31) - 1


def fits(starts, i, rows):
    return 0 <= starts[i] <= starts[i + 1] <= rows


@pytest.mark.parametrize("seqs,starts", [
    ([0, 1], [0, 3, 7]), ([0, 1], [0, 6, 7]), ([0, 1], [0, 3, MOST]), ([0, 1], [-1, 3, 6]), ([0], [-3, 4]),
    ([0], [LEAST + 7, 10]), ([0], [LEAST, 6]), ([0], [LEAST + 5, MOST]), ([0], [MOST, LEAST]), ([0], [6, 0]),
    ([0, 1], [0, 2, 1]), ([0, 1, 2], [0, 2, LEAST, 6]), ([0, 1], [7, 8, 9]), ([0, 1], [MOST - 1, MOST, MOST]),
    ([0, 99], [0, 2, 2]), ([-1, 0], [0, 0, 2]), ([0] + [3] * 9 + [12], [0, 2] + [6] * 10), ])
def test_append_leaves_out_sequences_whose_rows_do_not_fit(seqs, starts):
    """They are marked, too, where no row shows it; the others are written (where the list
    descends: those and no more)."""
    b = Both()
    b.add([0, 1, 2, 3], [20, 9, 8, 10])
    c = b.c
    x = torch.randn(6, 2, 32, generator=b.gen).bfloat16()
    before = state(c)
    rr.rr_cache_append(c, 1, x.cuda(), x.cuda(), ints(seqs), starts=ints(starts))
    for i, s in enumerate(seqs):
        if fits(starts, i, 6) and 0 <= s < 12 and starts[i] < starts[i + 1]:
            rows = x[starts[i]:starts[i + 1]]
            b.b.append(1, rows, rows, [s], [len(rows)])
    with pytest.raises(rr.RRError, match="range"):
        rr.rr_cache_check(c)
    assert torch.equal(c.book[64:], before[0][64:])
    if starts != sorted(starts):
        got, was, want = (y.cpu().view(torch.int16) for y in (c.pages, before[1], b.b.pages))
        assert bool(((got == was) | (got == want)).all())
    else:
        b.check()


@pytest.mark.parametrize("n", [12, 40])
def test_long_lists_are_looked_through(n):
    """One row, many sequences: a number out of range anywhere in the list, of no rows."""
    b = Both(max_seqs=n, n_pages=60)
    b.add([3], [9])
    x = torch.randn(1, 2, 32, generator=b.gen).bfloat16()
    for at in (0, 1, n - 1):
        seqs = [3] + [5] * (n - 1)
        seqs[at] = n if at else 3
        rr.rr_cache_append(b.c, 0, x.cuda(), x.cuda(), ints(seqs), starts=ints([0] + [1] * n))
        if at:
            with pytest.raises(rr.RRError, match="range"):
                rr.rr_cache_check(b.c)
        b.b.append(0, x, x, [3], [1])
        b.check()


@pytest.mark.parametrize("starts", [[MOST, LEAST], [LEAST, MOST], [5, 4], [LEAST + 1, LEAST], [0, LEAST]])
def test_extend_refuses_counts_that_are_none(starts):
    b = Both()
    b.add([0], [5])
    before = state(b.c)
    rr.rr_cache_extend(b.c, ints([0]), starts=ints(starts))
    with pytest.raises(rr.RRError, match="room" if starts[1] > starts[0] else "range"):
        rr.rr_cache_check(b.c)
    assert same(b.c, before)


@pytest.mark.parametrize("starts", [[MOST, LEAST], [LEAST, MOST], [LEAST, 1], [0, MOST], [1, LEAST], [-1, 1], [2, 1], [1, 3]])
def test_attend_leaves_out_what_does_not_fit(starts):
    b = Both()
    b.add([0], [5])
    x = torch.ones(2, 2, 32, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(x, 9.0)
    rr.rr_attend(b.c, 0, x, out, ints([0]), rr.AttendWorkspace(b.c, 2), starts=ints(starts))
    with pytest.raises(rr.RRError, match="range"):
        rr.rr_cache_check(b.c)
    assert bool((out == 9.0).all())
