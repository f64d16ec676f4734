"""Marked caches on the GPU: what a mark stops, what it leaves, and what is reported of it."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests.test_gpu_cache import Both, ints, same, starts_of, state

pytestmark = pytest.mark.gpu


def used(compacted, **kw):
    """A cache whose last extension took copies, with free pages between others; compacted
    before that, or never."""
    b = Both(n_pages=kw.pop("n_pages", 60), **kw)
    b.add([0, 2, 4], [19, 5, 9])
    if compacted:
        b.truncate([2])
        b.compact()
        b.add([2], [5])
    b.add([5, 6], [8, 8])
    b.truncate([5])
    b.fork([0], [1])
    b.add([1, 0], [3, 2])
    b.truncate([4])
    b.check()
    return b


def late_mark(b, by):
    """A mark by a call that does all but for what does not fit (here: nothing fits)."""
    x = torch.ones(1, 2, 32, dtype=torch.bfloat16, device="cuda")
    if by == "append":
        rr.rr_cache_append(b.c, 0, x, x, ints([12]))
    else:
        rr.rr_attend(b.c, 0, x, torch.empty_like(x), ints([-1]), rr.AttendWorkspace(b.c, 2))


@pytest.mark.parametrize("compacted", [False, True])
@pytest.mark.parametrize("by", ["append", "attend"])
@pytest.mark.parametrize("call", ["compact", "fork", "extend", "truncate"])
@pytest.mark.parametrize("n_pages", [60, 5000])
def test_calls_behind_a_late_mark(compacted, by, call, n_pages):
    """The first call that would write the book, and those behind it, leave the cache as it was."""
    b = used(compacted, n_pages=n_pages)
    c = b.c
    before = state(c)
    late_mark(b, by)
    calls = {"compact": lambda: rr.rr_cache_compact(c), "fork": lambda: rr.rr_cache_fork(c, ints([0]), ints([7])),
             "extend": lambda: rr.rr_cache_extend(c, ints([0, 1, 2])), "truncate": lambda: rr.rr_cache_truncate(c, ints([0]))}
    calls[call]()
    assert same(c, before)
    for again in calls.values():
        again()
    assert same(c, before)
    with pytest.raises(rr.RRError, match="range"):
        rr.rr_cache_check(c)
    rr.rr_cache_check(c)
    assert same(c, before)
    # And goes on as if nothing had been.
    b.compact()
    b.add([0, 1, 7], [2, 9, 17])
    b.check()


@pytest.mark.parametrize("kw", [dict(), dict(n_pages=3000, max_pages=400, max_seqs=40)])
@pytest.mark.parametrize("page", ["n_pages", -1, -(1 << 31), (1 << 31) - 1])
@pytest.mark.parametrize("call", ["fork", "truncate", "truncate to 9"])
def test_pages_out_of_range_are_found_before_anything_is_written(kw, page, call):
    b = Both(**kw)
    b.add([0, 2, 3, 4], [40, 5, 9, 30])
    c = b.c
    good = int(c.table[0, 3])
    c.table[0, 3] = c.n_pages if page == "n_pages" else page
    before = state(c)
    if call == "fork":
        rr.rr_cache_fork(c, ints([2, 0, 4, 0]), ints([1, 5, 6, 7]))
    elif call == "truncate":
        rr.rr_cache_truncate(c, ints([2, 0, 4]))
    else:
        rr.rr_cache_truncate(c, ints([2, 4, 0]), ints([1, 20, 31]))
    with pytest.raises(rr.RRError, match="table"):
        rr.rr_cache_check(c)
    assert same(c, before)
    c.table[0, 3] = good
    b.fork([2, 0, 4, 0], [1, 5, 6, 7])
    b.truncate([2, 0])
    b.check()


@pytest.mark.parametrize("by", ["append", "attend"])
def test_what_a_mark_says(by):
    """A call that left something out was done for the rest; one that was not done was not."""
    b = used(False)
    late_mark(b, by)
    with pytest.raises(rr.RRError) as e:
        rr.rr_cache_check(b.c)
    assert "left something out" in str(e.value) and "not done" not in str(e.value)
    rr.rr_cache_extend(b.c, ints([0, 0]))
    with pytest.raises(rr.RRError) as e:
        rr.rr_cache_check(b.c)
    assert "not done" in str(e.value) and "left something out" not in str(e.value)
    late_mark(b, by)
    rr.rr_cache_extend(b.c, ints([0]))
    with pytest.raises(rr.RRError) as e:
        rr.rr_cache_check(b.c)
    assert "left something out" in str(e.value) and "not done" in str(e.value)
    b.check()


def test_append_and_attend_go_on_behind_a_late_mark():
    """They do what fits, as they do in the call that marks."""
    b = used(False)
    late_mark(b, "append")
    b.append(1, [0, 1, 2])
    x = torch.ones(1, 2, 32, dtype=torch.bfloat16, device="cuda")
    out = [torch.zeros_like(x) for _ in range(2)]
    ws = rr.AttendWorkspace(b.c, 2)
    rr.rr_attend(b.c, 1, x, out[0], ints([0]), ws)
    with pytest.raises(rr.RRError, match="left something out"):
        rr.rr_cache_check(b.c)
    b.check()
    rr.rr_attend(b.c, 1, x, out[1], ints([0]), ws)
    assert out[0].any() and torch.equal(out[0], out[1])
    # Behind a call that was not done they leave all as it is.
    rr.rr_cache_extend(b.c, ints([0, 0]))
    before = state(b.c)
    out[0].fill_(9.0)
    rr.rr_cache_append(b.c, 0, x, x, ints([0]))
    rr.rr_attend(b.c, 1, x, out[0], ints([0]), ws)
    assert same(b.c, before) and bool((out[0] == 9.0).all())
    with pytest.raises(rr.RRError, match="not done.*twice"):
        rr.rr_cache_check(b.c)
