"""Pages of the cache on the GPU, against a plain restatement (tests/_cache.py)."""
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _cache as R

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return ints(out)


class Both:
    """A cache and its restatement; every call goes to both."""

    def __init__(self, layers=2, n_kv=2, dim=32, n_pages=40, max_seqs=12, max_pages=8, page=8,
                 dtype="bf16", seed=0):
        self.gen = torch.Generator().manual_seed(seed)
        self.c = rr.Cache(layers, n_kv, dim, n_pages, max_seqs, max_pages, page_tokens=page, dtype=dtype)
        pages = torch.randn(self.c.pages.shape, generator=self.gen).to(R.TYPES[dtype])
        self.c.pages.copy_(pages)
        self.b = R.Book(pages, max_seqs, page)

    def rows(self, n):
        x = torch.randn(n, self.c.n_kv, self.c.dim, generator=self.gen).to(self.c.torch_dtype)
        return x

    def extend(self, seqs, counts=None):
        ok = self.b.extend(seqs, counts or [1] * len(seqs))
        rr.rr_cache_extend(self.c, ints(seqs), starts=None if counts is None else starts_of(counts))
        return ok

    def append(self, layer, seqs, counts=None):
        n = len(seqs) if counts is None else sum(counts)
        k, v = self.rows(n), self.rows(n)
        self.b.append(layer, k, v, seqs, counts or [1] * len(seqs))
        rr.rr_cache_append(self.c, layer, k.cuda(), v.cuda(), ints(seqs),
                           starts=None if counts is None else starts_of(counts))

    def add(self, seqs, counts=None):
        self.extend(seqs, counts)
        for layer in range(self.c.layers):
            self.append(layer, seqs, counts)

    def fork(self, parents, children):
        self.b.fork(parents, children)
        rr.rr_cache_fork(self.c, ints(parents), ints(children))

    def truncate(self, seqs, drop=None):
        self.b.truncate(seqs, drop or [self.b.lens[s] for s in seqs])
        rr.rr_cache_truncate(self.c, ints(seqs), None if drop is None else ints(drop))

    def compact(self):
        self.b.compact()
        rr.rr_cache_compact(self.c)

    def check(self):
        rr.rr_cache_check(self.c)
        assert self.c.lengths.tolist() == self.b.lens
        assert self.c.table.tolist() == self.b.table(self.c.max_pages)
        assert self.c.refs.tolist() == self.b.refs
        got, want = self.c.pages.cpu(), self.b.pages
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("kw", [
    dict(), dict(dim=36, page=16, dtype="f16", n_kv=1, layers=1), dict(dim=1, page=8, max_seqs=3, n_pages=9),
    dict(dim=129, page=128, n_pages=7, max_pages=2), dict(dim=256, page=64, n_kv=3, layers=5, n_pages=14),
    # More pages and sequences than one block's threads, so that eight share the work.
    dict(dim=8, page=8, layers=1, n_kv=1, n_pages=9001, max_seqs=700, max_pages=400)])
def test_a_run_of_calls(kw):
    b = Both(**kw)
    page, most = b.c.page_tokens, b.c.max_pages * b.c.page_tokens
    b.add([0, 2], [min(2 * page + 3, most - 9), 1])
    b.check()
    b.fork([0], [1])
    b.check()
    b.add([1])                       # 0 holds the page as well: a copy
    b.check()
    b.truncate([1])
    b.fork([0, ], [1])
    b.add([1, 0])                    # all holders are listed: one copy, the last keeps the page
    b.check()
    b.truncate([0, 1], [1, 4])
    b.check()
    b.compact()
    b.check()
    b.truncate([0, 2])
    b.compact()
    b.check()
    b.truncate([1])
    b.compact()
    b.check()
    assert not b.c.refs.any()


@pytest.mark.parametrize("seed", range(6))
def test_random_calls(seed):
    import random
    rng = random.Random(seed)
    b = Both(layers=rng.choice((1, 3)), n_kv=rng.choice((1, 2)), dim=rng.choice((8, 20, 64)),
             n_pages=rng.choice((60, 3000)), max_seqs=20, max_pages=9, page=rng.choice((8, 16, 32)), seed=seed)
    for _ in range(25):
        held = [s for s in range(20) if b.b.lens[s]]
        empty = [s for s in range(20) if not b.b.lens[s]]
        what = rng.choice(("add", "add", "fork", "truncate", "compact"))
        if what == "add":
            seqs = rng.sample(range(20), rng.randint(1, 8))
            counts = [rng.randint(0, min(2 * b.b.page, 9 * b.b.page - b.b.lens[s])) for s in seqs]
            need = sum(1 + -(-n // b.b.page) for n in counts)
            if need <= b.b.refs.count(0):
                b.add(seqs, counts)
        elif what == "fork" and held and empty:
            children = rng.sample(empty, rng.randint(1, len(empty)))
            b.fork([rng.choice(held) for _ in children], children)
        elif what == "truncate" and held:
            seqs = rng.sample(held, rng.randint(1, len(held)))
            b.truncate(seqs, [rng.randint(0, b.b.lens[s]) for s in seqs])
        elif what == "compact":
            b.compact()
        b.check()


def state(c):
    return c.book.clone(), c.pages.clone()


def same(c, before):
    # (The calls' own words apart: the control block and what lies behind refs.)
    end = 64 + (c.max_seqs * c.max_pages + 3) // 4 * 4 + (c.max_seqs + 3) // 4 * 4 + c.n_pages
    return torch.equal(c.book[64:end], before[0][64:end]) and torch.equal(c.pages.view(torch.int16), before[1].view(torch.int16))


def test_refusals_leave_the_cache():
    b = Both(n_pages=12, max_pages=4)
    b.add([0, 1], [20, 9])
    c = b.c
    for call, why in (
            (lambda: rr.rr_cache_fork(c, ints([0, 1]), ints([2, 2])), "twice"),
            (lambda: rr.rr_cache_fork(c, ints([0]), ints([1])), "holds tokens"),
            (lambda: rr.rr_cache_fork(c, ints([0, 3]), ints([3, 4])), "twice"),
            (lambda: rr.rr_cache_fork(c, ints([0]), ints([12])), "range"),
            (lambda: rr.rr_cache_fork(c, ints([-1]), ints([3])), "range"),
            (lambda: rr.rr_cache_extend(c, ints([0, 0])), "twice"),
            (lambda: rr.rr_cache_extend(c, ints([0, 12])), "range"),
            (lambda: rr.rr_cache_extend(c, ints([0, 1]), starts=ints([0, 2, 1])), "range"),
            (lambda: rr.rr_cache_extend(c, ints([0]), starts=ints([0, 13])), "room"),
            (lambda: rr.rr_cache_extend(c, ints([2, 3, 4]), starts=ints([0, 32, 56, 57])), "room"),
            (lambda: rr.rr_cache_truncate(c, ints([0]), ints([21])), "range"),
            (lambda: rr.rr_cache_truncate(c, ints([0]), ints([-1])), "range"),
            (lambda: rr.rr_cache_truncate(c, ints([1, 1]), ints([1, 1])), "twice")):
        before = state(c)
        call()
        # A marked cache: later calls leave it, too.
        rr.rr_cache_truncate(c, ints([0]))
        rr.rr_cache_compact(c)
        k = torch.ones(1, 2, 32, dtype=torch.bfloat16, device="cuda")
        rr.rr_cache_append(c, 0, k, k, ints([0]))
        with pytest.raises(rr.RRError, match=why):
            rr.rr_cache_check(c)
        assert same(c, before)
        rr.rr_cache_check(c)
    # And goes on as if nothing had been.
    b.add([2, 3], [32, 16])
    b.check()
    assert b.c.refs.tolist().count(0) == 1


def test_append_leaves_out_what_does_not_fit():
    b = Both()
    b.add([0, 1], [10, 4])
    before = state(b.c)
    x = torch.ones(6, 2, 32, dtype=torch.bfloat16, device="cuda")
    rr.rr_cache_append(b.c, 0, x[:1], x[:1], ints([12]))
    with pytest.raises(rr.RRError, match="range"):
        rr.rr_cache_check(b.c)
    rr.rr_cache_append(b.c, 0, x, x, ints([1]), starts=ints([0, 6]))    # six of its last four
    with pytest.raises(rr.RRError, match="range"):
        rr.rr_cache_check(b.c)
    b.c.pages.copy_(before[1])
    # Rows of no sequence: before the first start and behind the last.
    rr.rr_cache_append(b.c, 0, x, x, ints([0, 1]), starts=ints([2, 3, 4]))
    rr.rr_cache_check(b.c)
    b.b.append(0, x[2:4].cpu(), x[2:4].cpu(), [0, 1], [1, 1])
    b.check()


def test_append_strided_rows():
    """Keys and values out of a fused product's rows, aligned and not."""
    for dim, off in ((32, 0), (32, 5), (36, 4), (7, 1)):
        b = Both(dim=dim)
        b.extend([3, 0], [5, 2])
        fused = torch.randn(7, 3 * 2 * dim + 2 * off, generator=b.gen).bfloat16().cuda()
        k, v = fused[:, off:off + 2 * dim], fused[:, off + 2 * dim:off + 4 * dim].view(7, 2, dim)
        rr.rr_cache_append(b.c, 1, k, v, ints([3, 0]), starts=ints([0, 5, 7]))
        b.b.append(1, k.cpu().view(7, 2, dim), v.cpu(), [3, 0], [5, 2])
        b.check()


def test_saved_book_and_graph():
    """A book put back, and a captured run of calls replayed on it."""
    b = Both()
    b.add([0, 1], [13, 8])
    saved = b.c.book.clone()
    parents, children, seqs, drop = ints([0, 0]), ints([2, 3]), ints([0, 1, 2, 3]), ints([0, 1, 1, 0])
    x = torch.randn(4, 2, 32, device="cuda").bfloat16()

    def run():
        b.c.book.copy_(saved)
        rr.rr_cache_fork(b.c, parents, children)
        rr.rr_cache_extend(b.c, seqs)
        rr.rr_cache_append(b.c, 0, x, x, seqs)
        rr.rr_cache_truncate(b.c, seqs, drop)
        rr.rr_cache_compact(b.c)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    b.b.fork([0, 0], [2, 3])
    b.b.extend([0, 1, 2, 3], [1] * 4)
    b.b.append(0, x.cpu(), x.cpu(), [0, 1, 2, 3], [1] * 4)
    b.b.truncate([0, 1, 2, 3], [0, 1, 1, 0])
    b.b.compact()
    for _ in range(3):
        g.replay()
        b.check()


def test_no_sequences():
    b = Both()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rr.rr_cache_fork(b.c, none, none)
    rr.rr_cache_extend(b.c, none)
    rr.rr_cache_truncate(b.c, none)
    k = torch.empty(0, 2, 32, dtype=torch.bfloat16, device="cuda")
    rr.rr_cache_append(b.c, 0, k, k, none)
    rr.rr_cache_compact(b.c)
    b.check()


def test_clear():
    """A used and marked cache is as a new one again."""
    b = Both()
    b.add([0, 4], [20, 7])
    b.fork([0], [1])
    rr.rr_cache_truncate(b.c, ints([0, 0]))          # (twice: marked)
    rr.rr_cache_clear(b.c)
    b.b = R.Book(b.b.pages, 12, 8)
    b.check()
    new = rr.Cache(2, 2, 32, 40, 12, 8, page_tokens=8)
    assert torch.equal(b.c.book[64:], new.book[64:])
    b.add([4, 2], [9, 9])
    b.check()
