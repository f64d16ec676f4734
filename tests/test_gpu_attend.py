"""Attention over the paged cache on the GPU, against a plain restatement in 64 bits with
derived bounds (tests/_cache.py)."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _cache as R

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Sequences of given lengths whose last counts[i] tokens are new, their pages in random order
    and with NaN wherever no token is."""

    def __init__(self, lengths, counts, n_q=4, n_kv=2, dim=64, page=16, kind="bf16", layers=2, layer=1,
                 seed=0, spread=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.lengths, self.counts, self.kind, self.layer = lengths, counts, kind, layer
        t = R.TYPES[kind]
        need = [-(-n // page) for n in lengths]
        n_pages, max_pages = sum(need) + 3, max(need + [1]) + 1
        self.c = rr.Cache(layers, n_kv, dim, n_pages, len(lengths) + 2, max_pages, page_tokens=page, dtype=kind)
        pages = torch.full(self.c.pages.shape, math.nan, dtype=t)
        order = torch.randperm(n_pages, generator=gen).tolist()
        slots = torch.randperm(len(lengths) + 2, generator=gen).tolist()[:len(lengths)]
        table = torch.full((len(lengths) + 2, max_pages), -1, dtype=torch.int32)
        lens = torch.zeros(len(lengths) + 2, dtype=torch.int32)
        self.k, self.v = [], []
        for i, n in enumerate(lengths):
            k = (spread * torch.randn(n, n_kv, dim, generator=gen)).to(t)
            v = torch.randn(n, n_kv, dim, generator=gen).to(t)
            self.k.append(k)
            self.v.append(v)
            lens[slots[i]] = n
            held = [order.pop() for _ in range(need[i])]
            table[slots[i], :len(held)] = torch.tensor(held, dtype=torch.int32)
            pos = torch.arange(n)
            at = torch.tensor(held, dtype=torch.long)[pos // page] if n else pos
            pages[at, layer, 0, :, pos % page, :dim] = k
            pages[at, layer, 1, :, pos % page, :dim] = v
        self.c.pages.copy_(pages)
        self.c.table.copy_(table)
        self.c.lengths.copy_(lens)
        self.seqs = ints(slots)
        self.rows = sum(counts)
        at = [0]
        for n in counts:
            at.append(at[-1] + n)
        self.at = at
        self.starts = None if counts == [1] * len(counts) else ints(at)
        self.q = torch.randn(self.rows, n_q, dim, generator=gen).to(t)
        self.ws = rr.AttendWorkspace(self.c, n_q)
        self.scale = dim ** -0.5

    def run(self, q=None, scale=None):
        q = self.q.cuda() if q is None else q
        out = torch.full_like(self.q, 7.0, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        rr.rr_attend(self.c, self.layer, q, out, self.seqs, self.ws, starts=self.starts, lse=lse, scale=scale)
        rr.rr_cache_check(self.c)
        return out.cpu(), lse.cpu()

    def check(self, out, lse, scale=None):
        for i, n in enumerate(self.counts):
            a, b = self.at[i], self.at[i + 1]
            o, ot, e, et = R.attend(self.q[a:b], self.k[i], self.v[i], n, self.scale if scale is None else scale, self.kind)
            far = (out[a:b].double() - o).abs()
            assert bool((far <= ot).all()), (i, float((far / ot.clamp_min(1e-30)).max()))
            none = e == -math.inf
            assert torch.equal(lse[a:b].double() == -math.inf, none)
            far = (lse[a:b].double() - e)[~none].abs()
            assert bool((far <= et[~none]).all()), (i, float((far / et[~none]).max()))


@pytest.mark.parametrize("dim", [1, 8, 32, 36, 64, 65, 80, 96, 128, 130, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_head_sizes(dim, kind):
    c = Case([1, 33, 200, 17], [1, 1, 1, 1], dim=dim, kind=kind, seed=dim)
    c.check(*c.run())


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
def test_page_sizes_and_lengths(page):
    c = Case([0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500], [1] * 16, page=page, dim=32)
    c.check(*c.run())


@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (3, 1), (8, 1), (9, 3), (16, 2), (32, 4), (40, 1), (48, 1), (5, 5), (100, 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_heads(n_q, n_kv, dim):
    c = Case([40, 75], [1, 1], n_q=n_q, n_kv=n_kv, dim=dim, seed=n_q)
    c.check(*c.run())


@pytest.mark.parametrize("dim", [1, 36, 80, 96, 130, 192])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,count", [(24, 1), (10, 3), (33, 2)])
def test_many_rows_of_odd_heads(dim, kind, n_q, count):
    """Tiles of more than 16 rows, full and not, of heads that are not whole 64s of elements."""
    c = Case([300, 17, 2, 129], [count] * 4, n_q=n_q, n_kv=1, dim=dim, kind=kind, page=8, seed=dim)
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,dim", [(8, 128), (2, 64), (6, 200)])
def test_many_short_tiles(kind, n_q, dim):
    """Runs that hold many tiles whole, beside one that is cut many times."""
    gen = torch.Generator().manual_seed(n_q)
    lengths = torch.randint(1, 400, (150,), generator=gen).tolist() + [7000]
    counts = torch.randint(1, 6, (151,), generator=gen).tolist()
    c = Case(lengths, counts, n_q=n_q, n_kv=1, dim=dim, kind=kind, page=32, seed=1)
    first = c.run()
    c.check(*first)
    again = c.run()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,n_kv,dim", [(8, 1, 128), (4, 2, 36), (14, 2, 80), (16, 1, 256)])
def test_drafted_tokens(kind, n_q, n_kv, dim):
    """Several new tokens, ragged; more than a sequence has (rows that see nothing); none."""
    c = Case([70, 5, 3, 0, 129, 64, 33], [5, 5, 6, 2, 8, 0, 1], n_q=n_q, n_kv=n_kv, dim=dim, kind=kind)
    out, lse = c.run()
    c.check(out, lse)
    assert torch.equal(out[c.at[2]:c.at[2] + 3], torch.zeros_like(out[:3]))


@pytest.mark.parametrize("n", [1, 40, 300])
def test_many_new_tokens(n):
    """A prompt's tokens at once."""
    c = Case([n, n + 100], [n, n], n_q=4, n_kv=2, dim=64, seed=n)
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_split_over_blocks(kind):
    """Long sequences, cut within and between blocks, beside short ones."""
    c = Case([9000, 1, 3001, 40, 20000, 0, 65], [1] * 7, n_q=4, n_kv=1, dim=128, kind=kind, seed=3)
    first = c.run()
    c.check(*first)
    again = c.run()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_a_million_tokens(kind):
    """One sequence of 2^20 tokens, whose values have a mean: long sums do not drift.

    8192 units over 152 blocks or fewer: a sum goes through at most 64 additions that cut off at
    2^-23 (8 units, 8 products each), then 54 / 8 of a block's and 152 of the joined pieces, which
    round; the weights' own through 54 + 9 + 152.  Less than 2^-15 of A in all (GPUs of fewer
    SMs: twice that many units a block for half the pieces)."""
    n, dim = 1 << 20, 64
    gen = torch.Generator("cuda").manual_seed(3)
    t = R.TYPES[kind]
    c = rr.Cache(1, 1, dim, n // 64, 1, n // 64, page_tokens=64, dtype=kind)
    c.pages.normal_(0, 1, generator=gen)
    c.pages[:, 0, 1] = (c.pages[:, 0, 1].float().abs() * 0.5 + 0.5).to(t)
    c.table[0] = torch.randperm(n // 64, device="cuda", generator=gen).int()
    c.lengths.fill_(n)
    q = (0.5 * torch.randn(1, 2, dim, device="cuda", generator=gen)).to(t)
    out, lse = torch.empty_like(q), torch.empty(1, 2, device="cuda")
    rr.rr_attend(c, 0, q, out, ints([0]), rr.AttendWorkspace(c, 2), lse=lse)
    rr.rr_cache_check(c)
    order = c.table[0].long()
    k, v = (c.pages[order, 0, x, 0].flatten(0, 1).double() for x in (0, 1))
    for h in range(2):
        s = dim ** -0.5 * (k @ q[0, h].double())
        size = dim ** -0.5 * (k.abs() @ q[0, h].double().abs())
        e = float((size * (dim / 8 + 64) * 2.0 ** -23 + 4 * s.abs() * 2.0 ** -24).max())
        w = torch.softmax(s, 0)
        want, a = w @ v, w @ v.abs()
        tol = a * (2 * math.expm1(e) + 2.0 ** -20 + R.CUT[kind] + 2.0 ** -15) * (1 + R.ROUND[kind]) + R.ROUND[kind] * want.abs()
        assert bool(((out[0, h].double() - want).abs() <= tol).all())
        assert abs(float(lse[0, h]) - float(torch.logsumexp(s, 0))) <= e + 2.0 ** -15 + 2.0 ** -22 * 20


def test_first_calls_captured():
    """A process whose first calls are captured ones."""
    import os
    import subprocess
    import sys
    code = """
import torch
import paper_2512_22492_gb300 as rr
ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
c = rr.Cache(1, 2, 64, 8, 4, 4, page_tokens=8)
ws = rr.AttendWorkspace(c, 4)
seqs, drop = ints(0, 2), ints(1, 0)
q = torch.randn(2, 4, 64, device="cuda").bfloat16()
k = torch.randn(2, 2, 64, device="cuda").bfloat16()
out = torch.empty_like(q)
p = torch.full((2, 50), 0.02, device="cuda")
v, acc, tok = torch.tensor([0.0, 0.5], device="cuda"), ints(0, 0), ints(0, 0)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    rr.rr_cache_extend(c, seqs)
    rr.rr_cache_append(c, 0, k, k, seqs)
    rr.rr_attend(c, 0, q, out, seqs, ws)
    rr.rr_accept(p, None, None, v, acc, tok)
    rr.rr_cache_truncate(c, seqs, drop)
    rr.rr_cache_compact(c)
g.replay()
rr.rr_cache_check(c)
assert c.lengths.tolist() == [0, 0, 1, 0], c.lengths.tolist()
assert torch.equal(out, k.repeat_interleave(2, 1)) and tok.tolist() == [0, 25]
g.replay()
rr.rr_cache_check(c)
assert c.lengths.tolist() == [0, 0, 2, 0]
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]


def test_many_sequences():
    """More of them than a block has threads, and than a warp looks at at once."""
    gen = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 60, (700,), generator=gen).tolist()
    c = Case(lengths, [1] * 700, n_q=2, n_kv=1, dim=32, page=8)
    c.check(*c.run())
    counts = torch.randint(0, 4, (700,), generator=gen).tolist()
    c = Case(lengths, counts, n_q=2, n_kv=1, dim=32, page=8)
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_sharp_scores(kind):
    """Scores far apart, growing along the keys, so that the reference keeps moving; and a
    scale of either sign."""
    c = Case([2000, 300], [1, 3], n_q=4, n_kv=2, dim=64, kind=kind, spread=4.0)
    for i in range(2):
        c.k[i] = (c.k[i].float() * torch.linspace(0.01, 1, len(c.k[i]))[:, None, None]).to(R.TYPES[kind])
    put(c)
    for scale in (None, 0.5, -0.3, 0.0):
        c.check(*c.run(scale=scale), scale=scale)


def put(c):
    """Writes c.k and c.v where the table says."""
    page = c.c.page_tokens
    for i, s in enumerate(c.seqs.tolist()):
        pos = torch.arange(c.lengths[i], device="cuda")
        at = c.c.table[s].long()[pos // page]
        c.c.pages[at, c.layer, 0, :, pos % page, :c.c.dim] = c.k[i].cuda()
        c.c.pages[at, c.layer, 1, :, pos % page, :c.c.dim] = c.v[i].cuda()


def test_tiny_weights_of_float16():
    """Many keys of little weight beside one of much: their values still count."""
    c = Case([5000], [1], n_q=1, n_kv=1, dim=64, kind="f16")
    c.q = torch.zeros(1, 1, 64).half()
    c.q[0, 0, 0] = 8.0
    k = torch.zeros(5000, 1, 64).half()
    k[77, 0, 0] = 18.0            # exp(18 - 0): the others have 2^-26 of its weight each
    v = torch.full((5000, 1, 64), 1.0).half()
    v[77] = 0.0
    c.k, c.v = [k], [v]
    put(c)
    out, lse = c.run()
    c.check(out, lse)
    assert float(out.min()) > 0


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(kind, what):
    """They reach the rows that see them, as the formula says, and no others: not those
    whose new token is an earlier one, not other heads, elements or sequences."""
    c = Case([100, 70, 3000], [4, 1, 2], n_q=4, n_kv=2, dim=64, kind=kind)
    clean = c.run()
    v = [x.clone() for x in c.v]
    c.v[0][97, 0, 5] = what            # seen by new tokens 1..3
    c.v[0][99, 1, :] = what            # by the last one only
    c.v[2][2998, 1, 9] = what          # (both new tokens of the long one)
    put(c)
    out, lse = c.run()
    # (check() holds lse to its bounds: the reference of its sums may be another here.)
    touched = torch.zeros(out.shape, dtype=torch.bool)
    touched[1:4, :2, 5] = True
    touched[3, 2:] = True
    touched[5:7, 2:, 9] = True
    same = lambda a: bool((a.isnan() if math.isnan(what) else a == what).all())
    assert same(out[touched].float())
    c.v = v
    out[touched] = clean[0][touched]
    c.check(out, lse)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_keys_that_are_not_finite(kind):
    """A NaN key makes the rows that see it NaN; keys of -infinity scores have no weight."""
    c = Case([90, 40], [3, 1], n_q=2, n_kv=1, dim=64, kind=kind)
    clean = c.run()
    c.k[0][88, 0, 3] = math.nan
    put(c)
    out, lse = c.run()
    assert torch.equal(out[0], clean[0][0]) and torch.equal(lse[3], clean[1][3])
    assert bool(out[1:3].isnan().all()) and bool(lse[1:3].isnan().all())
    c.k[0][88, 0, 3] = -math.inf
    c.q = c.q.abs()
    put(c)
    out, lse = c.run()
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    c.k[0][:, 0, 3] = -math.inf
    put(c)
    out, lse = c.run()
    assert not out[:3].any() and bool((lse[:3] == -math.inf).all())


def test_largest_values():
    """Sums of the largest bfloat16 values pass float32 before they are normalised."""
    c = Case([600, 31], [2, 1], n_q=2, n_kv=1, dim=64)
    big = torch.finfo(torch.bfloat16).max
    c.v = [torch.where(x > 0, big, -big).to(torch.bfloat16) for x in c.v]
    c.v[0][:, 0, 0] = big
    put(c)
    out, lse = c.run()
    assert bool((out[:2, :, 0] == big).all())
    c.check(out, lse)


def test_strides_and_alignment():
    """Queries out of a fused product's rows, results to wider ones; the bits stay."""
    for dim in (64, 36):
        c = Case([100, 7, 260], [2, 1, 4], dim=dim)
        want, _ = c.run()
        for off in (0, 1, 4, 8):
            q = torch.zeros(c.rows, 4 * dim + 24, dtype=torch.bfloat16, device="cuda")
            o = torch.full_like(q, 9.0)
            q[:, off:off + 4 * dim] = c.q.flatten(1).cuda()
            rr.rr_attend(c.c, c.layer, q[:, off:off + 4 * dim], o[:, off:off + 4 * dim], c.seqs, c.ws, starts=c.starts)
            assert torch.equal(o[:, off:off + 4 * dim].cpu(), want.flatten(1))
            o[:, off:off + 4 * dim] = 9.0
            assert bool((o == 9.0).all())


def test_rows_of_no_sequence_stay():
    c = Case([50, 60], [2, 3], dim=64)
    want = c.run()
    q = torch.cat([c.q[:1], c.q, c.q[:4]]).cuda()
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    rr.rr_attend(c.c, c.layer, q, out, c.seqs, c.ws, starts=c.starts + 1, lse=lse)
    assert torch.equal(out[1:6].cpu(), want[0]) and torch.equal(lse[1:6].cpu(), want[1])
    assert bool((out[0] == 9).all()) and bool((out[6:] == 9).all()) and bool((lse[6:] == 9).all())
    # An empty pass, and the same sequence twice: each listing is one of its own.
    rr.rr_attend(c.c, c.layer, q[:0], out[:0], c.seqs[:0], c.ws)
    seqs, starts = c.seqs[[0, 0]], ints([0, 2, 4])
    q = torch.cat([c.q[:2], c.q[:2]]).cuda()
    rr.rr_attend(c.c, c.layer, q, out[:4], seqs, c.ws, starts=starts)
    assert torch.equal(out[:2], out[2:4])


def test_lists_out_of_range_are_left_out_and_marked():
    c = Case([50, 60, 20], [1, 1, 1], dim=64)
    want, _ = c.run()
    q = c.q.cuda()
    for seqs, starts, stay in (([5, None, None], None, [0]), ([None, -1, None], None, [1]),
                               ([None] * 3, [0, 1, 0, 1], [1, 2]), ([None] * 3, [0, 4, 4, 4], [0, 1, 2]),
                               ([None] * 3, [0, 1, 2, 4], [2])):
        s = [a if b is None else b for a, b in zip(c.seqs.tolist(), seqs)]
        out = torch.full_like(q, 9.0)
        rr.rr_attend(c.c, c.layer, q, out, ints(s), c.ws, starts=None if starts is None else ints(starts))
        with pytest.raises(rr.RRError, match="range"):
            rr.rr_cache_check(c.c)
        for r in stay:
            assert bool((out[r] == 9.0).all())
    # A page number out of range: marked, and nothing is read there.
    table = c.c.table.clone()
    c.c.table[int(c.seqs[1]), 1] = c.c.n_pages
    rr.rr_attend(c.c, c.layer, q, torch.empty_like(q), c.seqs, c.ws)
    with pytest.raises(rr.RRError, match="table"):
        rr.rr_cache_check(c.c)
    c.c.table.copy_(table)
    out, _ = c.run()
    assert torch.equal(out, want)


def test_graphs_and_streams():
    """A captured call, replayed after the cache has grown; two streams, a workspace each."""
    c = Case([300, 41], [1, 1], n_q=8, n_kv=2, dim=128)
    q, out = c.q.cuda(), torch.empty_like(c.q, device="cuda")
    rr.rr_attend(c.c, c.layer, q, out, c.seqs, c.ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rr.rr_attend(c.c, c.layer, q, out, c.seqs, c.ws)
    out.zero_()
    g.replay()
    full, _ = c.run()
    assert torch.equal(out.cpu(), full)
    c.c.lengths.clamp_(max=30)
    g.replay()
    short, _ = c.run()
    assert torch.equal(out.cpu(), short) and not torch.equal(short, full)
    big = Case([5000, 900], [1, 1], n_q=8, n_kv=2, dim=128, seed=9)
    want, _ = big.run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [rr.AttendWorkspace(big.c, 8) for _ in range(2)]
    outs = [torch.empty_like(big.q, device="cuda") for _ in range(2)]
    bq = big.q.cuda()
    torch.cuda.synchronize()
    for _ in range(20):
        for s, w, o in zip(streams, spaces, outs):
            with torch.cuda.stream(s):
                rr.rr_attend(big.c, big.layer, bq, o, big.seqs, w)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.cpu(), want)


def test_far_pages():
    """Pages past 2^31 elements of the pool."""
    page, dim, layers = 128, 256, 32
    c = rr.Cache(layers, 4, dim, 300, 2, 2, page_tokens=page)
    assert c.pages[-1].storage_offset() > 2 ** 31
    k = torch.randn(2, 4, dim, device="cuda").bfloat16()
    v = torch.randn(2, 4, dim, device="cuda").bfloat16()
    c.refs[:298] = 1              # only the last pages are free
    seqs = ints([1])
    rr.rr_cache_extend(c, seqs, starts=ints([0, 2]))
    rr.rr_cache_append(c, layers - 1, k, v, seqs, starts=ints([0, 2]))
    rr.rr_cache_check(c)
    assert c.table[1].tolist() == [298, -1]
    assert torch.equal(c.pages[298, layers - 1, 0, :, :2], k.transpose(0, 1))
    q = torch.randn(1, 4, dim, device="cuda").bfloat16()
    out = torch.empty_like(q)
    rr.rr_attend(c, layers - 1, q, out, seqs, rr.AttendWorkspace(c, 4))
    o, tol, _, _ = R.attend(q.cpu(), k.cpu(), v.cpu(), 1, dim ** -0.5, "bf16")
    assert bool(((out.cpu().double() - o).abs() <= tol).all())


def test_a_step_of_drafted_tokens():
    """fork, extend, append, attend, accept, truncate in a row, as a rollout runs them, for one
    prompt's samples."""
    gen = torch.Generator().manual_seed(4)
    n_q, n_kv, dim, page = 4, 2, 32, 8
    cache = rr.Cache(1, n_kv, dim, 30, 6, 6, page_tokens=page)
    ws = rr.AttendWorkspace(cache, n_q)
    new = lambda n, h: torch.randn(n, h, dim, generator=gen).bfloat16()
    k, v = [new(11, n_kv)] * 3, [new(11, n_kv)] * 3
    rr.rr_cache_extend(cache, ints([0]), starts=ints([0, 11]))
    rr.rr_cache_append(cache, 0, k[0].cuda(), v[0].cuda(), ints([0]), starts=ints([0, 11]))
    rr.rr_cache_fork(cache, ints([0, 0]), ints([3, 5]))
    seqs, drafted = ints([0, 3, 5]), [3, 2, 3]
    for step in range(4):
        starts = [0]
        for n in drafted:
            starts.append(starts[-1] + n)
        rows = starts[-1]
        at = ints(starts)
        rr.rr_cache_extend(cache, seqs, starts=at)
        kk, vv, q = new(rows, n_kv), new(rows, n_kv), new(rows, n_q)
        rr.rr_cache_append(cache, 0, kk.cuda(), vv.cuda(), seqs, starts=at)
        out = torch.empty(rows, n_q, dim, dtype=torch.bfloat16, device="cuda")
        rr.rr_attend(cache, 0, q.cuda(), out, seqs, ws, starts=at)
        p = torch.softmax(out.float().flatten(1)[:, :100], 1).contiguous()
        drafts = torch.randint(0, 100, (rows,), generator=gen).int().cuda()
        u, vs = torch.rand(rows, generator=gen).cuda() / 50, torch.rand(3, generator=gen).cuda()
        acc, rej = ints([0] * 3), ints([0] * 3)
        tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        rr.rr_accept(p, drafts, u, vs, acc, tokens, starts=at, rejected=rej)
        rr.rr_cache_truncate(cache, seqs, rej)
        rr.rr_cache_check(cache)
        for i in range(3):
            a, b = starts[i], starts[i + 1]
            k[i], v[i] = torch.cat([k[i], kk[a:b]]), torch.cat([v[i], vv[a:b]])
            o, tol, _, _ = R.attend(q[a:b], k[i], v[i], b - a, dim ** -0.5, "bf16")
            assert bool(((out[a:b].cpu().double() - o).abs() <= tol).all())
            n = len(k[i]) - int(rej[i])
            k[i], v[i] = k[i][:n], v[i][:n]
            assert int(cache.lengths[seqs[i]]) == n and int(acc[i]) + int(rej[i]) == b - a - 1
    held = [int(-(-int(cache.lengths[s]) // page)) for s in (0, 3, 5)]
    # The prompt's first page stays shared by all three.
    assert int(cache.refs.max()) == 3 and int((cache.refs > 0).sum()) == sum(held) - 2
