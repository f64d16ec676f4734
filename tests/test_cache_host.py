"""The cache, its attention and drafted tokens: sizes and refusals (no GPU), and the tests' own
restatement held against hand-worked numbers."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _cache as R

BF = torch.bfloat16


def cache(**kw):
    a = dict(layers=2, n_kv=2, dim=36, n_pages=10, max_seqs=3, max_pages=4, page_tokens=8, dtype="bf16")
    a.update(kw)
    pitch = (a["dim"] + 7) // 8 * 8
    shape = (a["n_pages"], a["layers"], 2, a["n_kv"], a["page_tokens"], pitch)
    few = all(0 < n < 10 ** 4 for n in shape)
    pages = torch.zeros(shape if few else (1,), dtype=R.TYPES.get(a["dtype"], BF))
    return rr.Cache(pages=pages, **a)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_sizes():
    c = cache()
    assert (c.pitch, c.page_bytes) == (40, 2 * 2 * 2 * 8 * 40 * 2)
    assert c.table.shape == (3, 4) and c.lengths.shape == (3,) and c.refs.shape == (10,)
    assert bool((c.table == -1).all()) and not c.lengths.any() and not c.refs.any()
    # The parts follow one another, each from a multiple of four.
    at = [x.storage_offset() for x in (c.table, c.lengths, c.refs)]
    assert at == [64, 76, 80] and c.book.numel() > 90
    c.refs[0] = 5
    assert int(c.book[80]) == 5


@pytest.mark.parametrize("kw", [dict(layers=0), dict(layers=1025), dict(n_kv=0), dict(dim=0), dict(dim=257),
                                dict(page_tokens=4), dict(page_tokens=12), dict(page_tokens=256), dict(n_pages=0),
                                dict(max_seqs=0), dict(max_seqs=65537), dict(max_pages=0), dict(max_pages=1 << 28)])
def test_shapes_refused(kw):
    with pytest.raises(rr.RRError, match="RR_ELAYOUT"):
        cache(**kw)


def test_bad_tensors_refused():
    c = cache()
    with pytest.raises(ValueError):
        cache(dtype="f32")
    for pages in (torch.zeros(c.pages.shape), c.pages[:9], c.pages.transpose(0, 1), c.pages[..., :36]):
        with pytest.raises(ValueError):
            rr.Cache(2, 2, 36, 10, 3, 4, page_tokens=8, pages=pages)
    one = ints(0)
    for bad in (one.long(), one.view(1, 1), torch.zeros(4, dtype=torch.int32)[::2]):
        for call in (lambda x: rr.rr_cache_extend(c, x, stream=0), lambda x: rr.rr_cache_truncate(c, x, stream=0),
                     lambda x: rr.rr_cache_fork(c, x, one, stream=0)):
            with pytest.raises(ValueError):
                call(bad)
    with pytest.raises(ValueError):
        rr.rr_cache_fork(c, one, ints(1, 2), stream=0)
    with pytest.raises(ValueError):
        rr.rr_cache_extend(c, one, starts=one, stream=0)
    with pytest.raises(ValueError):
        rr.rr_cache_truncate(c, one, ints(1, 2), stream=0)
    k = torch.zeros(1, 2, 36, dtype=BF)
    for a, b in ((k.float(), k), (k, k[:0]), (k[:, :1], k), (torch.zeros(1, 71, dtype=BF), k),
                 (torch.zeros(1, 2, 72, dtype=BF)[:, :, ::2], k), (torch.zeros(1, 36, 2, dtype=BF).transpose(1, 2), k),
                 (k.expand(3, 2, 36), torch.zeros(3, 2, 36, dtype=BF)), (k, k.half())):
        with pytest.raises(ValueError):
            rr.rr_cache_append(c, 0, a, b, ints(*range(a.shape[0])), stream=0)
    for layer in (-1, 2):
        with pytest.raises(rr.RRError, match="layer"):
            rr.rr_cache_append(c, layer, k, k, one, stream=0)
    with pytest.raises(rr.RRError, match="rows"):
        rr.rr_cache_append(c, 0, k, k, ints(0, 1), stream=0)
    with pytest.raises(rr.RRError, match="sequences"):
        rr.rr_cache_extend(c, ints(0, 1, 2, 0), stream=0)


def test_attention_refused():
    c = cache()
    for n_q in (0, 3, 2 * 1025):
        with pytest.raises(rr.RRError, match="heads"):
            rr.AttendWorkspace(c, n_q)
    ws = rr.AttendWorkspace(c, 4)
    q, out, one = torch.zeros(1, 4, 36, dtype=BF), torch.zeros(1, 4, 36, dtype=BF), ints(0)
    for a, b, kw in ((q.half(), out, {}), (q, out.float(), {}), (q[:, :3], out, {}), (q, torch.zeros(2, 4, 36, dtype=BF), {}),
                     (q, out, dict(starts=one)), (q, out, dict(lse=torch.zeros(1, 3))),
                     (q, out, dict(lse=torch.zeros(1, 4, dtype=torch.float64)))):
        with pytest.raises(ValueError):
            rr.rr_attend(c, 0, a, b, one, ws, stream=0, **kw)
    with pytest.raises(rr.RRError, match="layer"):
        rr.rr_attend(c, 2, q, out, one, ws, stream=0)
    with pytest.raises(rr.RRError, match="rows"):
        rr.rr_attend(c, 0, q, out, ints(0, 1), ws, stream=0)
    small = rr.AttendWorkspace(cache(dim=300 // 8), 4)
    small.nbytes -= 1
    with pytest.raises(rr.RRError, match="workspace"):
        rr.rr_attend(c, 0, q, out, one, small, stream=0)


def test_drafts_refused():
    p, d, u, v = torch.zeros(3, 8), ints(0, 0, 0), torch.zeros(3), torch.zeros(1)
    acc, tok, starts = ints(0), ints(0, 0, 0), ints(0, 3)
    good = dict(p=p, drafts=d, u=u, v=v, accepted=acc, tokens=tok, starts=starts)
    for kw in (dict(p=p.half()), dict(p=p[0]), dict(p=p.T), dict(p=torch.zeros(1, 8).expand(3, 8)), dict(q=torch.zeros(3, 7)),
               dict(q=p.double()), dict(drafts=d.long()), dict(drafts=d[:2]), dict(u=u.double()), dict(v=u), dict(tokens=acc),
               dict(starts=d), dict(rejected=d)):
        with pytest.raises(ValueError):
            rr.rr_accept(**dict(good, **kw), stream=0)
    with pytest.raises(rr.RRError, match="rows"):
        rr.rr_accept(p, None, None, v, acc, tok, stream=0)
    with pytest.raises(rr.RRError, match="vocabulary"):
        rr.rr_accept(torch.zeros(1, (1 << 20) + 1), None, None, v, acc, acc.clone(), stream=0)


def test_host_memory_refused():
    """Memory that is not this GPU's is refused before a launch (without a GPU: any)."""
    c = cache()
    for call in (lambda: rr.rr_cache_extend(c, ints(0), stream=0), lambda: rr.rr_cache_compact(c, stream=0)):
        with pytest.raises(rr.RRError):
            call()


def test_restatement_of_pages_by_hand():
    """Pages of 4 tokens: a prompt of 6 tokens, two samples of it, a token each."""
    pages = torch.arange(8.0).view(8, 1, 1, 1, 1, 1).expand(8, 1, 2, 1, 4, 1).clone()
    b = R.Book(pages, 4, 4)
    assert b.extend([0], [6]) and b.held[0] == [0, 1]
    b.fork([0], [2])
    assert b.refs == [2, 2, 0, 0, 0, 0, 0, 0]
    assert b.extend([2], [1]) and b.held == [[0, 1], [], [0, 2], []]      # a copy of page 1
    assert b.pages[2, 0, 0, 0, :, 0].tolist() == [1, 1, 2, 2]             # of its two tokens
    b.fork([0], [1])
    assert b.extend([0, 1], [3, 2])       # 0 takes a copy and a new page, 1 keeps page 1
    assert b.held[0] == [0, 3, 4] and b.held[1] == [0, 1]
    b.truncate([0, 2], [3, 7])
    assert b.held[0] == [0, 3] and b.held[2] == [] and b.refs == [2, 1, 0, 1, 0, 0, 0, 0]
    b.compact()
    assert b.held[0] == [0, 2] and b.table(3)[1] == [0, 1, -1]
    assert not b.extend([0], [100])


def test_restatement_of_attention_by_hand():
    """Scores ln 3 and 0: weights 3/4 and 1/4; the first new token sees the first key only."""
    k = torch.tensor([[[math.log(3.0)]], [[0.0]]], dtype=torch.float64)
    v = torch.tensor([[[4.0]], [[8.0]]], dtype=torch.float64)
    q = torch.ones(2, 1, 1, dtype=torch.float64)
    out, _, lse, _ = R.attend(q, k, v, 2, 1.0, "bf16")
    assert torch.allclose(out.flatten(), torch.tensor([4.0, 5.0], dtype=torch.float64))
    assert torch.allclose(lse.flatten(), torch.tensor([math.log(3.0), math.log(4.0)], dtype=torch.float64))
    out, _, lse, _ = R.attend(torch.cat([q, q]), k, v, 4, 1.0, "bf16")
    assert out.flatten()[:2].tolist() == [0, 0] and lse.flatten()[:2].tolist() == [-math.inf] * 2


def test_restatement_of_acceptance_by_hand():
    assert R.units(torch.tensor([1.0, 2.0 ** -42, 1.5 * 2.0 ** -42, 2.5 * 2.0 ** -42, 2.0 ** -43, math.nan, -1.0, 3.0])) == \
        [1 << 42, 1, 2, 2, 0, 0, 0, 1 << 42]
    p = torch.tensor([[0.5, 0.25, 0.25], [0.0, 0.0, 1.0]])
    q = torch.tensor([[0.25, 0.75, 0.0], [1.0, 0.0, 0.0]])
    assert R.accept(p, q, [1], [0.3], 0.0) == (1, 2)             # 0.3 x 0.75 < 0.25
    # 0.4 x 0.75 is not: the rest is [1/4, 0, 1/4].
    assert R.accept(p, q, [1], [0.4], 0.49) == (0, 0) and R.accept(p, q, [1], [0.4], 0.5) == (0, 2)
    assert R.accept(p, None, [0], [0.5], 0.5) == (0, 2)          # [0, 1/4, 1/4]
    assert R.accept(p, None, [7], [0.0], 0.49) == (0, 0)
