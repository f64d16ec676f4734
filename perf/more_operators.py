"""A rollout's sequences between one token step and the next, as timed cases.

Kinds of pass (``op``):
  attend   attention of every sequence's newest tokens (one, or a few drafted ones)
           over a paged key-value cache (``rr_attend``)
  fork     samples of one prompt: children share their parent's pages
           (``rr_cache_fork``), every sequence gets new tokens, which takes pages and
           copies the ones that are shared and partly filled (``rr_cache_extend``),
           one layer's keys and values are written (``rr_cache_append``), and some
           tokens are taken back (``rr_cache_truncate``)
  compact  finished sequences leave (``rr_cache_truncate``) and the pages still in use
           move to the front of the pool (``rr_cache_compact``)
  accept   drafted tokens held against the target's probabilities, and the token that
           follows them, from given random numbers (``rr_accept``)

``run`` computes them in elementary torch operations, or, where ``own`` is true, with
the library's kernels.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
GIB = 1 << 30


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _attend(n_q, n_kv, dim, seqs, lo, hi, new=1, ragged=False, page=16, layers=1, dtype="bf16",
            name=None):
    """lo..hi: the sequences' lengths, the new tokens among them; ragged: 1..new new
    tokens a sequence, else `new` each."""
    c = dict(op="attend", n_q=n_q, n_kv=n_kv, dim=dim, seqs=seqs, lo=lo, hi=hi, new=new,
             ragged=ragged, page=page, layers=layers, dtype=dtype)
    return dict(c, name=name) if name else c


def _fork(layers, n_kv, dim, parents, children, lo, hi, new=1, page=16, dtype="bf16", name=None):
    """`children` of each of `parents` prompts of lo..hi tokens."""
    c = dict(op="fork", layers=layers, n_kv=n_kv, dim=dim, parents=parents, children=children,
             lo=lo, hi=hi, new=new, page=page, dtype=dtype)
    return dict(c, name=name) if name else c


def _compact(layers, n_kv, dim, seqs, lo, hi, leave, spare, page=16, dtype="bf16", name=None):
    """`leave` of `seqs` sequences of lo..hi tokens leave; `spare` pages were free before."""
    c = dict(op="compact", layers=layers, n_kv=n_kv, dim=dim, seqs=seqs, lo=lo, hi=hi,
             leave=leave, spare=spare, page=page, dtype=dtype)
    return dict(c, name=name) if name else c


def _accept(seqs, drafts, vocab, ragged=False, sure=False, name=None):
    """sure: the drafts come without probabilities of their own (looked up in the text)."""
    c = dict(op="accept", seqs=seqs, drafts=drafts, vocab=vocab, ragged=ragged, sure=sure)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The small MoE test model's first tokens: a call's latency.
        _attend(4, 2, 32, 3, 1, 20, name="attend_tiny"),
        # The odd test model: a head size that no vector width divides, drafted tokens.
        _attend(2, 1, 36, 7, 3, 700, new=3, ragged=True, page=8, layers=2, dtype="f16",
                name="attend_odd_f16"),
        # One long trajectory in Qwen3-8B: the cache has to be split over its length.
        _attend(32, 8, 128, 1, 40001, 40001, layers=2, name="attend_8b_1_long"),
        # A rollout's batch in Qwen3-30B-A3B, short and long trajectories side by side.
        _attend(32, 4, 128, 64, 200, 16000, layers=2, name="attend_30b_64"),
        # Qwen3-32B with four drafted tokens a sequence, to be verified at once.
        _attend(64, 8, 128, 96, 500, 7500, new=5, dtype="f16", name="attend_32b_96_drafts_f16"),
        # Two prompts of the small MoE test model, four samples of each.
        _fork(2, 2, 32, 2, 3, 5, 90, name="fork_tiny"),
        # Eight samples of each of six prompts in Qwen3-8B, all of its layers.
        _fork(36, 8, 128, 6, 7, 150, 405, new=2, name="fork_8b"),
        # A few short sequences of the odd test model.
        _compact(2, 1, 36, 9, 1, 60, 4, 3, page=8, dtype="f16", name="compact_odd_f16"),
        # Qwen3-30B-A3B: half the trajectories have ended.
        _compact(48, 4, 128, 16, 60, 700, 8, 30, name="compact_30b"),
        # The test model's vocabulary, two sequences.
        _accept(2, 3, 512, name="accept_tiny"),
        # One trajectory, its drafts looked up in its own text.
        _accept(1, 7, 151936, sure=True, name="accept_1_lookup"),
        # A batch with a draft model: the rollout that still holds the weights of before
        # the sync, for instance.
        _accept(64, 4, 151936, ragged=True, name="accept_64"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("attend", "attend", "attend", "fork", "compact", "accept"))
    dtype = rng.choice(("bf16", "f16"))
    dim = rng.choice((32, 36, 64, 80, 96, 128, 128, 128, 192, 256))
    page = rng.choice((8, 16, 16, 32, 64))
    n_kv = rng.choice((1, 2, 4, 8))
    while True:
        if op == "accept":
            c = _accept(_log(rng, 1, 128), rng.randint(0, 8), _log(rng, 300, 160000),
                        rng.random() < 0.5, rng.random() < 0.3)
            if (c["drafts"] + 1) * c["seqs"] * c["vocab"] <= 64 * 5 * 151936:
                return c
            continue
        if op == "attend":
            new = rng.choice((1, 1, 1, 2, 3, 5, 8))
            lo = _log(rng, new, 4000)
            c = _attend(n_kv * rng.choice((1, 2, 4, 5, 7, 8, 8, 16)), n_kv, dim,
                        _log(rng, 1, 256), lo, _log(rng, lo, 50000), new, rng.random() < 0.5, page,
                        rng.choice((1, 2, 3)), dtype)
            # No more keys and values, nor products with them, than the largest listed case.
            kv = c["seqs"] * (c["lo"] + c["hi"]) // 2 * n_kv * dim
            rows = c["n_q"] // n_kv * new
            if kv * max(1, rows / 40) <= 96 * 4000 * 8 * 128 and c["layers"] * kv * 4 <= 6 * GIB:
                return c
            continue
        layers = _log(rng, 1, 48)
        lo = _log(rng, 1, 600)
        if op == "fork":
            c = _fork(layers, n_kv, dim, _log(rng, 1, 16), rng.randint(1, 15), lo,
                      _log(rng, lo, 2000), rng.randint(1, 5), page, dtype)
        else:
            seqs = _log(rng, 2, 64)
            c = _compact(layers, n_kv, dim, seqs, lo, _log(rng, lo, 2000), rng.randint(1, seqs - 1),
                         rng.randint(0, 100), page, dtype)
        if _n_pages(c) * _page_elements(c) * 2 <= 0.75 * GIB:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _counts(c):
    """New tokens of each sequence, before they are shuffled with the lengths."""
    if c["op"] == "accept":
        top = c["drafts"] + 1
    else:
        top = c["new"]
    if not c["ragged"]:
        return [top] * c["seqs"]
    return [max(1, top - i % top) for i in range(c["seqs"])]


def _lengths(c):
    """Lengths of each sequence, the new ones included."""
    return [max(a, b) for a, b in zip(_spread(c["lo"], c["hi"], c["seqs"]), _counts(c))]


def _pitch(c):
    """Elements from one token's row of a page to the next: whole 16-byte words."""
    return -(-c["dim"] // 8) * 8


def _page_elements(c):
    return c["layers"] * 2 * c["n_kv"] * c["page"] * _pitch(c)


def _n_pages(c):
    if c["op"] == "fork":
        held = sum(-(-n // c["page"]) for n in _spread(c["lo"], c["hi"], c["parents"]))
        all_ = c["parents"] * (1 + c["children"])
        return held + all_ * (1 + -(-c["new"] // c["page"])) + 5
    held = sum(-(-n // c["page"]) for n in
               (_lengths(c) if c["op"] == "attend" else _spread(c["lo"], c["hi"], c["seqs"])))
    return held + (c["spare"] if c["op"] == "compact" else 2)


def work(case):
    c = case
    if c["op"] == "accept":
        # Of each sequence the probabilities of one position, and the draft's where a draft
        # was refused; about half of the sequences' are, for the drafts that prepare makes.
        each = 4 * c["vocab"] * (1 if c["sure"] or not c["drafts"] else 1.5)
        rows = sum(_counts(c))
        return {"bytes": c["seqs"] * (each + 16) + 20 * rows,
                "flops": 4 * c["seqs"] * c["vocab"]}
    if c["op"] == "attend":
        rows = sum(_counts(c))
        seen = sum(n * (2 * length - n + 1) / 2 for n, length in zip(_counts(c), _lengths(c)))
        kv = sum(_lengths(c)) * c["n_kv"] * c["dim"] * 4
        pages = sum(-(-n // c["page"]) for n in _lengths(c))
        return {"bytes": kv + 4 * pages + rows * c["n_q"] * (4 * c["dim"] + 4),
                "flops": 4 * seen * c["n_q"] * c["dim"]}
    token = c["layers"] * 2 * c["n_kv"] * c["dim"] * 2
    if c["op"] == "fork":
        lengths = _spread(c["lo"], c["hi"], c["parents"])
        n = c["parents"] * (1 + c["children"])
        copied = sum(c["children"] * (length % c["page"]) for length in lengths)
        entries = sum(c["children"] * -(-length // c["page"]) for length in lengths)
        rows = n * c["new"] * 2 * c["n_kv"] * c["dim"] * 2
        return {"bytes": 2 * copied * token + 2 * rows + 16 * entries + 8 * _n_pages(c) + 24 * n,
                "flops": 0}
    pages = [-(-n // c["page"]) for n in _spread(c["lo"], c["hi"], c["seqs"])]
    stay = sum(pages[c["leave"]:])
    # Pages lie at random, so a page in use lies behind the front part with this share.
    moved = stay * (1 - stay / _n_pages(c))
    return {"bytes": 2 * moved * c["page"] * token + 8 * sum(pages) + 12 * _n_pages(c), "flops": 0}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _held(lengths, page, n_pages, max_seqs, max_pages, gen):
    """Table, lengths and holders of sequences whose pages lie at random in the pool."""
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(lengths):
        k = -(-n // page)
        table[i, :k] = order[at:at + k]
        at += k
    refs[order[:at].long()] = 1
    lens = _ints(lengths + [0] * (max_seqs - len(lengths)))
    return table, lens, refs


def _shuffled(values, gen):
    order = torch.randperm(len(values), device="cuda", generator=gen).tolist()
    return [values[i] for i in order], order


def _inputs(c, seed):
    """A case's tensors, from the seed alone."""
    gen = torch.Generator("cuda").manual_seed(seed)
    d = SimpleNamespace()
    case = vars(c)

    def normal(*shape, scale=1.0):
        x = torch.empty(*shape, dtype=TYPES[c.dtype], device="cuda")
        return x.normal_(0.0, scale, generator=gen)

    if c.op == "accept":
        d.counts, _ = _shuffled(_counts(case), gen)
        d.starts = _ints(_starts(d.counts))
        rows = sum(d.counts)
        # Logits of a text model: a few likely tokens, a long flat tail.
        a = 3 * torch.randn(rows, c.vocab, device="cuda", generator=gen)
        e = torch.exp(a - a.amax(1, keepdim=True))
        d.p = e / e.sum(1, keepdim=True)
        # The draft's: the same, somewhat off; its tokens are drawn from it.
        a += 0.7 * torch.randn(rows, c.vocab, device="cuda", generator=gen)
        e = torch.exp(a - a.amax(1, keepdim=True))
        q = e / e.sum(1, keepdim=True)
        noise = torch.rand(rows, c.vocab, device="cuda", generator=gen)
        d.drafts = (q / -torch.log(noise.clamp(1e-30, 1 - 1e-7))).argmax(1).to(torch.int32)
        d.q = None if c.sure else q
        d.u = torch.rand(rows, device="cuda", generator=gen)
        d.v = torch.rand(c.seqs, device="cuda", generator=gen)
        return d
    n_pages = _n_pages(case)
    if c.op == "attend":
        lengths, order = _shuffled(_lengths(case), gen)
        counts = _counts(case)
        d.counts = [counts[i] for i in order]
        d.lengths, max_seqs = lengths, c.seqs
        max_pages = -(-max(lengths) // c.page)
        d.seqs = _ints(list(range(c.seqs)))
        d.starts = _ints(_starts(d.counts))
        rows = sum(d.counts)
        d.layer = c.layers - 1
        # Normalised queries and keys; some heads attend sharply.
        d.q = normal(rows, c.n_q, c.dim)
        d.q *= torch.linspace(0.5, 4, c.n_q, device="cuda").to(d.q.dtype)[:, None]
    elif c.op == "fork":
        lengths, _ = _shuffled(_spread(c.lo, c.hi, c.parents), gen)
        n = c.parents * (1 + c.children)
        max_seqs = n + 1
        max_pages = -(-(c.hi + c.new) // c.page)
        d.parents = _ints([i for i in range(c.parents) for _ in range(c.children)])
        d.children = _ints(list(range(c.parents, n)))
        d.seqs = _ints(list(range(n)))
        d.n, d.starts = n, _ints([c.new * i for i in range(n + 1)])
        d.layer = c.layers - 1
        d.k, d.v = normal(n * c.new, c.n_kv, c.dim), normal(n * c.new, c.n_kv, c.dim)
        # Every other sequence takes its last new token back.
        d.back, d.drop = d.seqs[::2].contiguous(), _ints([1] * len(range(0, n, 2)))
    else:
        spread = _spread(c.lo, c.hi, c.seqs)
        _, order = _shuffled(spread, gen)
        lengths = [spread[i] for i in order]
        max_seqs, max_pages = c.seqs, -(-c.hi // c.page)
        # The shortest leave, wherever they stand.
        d.gone = _ints([s for s in range(c.seqs) if order[s] < c.leave])
        d.drop = _ints([lengths[s] for s in range(c.seqs) if order[s] < c.leave])
    d.max_seqs, d.max_pages, d.n_pages = max_seqs, max_pages, n_pages
    d.table, d.lens, d.refs = _held(lengths, c.page, n_pages, max_seqs, max_pages, gen)
    d.pages = normal(n_pages, c.layers, 2, c.n_kv, c.page, _pitch(case))
    d.pages[..., c.dim:] = 0
    return d


def prepare(case, seed):
    c = SimpleNamespace(**case)
    s = _inputs(c, seed)
    s.c = c
    if not own:
        return s
    import paper_2512_22492_gb300 as rr
    s.rr = rr
    if c.op == "accept":
        rows = sum(s.counts)
        s.accepted, s.rejected = (torch.empty(c.seqs, dtype=torch.int32, device="cuda")
                                  for _ in range(2))
        s.tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        return s
    s.cache = rr.Cache(c.layers, c.n_kv, c.dim, s.n_pages, s.max_seqs, s.max_pages,
                       page_tokens=c.page, dtype=c.dtype, pages=s.pages)
    s.cache.table.copy_(s.table)
    s.cache.lengths.copy_(s.lens)
    s.cache.refs.copy_(s.refs)
    if c.op == "attend":
        s.workspace = rr.AttendWorkspace(s.cache, c.n_q)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(s.q.shape[:2], dtype=torch.float32, device="cuda")
        if c.new == 1:
            s.starts = None
    else:
        # What a pass begins with, as a program keeps it that may have to go back.
        s.saved = s.cache.book.clone()
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _run_own(s):
    c, rr = s.c, s.rr
    if c.op == "accept":
        rr.rr_accept(s.p, s.drafts, s.u, s.v, s.accepted, s.tokens, q=s.q, starts=s.starts,
                     rejected=s.rejected)
        return {"accepted": s.accepted, "tokens": s.tokens, "rejected": s.rejected}
    if c.op == "attend":
        rr.rr_attend(s.cache, s.layer, s.q, s.out, s.seqs, s.workspace, starts=s.starts, lse=s.lse)
        return {"out": s.out, "lse": s.lse}
    s.cache.book.copy_(s.saved)
    if c.op == "fork":
        rr.rr_cache_fork(s.cache, s.parents, s.children)
        rr.rr_cache_extend(s.cache, s.seqs, starts=s.starts)
        rr.rr_cache_append(s.cache, s.layer, s.k, s.v, s.seqs, starts=s.starts)
        rr.rr_cache_truncate(s.cache, s.back, s.drop)
    else:
        rr.rr_cache_truncate(s.cache, s.gone, s.drop)
        rr.rr_cache_compact(s.cache)
    return {"pages": s.cache.pages, "table": s.cache.table, "lengths": s.cache.lengths,
            "refs": s.cache.refs}


def _attend_plain(s):
    c = s.c
    out, lse, at = [], [], 0
    scale = c.dim ** -0.5
    for i, (length, n) in enumerate(zip(s.lengths, s.counts)):
        held = s.table[i, :-(-length // c.page)].long()
        # [2, kv heads, tokens, dim]
        kv = s.pages[held, s.layer].float().permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :length, :c.dim]
        q = s.q[at:at + n].float().view(n, c.n_kv, -1, c.dim).transpose(0, 1).flatten(1, 2)
        score = torch.matmul(q, kv[0].transpose(1, 2)) * scale
        if n > 1:
            row = torch.arange(n, device="cuda").repeat_interleave(c.n_q // c.n_kv)
            hidden = torch.arange(length, device="cuda") > (length - n + row)[:, None]
            score = torch.where(hidden, -math.inf, score)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - top)
        total = e.sum(-1, keepdim=True)
        y = torch.matmul(e, kv[1]) / total
        out.append(y.view(c.n_kv, n, -1, c.dim).transpose(0, 1).reshape(n, c.n_q, c.dim))
        lse.append((top + torch.log(total)).view(c.n_kv, n, -1).transpose(0, 1).reshape(n, c.n_q))
        at += n
    return {"out": torch.cat(out).to(s.q.dtype), "lse": torch.cat(lse)}


def _free_pages(refs):
    """The pool's pages, the free ones first, each part in ascending order."""
    return torch.sort((refs > 0).to(torch.int8), stable=True).indices


def _truncate_plain(c, table, lens, refs, seqs, drop):
    seqs = seqs.long()
    rows = table[seqs]
    n = lens[seqs] - drop
    column = torch.arange(table.shape[1], device="cuda")
    gone = (column >= ((n + c.page - 1) // c.page)[:, None]) & (rows >= 0)
    refs.index_add_(0, rows.clamp_min(0).flatten().long(), -gone.flatten().to(torch.int32))
    table[seqs] = torch.where(gone, -1, rows)
    lens[seqs] = n.to(torch.int32)


def _fork_plain(s):
    c = s.c
    table, lens, refs, pages = s.table.clone(), s.lens.clone(), s.refs.clone(), s.pages
    # Children share their parent's pages.
    parents, children, seqs = s.parents.long(), s.children.long(), s.seqs.long()
    rows = table[parents]
    table[children] = rows
    lens[children] = lens[parents]
    refs.index_add_(0, rows.clamp_min(0).flatten().long(), (rows >= 0).flatten().to(torch.int32))
    # New tokens: a shared page that is partly filled is copied by all its holders, or,
    # where all of them are listed, by all but the last.
    n = lens[seqs].long()
    column = torch.arange(table.shape[1], device="cuda")
    rows = table[seqs]
    held = rows.gather(1, (n // c.page).clamp_max(table.shape[1] - 1)[:, None]).squeeze(1).long()
    held = torch.where(n % c.page > 0, held, -1)
    holders = torch.where(held >= 0, refs[held.clamp_min(0)].long(), 0)
    same = (held[:, None] == held) & (holders > 1)[:, None]
    last = ~same.triu(1).any(1)
    copies = (holders > 1) & ~((same.sum(1) == holders) & last)
    first, end = (n + c.page - 1) // c.page, (n + c.new + c.page - 1) // c.page
    need = copies.long() + end - first
    at = need.cumsum(0) - need
    free = _free_pages(refs)
    to = free[at.clamp_max(len(free) - 1)]
    grown = (column >= first[:, None]) & (column < end[:, None])
    fresh = free[((at + copies)[:, None] + column - first[:, None]).clamp(0, len(free) - 1)]
    moved = (column == (n // c.page)[:, None]) & copies[:, None]
    table[seqs] = torch.where(grown, fresh, torch.where(moved, to[:, None], rows)).to(torch.int32)
    refs.index_add_(0, held.clamp_min(0), -copies.to(torch.int32))
    refs[free] += (torch.arange(len(free), device="cuda") < need.sum()).to(torch.int32)
    lens[seqs] = (n + c.new).to(torch.int32)
    src, dst = held[copies], to[copies]
    filled = torch.arange(c.page, device="cuda") < (n % c.page)[copies][:, None]
    pages[dst] = torch.where(filled[:, None, None, None, :, None], pages[src], pages[dst])
    # The new tokens' keys and values.
    pos = (n[:, None] + torch.arange(c.new, device="cuda")).flatten()
    page = table[seqs.repeat_interleave(c.new), pos // c.page].long()
    for half, x in enumerate((s.k, s.v)):
        padded = torch.nn.functional.pad(x, (0, pages.shape[-1] - c.dim))
        pages[page, s.layer, half, :, pos % c.page] = padded
    _truncate_plain(c, table, lens, refs, s.back, s.drop)
    return {"pages": pages, "table": table, "lengths": lens, "refs": refs}


def _compact_plain(s):
    c = s.c
    table, lens, refs, pages = s.table.clone(), s.lens.clone(), s.refs.clone(), s.pages
    _truncate_plain(c, table, lens, refs, s.gone, s.drop)
    page = torch.arange(len(refs), device="cuda")
    front = page < (refs > 0).sum()
    src, dst = page[~front & (refs > 0)], page[front & (refs == 0)]
    pages[dst] = pages[src]
    refs[dst] = refs[src]
    refs[src] = 0
    page[src] = dst
    table = torch.where(table >= 0, page[table.clamp_min(0).long()], -1).to(torch.int32)
    return {"pages": pages, "table": table, "lengths": lens, "refs": refs}


def _units(x):
    """Probabilities as whole numbers of 2^-42; products of 2^42 are exact in 64 bits."""
    x = torch.nan_to_num(x, nan=0.0).clamp(0, 1)
    return torch.round(x.double() * 2.0 ** 42).long()


def _accept_plain(s):
    c = s.c
    start = s.starts.long()
    n = start[1:] - start[:-1] - 1
    row = torch.arange(c.drafts + 1, device="cuda")
    at = (start[:-1, None] + row).clamp_max(s.p.shape[0] - 1)
    x = s.drafts.long()[:, None]
    px = s.p.gather(1, x).squeeze(1).double()
    qx = torch.ones_like(px) if s.q is None else s.q.gather(1, x).squeeze(1).double()
    passed = ((s.u.double() * qx < px)[at]) & (row < n[:, None])
    accepted = passed.long().cumprod(1).sum(1)
    final = start[:-1] + accepted
    refused = (accepted < n)[:, None]
    p = s.p[final]
    if s.q is None:
        r = torch.where(refused & (torch.arange(c.vocab, device="cuda") == x[final]), 0.0, p)
    else:
        r = torch.where(refused, p - s.q[final], p)
    w = _units(r)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, _units(p))
    sums = w.cumsum(1)
    total = sums[:, -1]
    # floor(total * v): v in whole numbers of 2^-31, the total in two halves.
    v = torch.floor(s.v.double().clamp(0, 1) * 2.0 ** 31).long().clamp_max((1 << 31) - 1)
    t = (total >> 31) * v + ((total & ((1 << 31) - 1)) * v >> 31)
    token = (sums <= t[:, None]).sum(1)
    token = torch.where(total > 0, token, -1)
    seq = torch.repeat_interleave(torch.arange(c.seqs, device="cuda"), n + 1,
                                  output_size=s.p.shape[0])
    j = torch.arange(s.p.shape[0], device="cuda") - start[seq]
    a = accepted[seq]
    tokens = torch.where(j < a, s.drafts.long(), torch.where(j == a, token[seq], -1))
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32),
            "rejected": (n - accepted).to(torch.int32)}


def run(s):
    if own:
        return _run_own(s)
    return {"attend": _attend_plain, "fork": _fork_plain, "compact": _compact_plain,
            "accept": _accept_plain}[s.c.op](s)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_attend(c, d):
    group = c.n_q // c.n_kv
    out = torch.empty(d.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(d.q.shape[:2], dtype=torch.float64, device="cuda")
    first = 0
    for i in range(c.seqs):
        held = d.table[i][d.table[i] >= 0].long()
        for h in range(c.n_kv):
            k = d.pages[held, d.layer, 0, h].reshape(-1, d.pages.shape[-1])[:, :c.dim].double()
            v = d.pages[held, d.layer, 1, h].reshape(-1, d.pages.shape[-1])[:, :c.dim].double()
            for j in range(d.counts[i]):
                seen = d.lengths[i] - d.counts[i] + 1 + j
                heads = slice(h * group, (h + 1) * group)
                score = d.q[first + j, heads].double() @ k[:seen].T / math.sqrt(c.dim)
                lse[first + j, heads] = torch.logsumexp(score, 1)
                out[first + j, heads] = torch.softmax(score, 1) @ v[:seen]
        first += d.counts[i]
    return {"out": out, "lse": lse}


class _Book:
    """A cache's bookkeeping on the host, one page after another."""

    def __init__(self, c, d):
        self.c, self.d = c, d
        self.refs = d.refs.tolist()
        lens = d.lens.tolist()
        self.held = [row[:-(-n // c.page)] for row, n in zip(d.table.tolist(), lens)]
        self.lens = lens
        self.pages = d.pages.clone()

    def drop(self, seq, n):
        self.lens[seq] -= n
        while len(self.held[seq]) > -(-self.lens[seq] // self.c.page):
            self.refs[self.held[seq].pop()] -= 1

    def result(self):
        table = [row + [-1] * (self.d.max_pages - len(row)) for row in self.held]
        return {"pages": self.pages, "table": _ints(table), "lengths": _ints(self.lens),
                "refs": _ints(self.refs)}


def _exact_fork(c, d):
    b = _Book(c, d)
    for parent, child in zip(d.parents.tolist(), d.children.tolist()):
        b.held[child] = list(b.held[parent])
        b.lens[child] = b.lens[parent]
        for page in b.held[parent]:
            b.refs[page] += 1
    seqs = d.seqs.tolist()
    partly = {s: b.held[s][-1] for s in seqs if b.lens[s] % c.page}
    before = list(b.refs)
    free = iter([page for page, n in enumerate(before) if n == 0])
    for i, s in enumerate(seqs):
        filled = b.lens[s] % c.page
        if filled and before[partly[s]] > 1:
            listed_too = [t for t in seqs if partly.get(t) == partly[s]]
            if not (len(listed_too) == before[partly[s]] and listed_too[-1] == s):
                to = next(free)
                b.pages[to][..., :filled, :] = b.pages[partly[s]][..., :filled, :]
                b.refs[partly[s]] -= 1
                b.refs[to] = 1
                b.held[s][-1] = to
        while len(b.held[s]) * c.page < b.lens[s] + c.new:
            page = next(free)
            b.refs[page] = 1
            b.held[s].append(page)
    for i, s in enumerate(seqs):
        for j in range(c.new):
            pos = b.lens[s] + j
            page = b.held[s][pos // c.page]
            for half, x in enumerate((d.k, d.v)):
                row = b.pages[page, d.layer, half, :, pos % c.page]
                row.zero_()
                row[:, :c.dim] = x[i * c.new + j]
        b.lens[s] += c.new
    for s, n in zip(d.back.tolist(), d.drop.tolist()):
        b.drop(s, n)
    return b.result()


def _exact_compact(c, d):
    b = _Book(c, d)
    for s, n in zip(d.gone.tolist(), d.drop.tolist()):
        b.drop(s, n)
    used = sum(1 for n in b.refs if n)
    holes = [page for page in range(used) if b.refs[page] == 0]
    behind = [page for page in range(used, len(b.refs)) if b.refs[page]]
    goes = dict(zip(behind, holes))
    for page, to in goes.items():
        b.pages[to] = b.pages[page]
        b.refs[to], b.refs[page] = b.refs[page], 0
    b.held = [[goes.get(page, page) for page in row] for row in b.held]
    return b.result()


def _exact_accept(c, d):
    accepted, tokens = [], []
    starts, drafts, u, v = (x.tolist() for x in (d.starts, d.drafts, d.u, d.v))
    for i in range(c.seqs):
        lo, n = starts[i], starts[i + 1] - starts[i] - 1
        a = 0
        while a < n:
            x = drafts[lo + a]
            own_chance = 1.0 if d.q is None else d.q[lo + a, x].item()
            if not u[lo + a] * own_chance < d.p[lo + a, x].item():
                break
            a += 1
        p = d.p[lo + a].clone()
        rest = p.clone()
        if a < n and d.q is None:
            rest[drafts[lo + a]] = 0
        elif a < n:
            rest -= d.q[lo + a]
        for r in (rest, p):
            units = (r.clamp(0, 1).double() * 2.0 ** 42).round().cpu().numpy().astype("int64")
            total = int(units.sum())
            if total:
                break
        token = -1
        if total:
            t = total * min(int(v[i] * 2 ** 31), 2 ** 31 - 1) >> 31
            token = int(units.cumsum().searchsorted(t, side="right"))
        accepted.append(a)
        tokens += drafts[lo:lo + a] + [token] + [-1] * (n - a)
    counts = [b - a - 1 for a, b in zip(starts, starts[1:])]
    return {"accepted": _ints(accepted), "tokens": _ints(tokens),
            "rejected": _ints([n - a for n, a in zip(counts, accepted)])}


def exact(case, seed):
    c = SimpleNamespace(**case)
    d = _inputs(c, seed)
    return {"attend": _exact_attend, "fork": _exact_fork, "compact": _exact_compact,
            "accept": _exact_accept}[c.op](c, d)
