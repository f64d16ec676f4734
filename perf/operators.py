"""The operators on weights that have arrived in a rollout's layout, as timed cases.

Kinds of pass (``op``):
  quantize  a 16-bit weight matrix, as ``rr_unpack`` leaves it, to 4-bit codes with
            group scales, and back to the values that these stand for
            (``rr_quantize``, ``rr_dequantize``)
  matvec    products of such a matrix with 1 to 16 tokens (``rr_matvec``);
            ``pair``: the matrix is [gate; up] and the result silu(gate) * up
  moe       a whole mixture-of-experts layer for 1 to 64 tokens (``rr_moe``): router,
            choice of experts, their products and the weighted sum; ``first`` and
            ``local``: the experts that this rank holds; ``group`` 0: 16-bit experts,
            else 4-bit ones

``run`` computes them in elementary torch operations in 32 bits, or, where ``own``
is true, with the library's kernels.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MIB = 1 << 20


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _quantize(rows, cols, group, dtype="bf16", pair=False, name=None):
    c = dict(op="quantize", rows=rows, cols=cols, group=group, dtype=dtype, pair=pair)
    return dict(c, name=name) if name else c


def _matvec(rows, cols, tokens, group, dtype="bf16", pair=False, f32=False, name=None):
    c = dict(op="matvec", rows=rows, cols=cols, tokens=tokens, group=group, dtype=dtype,
             pair=pair, f32=f32)
    return dict(c, name=name) if name else c


def _moe(experts, hidden, inter, tokens, top_k, first=0, local=None, group=0, dtype="bf16",
         norm=True, name=None):
    c = dict(op="moe", experts=experts, hidden=hidden, inter=inter, tokens=tokens, top_k=top_k,
             first=first, local=experts if local is None else local, group=group, dtype=dtype,
             norm=norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The test model of odd sizes: a matrix that no vector width divides.
        _quantize(689, 257, 32, "f16", name="quantize_odd_f16"),
        # The largest dense matrix of a Qwen3-8B layer after a sync.
        _quantize(24576, 4096, 128, pair=True, name="quantize_8b_gate_up"),
        # The smallest product: one token through the two-layer test model's QKV.
        _matvec(512, 256, 1, 32, name="matvec_tiny_qkv"),
        # Odd sizes, three tokens.
        _matvec(1378, 257, 3, 64, "f16", name="matvec_odd_f16"),
        # One sequence's token step in Qwen3-8B.
        _matvec(6144, 4096, 1, 128, name="matvec_8b_qkv"),
        # A few sequences, fused gate and up.
        _matvec(24576, 4096, 4, 128, pair=True, name="matvec_8b_gate_up_4"),
        # Eight sequences, a long inner dimension.
        _matvec(5120, 25600, 8, 64, "f16", name="matvec_32b_down_8_f16"),
        # Logits in 32 bits, as sampling reads them.
        _matvec(151936, 4096, 1, 128, f32=True, name="matvec_8b_lm_head_f32"),
        # The test model's MoE layer, where launch and waits count.
        _moe(8, 128, 96, 1, 2, name="moe_tiny"),
        # One sequence's token step in Qwen3-30B-A3B.
        _moe(128, 2048, 768, 1, 8, name="moe_30b_1"),
        # A full batch of the same: nearly every expert is read.
        _moe(128, 2048, 768, 64, 8, name="moe_30b_64"),
        # An expert-parallel rank (3 of 8) with 4-bit experts: tokens without a local expert.
        _moe(128, 2048, 768, 16, 8, first=48, local=16, group=64, dtype="f16",
             name="moe_30b_ep8_16_q4_f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("quantize", "matvec", "matvec", "moe", "moe"))
    dtype = rng.choice(("bf16", "f16"))
    group = rng.choice((32, 64, 128))
    while True:
        if op == "quantize":
            pair = rng.random() < 0.3
            rows = _log(rng, 64, 65536)
            c = _quantize(2 * rows if pair else rows, _log(rng, 64, 16384), group, dtype, pair)
        elif op == "matvec":
            pair = rng.random() < 0.3
            rows = _log(rng, 64, 65536)
            c = _matvec(2 * rows if pair else rows, _log(rng, 64, 25600), rng.randint(1, 16),
                        group, dtype, pair, f32=rng.random() < 0.25)
        else:
            local = rng.choice((4, 8, 16, 32, 64, 128))
            ranks = rng.choice((1, 1, 2, 4)) if local < 128 else 1
            experts = local * ranks
            c = _moe(experts, _log(rng, 64, 4096), _log(rng, 48, 2048), _log(rng, 1, 64),
                     rng.randint(1, min(8, experts)), first=local * rng.randrange(ranks),
                     local=local, group=rng.choice((0, 0, group)), dtype=dtype,
                     norm=rng.random() < 0.75)
        weights = 3 * c["local"] * c["hidden"] * c["inter"] if op == "moe" \
            else c["rows"] * c["cols"]
        if weights <= (96 * MIB if op == "quantize" else 576 * MIB):
            return c


def _packed_bytes(rows, cols, group):
    return rows * cols / 2 + 2 * rows * math.ceil(cols / group)


def work(case):
    c = SimpleNamespace(**case)
    if c.op == "quantize":
        n = c.rows * c.cols
        return {"bytes": 4 * n + _packed_bytes(c.rows, c.cols, c.group), "flops": 3 * n}
    if c.op == "matvec":
        n_out = c.rows // 2 if c.pair else c.rows
        return {"bytes": _packed_bytes(c.rows, c.cols, c.group) + 2 * c.tokens * c.cols
                + (4 if c.f32 else 2) * c.tokens * n_out,
                "flops": 2 * c.tokens * c.rows * c.cols}
    # Experts that at least one token chooses, when every choice is as likely.
    used = c.local * (1 - (1 - c.top_k / c.experts) ** c.tokens)
    each = 6 * c.hidden * c.inter
    if c.group:
        each = _packed_bytes(2 * c.inter, c.hidden, c.group) \
            + _packed_bytes(c.hidden, c.inter, c.group)
    pairs = c.tokens * c.top_k * c.local / c.experts
    return {"bytes": 2 * c.experts * c.hidden + used * each + 4 * c.tokens * c.hidden
            + 8 * c.tokens * c.top_k,
            "flops": 6 * pairs * c.hidden * c.inter + 2 * c.tokens * c.experts * c.hidden}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _weights(shape, dtype, gen, std=0.02):
    return torch.empty(shape, dtype=TYPES[dtype], device="cuda").normal_(0.0, std, generator=gen)


def _activations(tokens, cols, dtype, gen):
    """Normalised activations: unit variance, a few channels far above the others."""
    x = torch.randn(tokens, cols, device="cuda", generator=gen)
    loud = torch.rand(cols, device="cuda", generator=gen) < 0.002
    return torch.where(loud, 20 * x, x).to(TYPES[dtype])


def _codes(w, group):
    """Codes (whole numbers, int8) and scales of a matrix [..., rows, cols], by group."""
    cols = w.shape[-1]
    n = -(-cols // group)
    v = torch.nn.functional.pad(w.float(), (0, n * group - cols)).unflatten(-1, (n, group))
    top = v.abs().amax(-1)
    s = (top / 7).to(w.dtype)
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    s = torch.where(torch.isfinite(top), s, torch.full_like(s, math.nan))
    f = s.float().unsqueeze(-1)
    q = torch.where(f > 0, torch.round(v / f).clamp(-7, 7), torch.zeros_like(v))
    return q.flatten(-2)[..., :cols].to(torch.int8), s


def _values(q, s, group):
    """The values that codes and scales stand for, in 32 bits."""
    return q.float() * s.float().repeat_interleave(group, -1)[..., :q.shape[-1]]


def _inputs(c, seed):
    """A case's tensors, from the seed alone."""
    gen = torch.Generator("cuda").manual_seed(seed)
    d = SimpleNamespace()
    if c.op == "moe":
        # Tokens and router on coarse grids, so that logits are exact in 32 bits in any
        # order of summation, and the choice of experts does not hang on that order.
        t = TYPES[c.dtype]
        x = torch.randn(c.tokens, c.hidden, device="cuda", generator=gen)
        d.x = (torch.round(x * 32) / 32).clamp(-7.9375, 7.9375).to(t)
        r = 0.02 * torch.randn(c.experts, c.hidden, device="cuda", generator=gen)
        d.router = (torch.round(r * 512) / 512).to(t)
        d.w13 = _weights((c.local, 2 * c.inter, c.hidden), c.dtype, gen)
        d.w2 = _weights((c.local, c.hidden, c.inter), c.dtype, gen)
    else:
        d.w = _weights((c.rows, c.cols), c.dtype, gen)
        if c.op == "matvec":
            d.x = _activations(c.tokens, c.cols, c.dtype, gen)
    return d


def prepare(case, seed):
    c = SimpleNamespace(**case)
    d = _inputs(c, seed)
    t = TYPES[c.dtype]
    s = SimpleNamespace(c=c)
    if c.op != "quantize" and not own:
        if c.op == "matvec":
            s.x = d.x
            s.q, s.s = _codes(d.w, c.group)
        elif c.group:
            s.x, s.router = d.x, d.router
            n = range(c.local)
            s.q13, s.s13 = (torch.stack(p) for p in zip(*(_codes(d.w13[e], c.group) for e in n)))
            s.q2, s.s2 = (torch.stack(p) for p in zip(*(_codes(d.w2[e], c.group) for e in n)))
        else:
            s.x, s.router, s.w13, s.w2 = d.x, d.router, d.w13, d.w2
        return s
    if not own:
        s.w = d.w
        return s
    import paper_2512_22492_gb300 as rr
    s.rr = rr
    if c.op == "quantize":
        s.w = d.w
        s.q = rr.Quantized(c.rows, c.cols, group=c.group, dtype=c.dtype, pair=c.pair)
        s.out = torch.empty(c.rows, c.cols, dtype=t, device="cuda")
    elif c.op == "matvec":
        s.x = d.x
        s.q = rr.Quantized(c.rows, c.cols, group=c.group, dtype=c.dtype, pair=c.pair)
        rr.rr_quantize(s.q, d.w)
        s.out = torch.empty(c.tokens, c.rows // 2 if c.pair else c.rows,
                            dtype=torch.float32 if c.f32 else t, device="cuda")
    else:
        s.x = d.x
        w13, w2 = d.w13, d.w2
        if c.group:
            w13 = rr.Quantized(2 * c.inter, c.hidden, group=c.group, dtype=c.dtype, pair=True,
                               count=c.local)
            w2 = rr.Quantized(c.hidden, c.inter, group=c.group, dtype=c.dtype, count=c.local)
            rr.rr_quantize(w13, d.w13)
            rr.rr_quantize(w2, d.w2)
        s.layer = rr.MoeLayer(d.router, w13, w2, top_k=c.top_k, first_expert=c.first,
                              norm_topk=c.norm)
        s.workspace = rr.MoeWorkspace(s.layer, c.tokens)
        s.out = torch.empty(c.tokens, c.hidden, dtype=t, device="cuda")
        s.ids = torch.empty(c.tokens, c.top_k, dtype=torch.int32, device="cuda")
        s.weights = torch.empty(c.tokens, c.top_k, dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _run_own(s):
    c, rr = s.c, s.rr
    if c.op == "quantize":
        rr.rr_quantize(s.q, s.w)
        rr.rr_dequantize(s.q, s.out)
        return s.out
    if c.op == "matvec":
        rr.rr_matvec(s.q, s.x, s.out)
        return s.out
    rr.rr_moe(s.layer, s.x, s.out, s.workspace, ids=s.ids, weights=s.weights)
    return {"out": s.out, "ids": s.ids, "weights": s.weights}


def _silu_mul(gate, up):
    return gate / (1 + torch.exp(-gate)) * up


def _moe_plain(s):
    c = s.c
    x = s.x.float()
    logits = x @ s.router.float().T
    ids = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :c.top_k]
    e = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = (e / e.sum(-1, keepdim=True)).gather(1, ids)
    if c.norm:
        p = p / p.sum(-1, keepdim=True)
    here = (ids >= c.first) & (ids < c.first + c.local)
    at = torch.where(here, ids - c.first, torch.zeros_like(ids)).flatten()
    few = c.tokens * c.top_k <= c.local
    # Each pair's own copy of its expert, or, where pairs outnumber experts, every expert
    # on every token.
    pick = at if few else slice(None)
    w13 = _values(s.q13[pick], s.s13[pick], c.group) if c.group else s.w13[pick].float()
    gu = torch.matmul(w13, x.repeat_interleave(c.top_k, 0).unsqueeze(-1) if few else x.T)
    del w13
    h = _silu_mul(gu[:, :c.inter], gu[:, c.inter:])
    w2 = _values(s.q2[pick], s.s2[pick], c.group) if c.group else s.w2[pick].float()
    y = torch.matmul(w2, h)
    del w2
    if few:
        y = y.squeeze(-1)
    else:
        y = y.transpose(1, 2)[at, torch.arange(c.tokens, device="cuda")
                              .repeat_interleave(c.top_k)]
    y = y.unflatten(0, (c.tokens, c.top_k))
    out = torch.where(here.unsqueeze(-1), p.unsqueeze(-1) * y, torch.zeros_like(y)).sum(1)
    return {"out": out.to(s.x.dtype), "ids": ids.to(torch.int32), "weights": p}


def run(s):
    if own:
        return _run_own(s)
    c = s.c
    if c.op == "quantize":
        return _values(*_codes(s.w, c.group), c.group).to(s.w.dtype)
    if c.op == "moe":
        return _moe_plain(s)
    y = s.x.float() @ _values(s.q, s.s, c.group).T
    if c.pair:
        y = _silu_mul(y[:, :c.rows // 2], y[:, c.rows // 2:])
    return y if c.f32 else y.to(s.x.dtype)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _stand_for(w, group):
    """What a matrix's codes and scales stand for, group after group, in 64 bits."""
    out = torch.empty(w.shape, dtype=torch.float64, device=w.device)
    for a in range(0, w.shape[1], group):
        v = w[:, a:a + group].double()
        top = v.abs().max(dim=1, keepdim=True).values
        s = (top / 7).to(w.dtype).double()
        s[s < 2.0 ** -126] = 0.0
        q = torch.round(v / s.clamp_min(2.0 ** -126)).clamp(-7, 7)
        out[:, a:a + group] = s * q
    return out


def exact(case, seed):
    c = SimpleNamespace(**case)
    d = _inputs(c, seed)
    if c.op == "quantize":
        return _stand_for(d.w, c.group)
    if c.op == "matvec":
        y = []
        for a in range(0, c.rows, 4096):
            w = _stand_for(d.w[a:a + 4096], c.group)
            y.append((w @ d.x.double().T).T)
        y = torch.cat(y, 1)
        if c.pair:
            gate, up = y.split(c.rows // 2, 1)
            y = gate * torch.sigmoid(gate) * up
        return y
    x = d.x.double()
    p = torch.softmax(x @ d.router.double().T, -1)
    order = torch.sort(p, dim=-1, descending=True, stable=True)
    weight, ids = order.values[:, :c.top_k], order.indices[:, :c.top_k]
    if c.norm:
        weight = weight / weight.sum(1, keepdim=True)
    out = torch.zeros(c.tokens, c.hidden, dtype=torch.float64, device="cuda")
    for e in range(c.local):
        t, j = torch.nonzero(ids == c.first + e, as_tuple=True)
        if not t.numel():
            continue
        w13 = _stand_for(d.w13[e], c.group) if c.group else d.w13[e].double()
        w2 = _stand_for(d.w2[e], c.group) if c.group else d.w2[e].double()
        gate, up = (x[t] @ w13.T).split(c.inter, 1)
        h = gate * torch.sigmoid(gate) * up
        out[t] += weight[t, j].unsqueeze(1) * (h @ w2.T)
    return {"out": out, "ids": None, "weights": weight}
