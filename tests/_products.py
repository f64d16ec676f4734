"""Plain restatements, in 64 bits on the CPU, of the products of include/rr.h,
with bounds on how far float32 sums and one final rounding may be from them.

They import nothing of the library.  Each function that the tests compare with
returns (value, tolerance).

How the bounds come about.  u is the most that rounding to nearest changes a
result of p significant bits, 2^-p relative: 2^-8 for bfloat16 (p = 8), 2^-11 for
float16 (p = 11; 2^-25 absolute under its normal range), 2^-24 for float32.  A float32 sum of K products goes through at most K / 8 + 64 additions
on any one path (a matrix instruction adds 8 or more products at once, warps and
groups split K further), each of which may cut off at 2^-23 of the partial
result, which is at most S = sum |w x|; products of 16-bit values are exact.
So |error| <= (K / 8 + 64) 2^-23 S, plus u |y| at the end.
"""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def sum_error(k: int) -> float:
    return (k / 8 + 64) * 2.0 ** -23


def rounding(y, kind: str):
    """The most that rounding a value near y to `kind` changes it."""
    return ROUND[kind] * y.abs() + (2.0 ** -25 if kind == "f16" else 0.0)


def quantize(w, group: int):
    """(codes, scales) of a 16-bit matrix [rows, cols]: int64, and the 16-bit scales."""
    rows, cols = w.shape
    n = math.ceil(cols / group)
    q = torch.zeros(rows, cols, dtype=torch.int64)
    s = torch.zeros(rows, n, dtype=w.dtype)
    v = w.double()
    for i in range(n):
        a, b = i * group, min((i + 1) * group, cols)
        part = v[:, a:b]
        top = part.abs().max(1).values          # NaN if any is
        # top and 7 are exact in float32: one division, rounded, then the type's.
        one = (top.float() / torch.tensor(7.0)).to(w.dtype)
        d = one.double()
        d[d < 2.0 ** -126] = 0.0
        code = torch.round(part / d.unsqueeze(1)).clamp(-7, 7)
        dead = (d == 0) | ~torch.isfinite(top)
        code[dead] = 0
        d[~torch.isfinite(top)] = math.nan
        q[:, a:b] = code.long()
        s[:, i] = d.to(w.dtype)
    return q, s


def values(q, s, group: int):
    """What codes and scales stand for, in 64 bits."""
    return q.double() * s.double().repeat_interleave(group, 1)[:, :q.shape[1]]


def pack(q, s, group: int, pair: bool) -> np.ndarray:
    """The packed bytes of one matrix, element by element from rr.h's words."""
    rows, cols = q.shape
    blocks = math.ceil(cols / 128)
    strips = math.ceil(rows / 2 / 8) if pair else math.ceil(rows / 16)
    size = 1024 + 4096 // group
    out = np.zeros(strips * blocks * size, np.uint8)
    per = 128 // group
    for strip in range(strips):
        for b in range(blocks):
            at = (strip * blocks + b) * size
            code = np.full((16, 128), 8, np.uint64)
            scale = np.zeros((16, per), np.uint16)
            for r in range(16):
                if pair:
                    i = 8 * strip + r % 8
                    row = (i if r < 8 else rows // 2 + i) if i < rows // 2 else -1
                else:
                    row = 16 * strip + r if 16 * strip + r < rows else -1
                if row < 0:
                    continue
                end = min(cols, 128 * b + 128)
                code[r, :end - 128 * b] = (q[row, 128 * b:end] + 8).numpy()
                for i in range(per):
                    k = b * per + i
                    if k < s.shape[1]:
                        scale[r, i] = s[row, k].reshape(1).view(torch.int16).numpy().view(np.uint16)[0]
            for h in range(2):
                for g in range(8):
                    for t in range(4):
                        for j in range(4):
                            word = 0
                            for i in range(8):
                                n = i // 2 + 4 * (i % 2)
                                word |= int(code[8 * h + g, 32 * j + 8 * t + i]) << (4 * n)
                            p = at + 512 * h + 16 * (4 * g + t) + 4 * j
                            out[p:p + 4] = np.frombuffer(np.uint32(word).tobytes(), np.uint8)
                    for i in range(per):
                        p = at + 1024 + 2 * (2 * (g * per + i) + h)
                        out[p:p + 2] = np.frombuffer(scale[8 * h + g, i].tobytes(), np.uint8)
    return out


def silu(z):
    return z / (1 + torch.exp(-z))


def swiglu(gate, up, gate_err, up_err):
    """(silu(gate) * up, bound): |silu'| <= 1.1, and exp, the division and the
    product are within 2^-20 of theirs (the few units in the last place that
    CUDA's exp, IEEE division and multiplication may be off)."""
    h = silu(gate) * up
    err = 1.1 * gate_err * (up.abs() + up_err) + silu(gate).abs() * up_err + 2.0 ** -20 * h.abs()
    return h, err


def matvec(w, x, pair: bool, kind: str):
    """w: values [rows, cols] in 64 bits; x: [tokens, cols]."""
    x = x.double()
    y = x @ w.T
    err = sum_error(w.shape[1]) * (x.abs() @ w.abs().T)
    if pair:
        n = w.shape[0] // 2
        y, err = swiglu(y[:, :n], y[:, n:], err[:, :n], err[:, n:])
    return y, err + rounding(y, kind)


def route(x, router, top_k: int, norm: bool):
    """(ids, weights): the top_k largest logits, ties to the lowest index."""
    l = x.double() @ router.double().T
    ids = torch.empty(x.shape[0], top_k, dtype=torch.int64)
    c = torch.empty(x.shape[0], top_k, dtype=torch.float64)
    for t in range(x.shape[0]):
        row = [math.inf if math.isnan(v) else v for v in l[t].tolist()]
        order = sorted(range(len(row)), key=lambda e: (-row[e], e))[:top_k]
        p = torch.softmax(l[t], 0)
        ids[t] = torch.tensor(order)
        c[t] = p[order]
        if norm:
            c[t] = c[t] / c[t].sum()
    return ids, c


def moe(x, ids, c, w13, w2, first: int, kind: str):
    """w13 [local, 2 inter, hidden], w2 [local, hidden, inter] in 64 bits.  Of the
    bounds: h is held in two 16-bit parts (2^-16 relative), c is within 2^-18
    (sum and exponentials of up to 512 logits), and the sum over top_k <= 16
    experts adds 16 * 2^-24."""
    x = x.double()
    out = torch.zeros(x.shape[0], w2.shape[1], dtype=torch.float64)
    err = torch.zeros_like(out)
    for t in range(x.shape[0]):
        for j in range(ids.shape[1]):
            e = int(ids[t, j]) - first
            if not 0 <= e < w13.shape[0]:
                continue
            n = w13.shape[1] // 2
            gu = w13[e] @ x[t]
            ge = sum_error(w13.shape[2]) * (w13[e].abs() @ x[t].abs())
            h, he = swiglu(gu[:n], gu[n:], ge[:n], ge[n:])
            he = he + 2.0 ** -16 * h.abs()
            y = w2[e] @ h
            ye = w2[e].abs() @ he + sum_error(n) * (w2[e].abs() @ h.abs())
            out[t] += c[t, j] * y
            err[t] += c[t, j] * (ye + (2.0 ** -18 + 16 * 2.0 ** -24) * y.abs())
    return out, err + rounding(out, kind)


def check(got, want, tol, what=""):
    """got (any type) within tol of want; NaN and infinities in the same places."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine] - tol[fine]
    assert off.numel() == 0 or off.max().item() <= 0, \
        f"{what}: {off.max().item():.3g} over the bound ({int((off > 0).sum())} of {off.numel()})"


def grid_tokens(gen, tokens, hidden, kind):
    """Tokens on multiples of 1/32: with grid_router, logits are exact in float32
    in any order of summation, so the choice of experts is, too."""
    x = torch.randn(tokens, hidden, generator=gen)
    return (torch.round(x * 32) / 32).clamp(-7.9375, 7.9375).to(TYPES[kind])


def grid_router(gen, experts, hidden, kind):
    r = torch.randn(experts, hidden, generator=gen) * (0.9 / math.sqrt(hidden))
    return (torch.round(r * 512) / 512).clamp(-0.49, 0.49).to(TYPES[kind])
