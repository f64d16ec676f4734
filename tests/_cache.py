"""Plain restatements, on the CPU, of the cache, its attention and the verification of drafted
tokens (include/rr.h); they import nothing of the library.

Bounds of the attention.  u is the most that rounding to nearest changes a value, relative:
2^-8 for bfloat16, 2^-11 for float16, 2^-24 for float32 (tests/_products.py).  A score
is a sum of dim exact products in float32, by at most dim / 8 + 64 additions on a path, each
of which may cut off at 2^-23 of S = sum |q k|: off by at most
    E = scale S (dim / 8 + 64) 2^-23 + 4 |s| 2^-24
with its factor (scale and log2(e), two roundings) and its difference from the reference.
Weights exp(s - max) are then off by exp(E) - 1, those in the sum and those of the products
alike, and by 2^-21 for the exponential itself; in the product they are cut to 2^-16
(bfloat16, two parts of 8 bits) or 2^-11 of themselves, float16 also to 2^-32 of the largest.
Sums of L of them go through at most L / 8 + 64 additions.  With A = sum w |v| / sum w:
    |out| is off by at most A (2 (exp(E) - 1) + 2^-20 + cut + (L / 8 + 64) 2^-22)
                            + 2^-32 L max |v| (float16) + u |out|,
    |lse| by E + 2^-21 + (L / 8 + 64) 2^-23 + 2^-22 |lse| + 2^-22.
"""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
CUT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -11}


class Book:
    """A cache's bookkeeping and contents: pages [n_pages, layers, 2, n_kv, page, pitch] on the CPU."""

    def __init__(self, pages, max_seqs, page):
        self.pages, self.page = pages.clone(), page
        self.held = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs

    @property
    def refs(self):
        n = [0] * len(self.pages)
        for row in self.held:
            for p in row:
                n[p] += 1
        return n

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            assert not self.lens[c]
        for p, c in zip(parents, children):
            self.held[c], self.lens[c] = list(self.held[p]), self.lens[p]

    def extend(self, seqs, counts):
        """False, and nothing done, if the pool has no room."""
        refs = self.refs
        free = [p for p, n in enumerate(refs) if not n]
        partly = [self.held[s][-1] if self.lens[s] % self.page and c else None
                  for s, c in zip(seqs, counts)]
        plan, k = [], 0
        for i, (s, c) in enumerate(zip(seqs, counts)):
            p = partly[i]
            listed = [j for j, o in enumerate(partly) if o == p]
            copy = p is not None and refs[p] > 1 and not (len(listed) == refs[p] and listed[-1] == i)
            grown = -(-(self.lens[s] + c) // self.page) - len(self.held[s])
            plan.append((copy, free[k:k + copy + grown]))
            k += copy + grown
        if k > len(free):
            return False
        for (copy, new), s, c, p in zip(plan, seqs, counts, partly):
            if copy:
                n = self.lens[s] % self.page
                self.pages[new[0], ..., :n, :] = self.pages[p, ..., :n, :]
                self.held[s][-1] = new[0]
                new = new[1:]
            self.held[s] += new
            self.lens[s] += c
        return True

    def append(self, layer, k, v, seqs, counts):
        row = 0
        for s, c in zip(seqs, counts):
            for j in range(c):
                pos = self.lens[s] - c + j
                to = self.pages[self.held[s][pos // self.page], layer, :, :, pos % self.page]
                to.zero_()
                to[0, :, :k.shape[-1]] = k[row]
                to[1, :, :k.shape[-1]] = v[row]
                row += 1

    def truncate(self, seqs, drop):
        for s, n in zip(seqs, drop):
            self.lens[s] -= n
            del self.held[s][-(-self.lens[s] // self.page):]

    def compact(self):
        refs = self.refs
        used = sum(1 for n in refs if n)
        holes = [p for p in range(used) if not refs[p]]
        goes = dict(zip([p for p in range(used, len(refs)) if refs[p]], holes))
        for a, b in goes.items():
            self.pages[b] = self.pages[a]
        self.held = [[goes.get(p, p) for p in row] for row in self.held]

    def table(self, max_pages):
        return [row + [-1] * (max_pages - len(row)) for row in self.held]


def attend(q, k, v, count, scale, kind):
    """One sequence: q [count, n_q, dim], k and v [tokens, n_kv, dim] of 16-bit values.
    (out, its bound, lse, its bound), in 64 bits."""
    m, n_q, dim = q.shape
    length, n_kv = k.shape[0], k.shape[1]
    group = n_q // n_kv
    out = torch.zeros(m, n_q, dim, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((m, n_q), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    for j in range(m):
        n = length - m + 1 + j
        if n <= 0:
            continue
        for h in range(n_q):
            kk, vv, qq = k[:n, h // group].double(), v[:n, h // group].double(), q[j, h].double()
            s = scale * (kk @ qq)
            size = abs(scale) * (kk.abs() @ qq.abs())
            e = float((size * (dim / 8 + 64) * 2.0 ** -23 + 4 * s.abs() * 2.0 ** -24).max())
            top = s.max()
            w = torch.exp(s - top)
            total = w.sum()
            out[j, h] = w @ vv / total
            a = w @ vv.abs() / total
            sums = (n / 8 + 64) * 2.0 ** -22
            tol[j, h] = a * (2 * math.expm1(e) + 2.0 ** -20 + CUT[kind] + sums) + \
                ROUND[kind] * (out[j, h].abs() + a * (2 * math.expm1(e) + CUT[kind] + sums))
            if kind == "f16":
                tol[j, h] += 2.0 ** -32 * n * vv.abs().max() + 2.0 ** -25
            lse[j, h] = top + math.log(total)
            lse_tol[j, h] = e + 2.0 ** -21 + sums / 2 + 2.0 ** -22 * (lse[j, h].abs() + 1)
    return out, tol, lse, lse_tol


def units(x):
    """Probabilities (float32) in whole numbers of 2^-42, as Python integers."""
    out = []
    for f in x.tolist():
        if not f > 0:            # NaN, too
            out.append(0)
            continue
        y = min(f, 1.0) * 2.0 ** 42
        n = math.floor(y)
        rest = y - n             # exact: y is a float32 times a power of two
        out.append(n + (rest > 0.5 or (rest == 0.5 and n % 2 == 1)))
    return out


def accept(p, q, drafts, u, v):
    """One sequence: p [n + 1, vocab] (q likewise or None), n drafts and their u, v.
    (accepted, next token)."""
    n, vocab = p.shape[0] - 1, p.shape[1]
    a = 0
    while a < n:
        x = drafts[a]
        if not 0 <= x < vocab:
            break
        own = 1.0 if q is None else float(q[a, x])
        if not float(u[a]) * own < float(p[a, x]):
            break
        a += 1
    rest = p[a].clone()
    if a < n and q is not None:
        rest = p[a] - q[a]
    elif a < n and 0 <= drafts[a] < vocab:
        rest[drafts[a]] = 0
    w = units(rest)
    if not sum(w):
        w = units(p[a])
    total = sum(w)
    if not total:
        return a, -1
    part = min(int(max(0.0, min(1.0, float(v))) * 2 ** 31), 2 ** 31 - 1)
    t = total * part >> 31
    up = 0
    for i, x in enumerate(w):
        up += x
        if up > t:
            return a, i
    raise AssertionError
