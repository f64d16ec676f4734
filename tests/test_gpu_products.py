"""Quantisation, matrix-vector products and the mixture-of-experts layer on the
GPU, against plain restatements in 64 bits (tests/_products.py, which derives the
bounds)."""
import math

import numpy as np
import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


def weights(gen, shape, kind, std=0.05):
    return (torch.randn(shape, generator=gen) * std).to(P.TYPES[kind])


def quantized(w, group, kind, pair=False):
    """(Quantized of a CPU stack [count, rows, cols] or matrix, its values in 64 bits)."""
    stack = w if w.dim() == 3 else w.unsqueeze(0)
    q = rr.Quantized(stack.shape[1], stack.shape[2], group, kind, pair, stack.shape[0])
    q.data.fill_(0x5A)
    rr.rr_quantize(q, w.cuda())
    vals = torch.stack([P.values(*P.quantize(m, group), group) for m in stack])
    return q, vals if w.dim() == 3 else vals[0]


# ---------------------------------------------------------------------------
# Quantisation
# ---------------------------------------------------------------------------

SHAPES = [(1, 1, False), (16, 128, False), (17, 129, False), (3, 300, False), (33, 96, False),
          (70, 257, False), (2, 8, True), (50, 130, True), (16, 256, True), (6, 31, True)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pair", SHAPES)
def test_quantize_bytes(rows, cols, pair, kind, group):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    w = weights(gen, (rows, cols), kind)
    q, vals = quantized(w, group, kind, pair)
    codes, scales = P.quantize(w, group)
    want = P.pack(codes, scales, group, pair)
    assert np.array_equal(q.data.cpu().numpy(), want)
    out = torch.full((rows, cols), 7.0, device="cuda")
    rr.rr_dequantize(q, out)
    assert torch.equal(out.cpu().double(), vals)
    out = torch.full((rows, cols), 7.0, dtype=P.TYPES[kind], device="cuda")
    rr.rr_dequantize(q, out)
    assert torch.equal(out.cpu(), vals.to(P.TYPES[kind]))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_quantize_special_values(kind):
    t = P.TYPES[kind]
    tiny = torch.finfo(t).smallest_normal
    rows = [torch.zeros(128), torch.full((128,), -0.0), torch.full((128,), tiny),
            torch.full((128,), tiny / 64), torch.full((128,), torch.finfo(t).max),
            # Quotients of exactly m + 1/2: the scale is 3/2, 1 or 2^-5.
            torch.arange(128) % 15 * 0.75 - 5.25 + torch.eye(1, 128)[0] * 15.75,
            torch.arange(128) % 14 * 0.5 + torch.eye(1, 128)[0] * 7,
            (torch.arange(128) % 29 - 14) / 64]
    for bad in (math.inf, -math.inf, math.nan):
        v = torch.randn(128, generator=torch.Generator().manual_seed(3))
        v[77] = bad
        rows.append(v)
    w = torch.stack(rows).to(t)
    for group in (32, 64, 128):
        codes, scales = P.quantize(w, group)
        q = rr.Quantized(*w.shape, group, kind)
        rr.rr_quantize(q, w.cuda())
        assert_same_packed(q, P.pack(codes, scales, group, False), group)
        out = torch.empty(w.shape, device="cuda")
        rr.rr_dequantize(q, out)
        P.check(out, P.values(codes, scales, group), torch.zeros(w.shape, dtype=torch.float64))


def assert_same_packed(q, want, group):
    """Equal bytes, but for which NaN a scale is."""
    got = q.data.cpu().numpy().reshape(-1, 1024 + 4096 // group)
    want = want.reshape(got.shape)
    assert np.array_equal(got[:, :1024], want[:, :1024])
    t = q.torch_dtype
    a = torch.from_numpy(got[:, 1024:].copy().view(np.int16)).view(t).float()
    b = torch.from_numpy(want[:, 1024:].copy().view(np.int16)).view(t).float()
    assert torch.equal(a.nan_to_num(12345.0), b.nan_to_num(12345.0))
    assert torch.equal(torch.isnan(a), torch.isnan(b))


@pytest.mark.parametrize("offset,extra", [(0, 8), (0, 3), (1, 0), (8, 16), (5, 7)])
def test_quantize_strides_and_stacks(offset, extra):
    """Rows at any alignment, a stack of matrices, and nothing written beside them."""
    gen = torch.Generator().manual_seed(5)
    count, rows, cols = 3, 34, 200
    w = weights(gen, (count, rows, cols), "bf16")
    ld = cols + extra
    buf = torch.full((offset + count * rows * ld + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
    view = buf[offset:offset + count * rows * ld].view(count, rows, ld)[:, :, :cols]
    view.copy_(w)
    q = rr.Quantized(rows, cols, 64, "bf16", True, count)
    rr.rr_quantize(q, view)
    want = [P.pack(*P.quantize(m, 64), 64, True) for m in w]
    assert np.array_equal(q.data.cpu().numpy(), np.concatenate(want))
    assert np.array_equal(q.matrix(1).data.cpu().numpy(), want[1])
    for t in (torch.bfloat16, torch.float32):
        out = torch.full((offset + count * rows * ld + 8,), 9.0, dtype=t, device="cuda")
        rr.rr_dequantize(q, out[offset:offset + count * rows * ld].view(count, rows, ld)[:, :, :cols])
        vals = torch.stack([P.values(*P.quantize(m, 64), 64) for m in w])
        mark = out[offset:offset + count * rows * ld].view(count, rows, ld)
        assert torch.equal(mark[:, :, :cols].cpu(), vals.to(t))
        assert bool((mark[:, :, cols:] == 9).all()) and bool((out[:offset] == 9).all()) \
            and bool((out[-8:] == 9).all())


@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 121, 127, 128, 129, 135, 136, 137, 250, 255, 257])
@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4, 5, 6, 7])
def test_quantize_every_alignment(cols, offset):
    """Rows that begin at every 2-byte offset from 16 bytes, of lengths around a
    block's and a vector's; NaN beside the matrix is not read into it."""
    gen = torch.Generator().manual_seed(cols)
    rows, ld = 19, cols + offset % 3
    w = weights(gen, (rows, cols), "f16")
    store = torch.full((offset + rows * ld + 9,), math.nan, dtype=torch.float16, device="cuda")
    view = store[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(w)
    q = rr.Quantized(rows, cols, 32, "f16")
    rr.rr_quantize(q, view)
    codes, scales = P.quantize(w, 32)
    assert np.array_equal(q.data.cpu().numpy(), P.pack(codes, scales, 32, False))
    out = torch.full_like(store, 9.0)
    to = out[offset:offset + rows * ld].view(rows, ld)
    rr.rr_dequantize(q, to[:, :cols])
    assert torch.equal(to[:, :cols].cpu(), P.values(codes, scales, 32).half())
    assert bool((to[:, cols:] == 9).all()) and bool((out[:offset] == 9).all()) and bool((out[-9:] == 9).all())


def test_quantize_flat_destination_tensor():
    """A sync's destination tensors are flat."""
    w = weights(torch.Generator().manual_seed(8), (48, 160), "f16")
    q = rr.Quantized(48, 160, 32, "f16")
    rr.rr_quantize(q, w.flatten().cuda())
    assert np.array_equal(q.data.cpu().numpy(), P.pack(*P.quantize(w, 32), 32, False))


# ---------------------------------------------------------------------------
# Matrix-vector products
# ---------------------------------------------------------------------------

MATVEC = [(1, 1, False), (16, 128, False), (512, 256, False), (130, 1000, False), (33, 77, False),
          (2, 5, True), (200, 384, True), (1378, 257, False), (48, 5000, False), (64, 4096, True),
          (2500, 640, False)]


@pytest.mark.parametrize("tokens", [1, 2, 5, 8, 9, 16])
@pytest.mark.parametrize("kind,group", [("bf16", 32), ("bf16", 128), ("f16", 64), ("f16", 128)])
@pytest.mark.parametrize("rows,cols,pair", MATVEC)
def test_matvec(rows, cols, pair, kind, group, tokens):
    gen = torch.Generator().manual_seed(rows + cols + tokens)
    w = weights(gen, (rows, cols), kind)
    q = rr.Quantized(rows, cols, group, kind, pair)
    rr.rr_quantize(q, w.cuda())
    vals = torch.empty(rows, cols, device="cuda")
    rr.rr_dequantize(q, vals)              # exact, as the tests above show
    x = torch.randn(tokens, cols, generator=gen).to(P.TYPES[kind])
    n = rows // 2 if pair else rows
    for t, name in ((P.TYPES[kind], kind), (torch.float32, "f32")):
        out = torch.full((tokens + 2, n), 3.0, dtype=t, device="cuda")
        rr.rr_matvec(q, x.cuda(), out[1:-1])
        want, tol = P.matvec(vals.cpu().double(), x, pair, name)
        P.check(out[1:-1], want, tol)
        assert bool((out[0] == 3).all()) and bool((out[-1] == 3).all())


@pytest.mark.parametrize("offset,extra", [(0, 8), (3, 0), (0, 5), (1, 7)])
def test_matvec_strides(offset, extra):
    gen = torch.Generator().manual_seed(17)
    rows, cols, tokens = 100, 328, 11
    q, vals = quantized(weights(gen, (rows, cols), "bf16"), 64, "bf16")
    x = torch.randn(tokens, cols, generator=gen).to(torch.bfloat16)
    ld = cols + extra
    store = torch.full((offset + tokens * ld + 8,), math.nan, dtype=torch.bfloat16, device="cuda")
    view = store[offset:offset + tokens * ld].view(tokens, ld)[:, :cols]
    view.copy_(x)
    lo = rows + extra
    out = torch.full((offset + tokens * lo + 8,), 3.0, dtype=torch.bfloat16, device="cuda")
    to = out[offset:offset + tokens * lo].view(tokens, lo)
    rr.rr_matvec(q, view, to[:, :rows])
    P.check(to[:, :rows], *P.matvec(vals, x, False, "bf16"))
    assert bool((to[:, rows:] == 3).all()) and bool((out[:offset] == 3).all()) \
        and bool((out[-8:] == 3).all())


@pytest.mark.parametrize("rows,cols,tokens,pair", [(40, 1 << 18, 3, False), (34, (1 << 18) - 5, 2, True),
                                                   (50, 100000, 16, False), (3000, 30000, 13, True)])
def test_matvec_longest_rows(rows, cols, tokens, pair):
    """Rows whose tokens fit no block's shared memory, in clusters and in several launches."""
    gen = torch.Generator().manual_seed(rows)
    q = rr.Quantized(rows, cols, 128, "bf16", pair)
    rr.rr_quantize(q, weights(gen, (rows, cols), "bf16", 0.01).cuda())
    vals = torch.empty(rows, cols, device="cuda")
    rr.rr_dequantize(q, vals)
    x = torch.randn(tokens, cols, generator=gen).bfloat16()
    out = torch.empty(tokens, q.n_out, device="cuda")
    rr.rr_matvec(q, x.cuda(), out)
    P.check(out, *P.matvec(vals.cpu().double(), x, pair, "f32"))


def test_matvec_one_dimensional_and_none():
    gen = torch.Generator().manual_seed(2)
    q, vals = quantized(weights(gen, (40, 96), "f16"), 32, "f16")
    x = torch.randn(96, generator=gen).half()
    out = torch.empty(40, dtype=torch.float16, device="cuda")
    rr.rr_matvec(q, x.cuda(), out)
    want, tol = P.matvec(vals, x.unsqueeze(0), False, "f16")
    P.check(out, want[0], tol[0])
    rr.rr_matvec(q, torch.empty(0, 96, dtype=torch.float16, device="cuda"),
                 torch.empty(0, 40, dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_matvec_not_finite(kind):
    """Infinities and NaN in a token stay in that token, and follow the sums: an
    infinite element times a code of zero is NaN.  A matrix row with a scale of
    NaN is NaN in every token."""
    gen = torch.Generator().manual_seed(23)
    w = weights(gen, (40, 256), kind)
    w[5, 130] = math.inf
    q = rr.Quantized(40, 256, 128, kind)
    rr.rr_quantize(q, w.cuda())
    vals = P.values(*P.quantize(w, 128), 128)
    x = torch.randn(4, 256, generator=gen).to(P.TYPES[kind])
    x[1, 9] = math.inf
    x[2, 200] = math.nan
    out = torch.empty(4, 40, dtype=P.TYPES[kind], device="cuda")
    rr.rr_matvec(q, x.cuda(), out)
    want = torch.stack([(vals * v.double()).sum(1) for v in x])
    _, tol = P.matvec(vals.nan_to_num(0.0), x.double().nan_to_num(0.0, 0.0, 0.0), False, kind)
    P.check(out, want, tol)


def test_matvec_large_values():
    """Loud channels, and float16 sums past 65504 that come back to it or go to infinity."""
    gen = torch.Generator().manual_seed(29)
    w = weights(gen, (64, 512), "f16", 20.0)
    q, vals = quantized(w, 64, "f16")
    x = torch.randn(3, 512, generator=gen)
    x[:, 100] *= 500
    x[1] *= 100
    x[2] *= 10
    x = x.half()
    out = torch.empty(3, 64, device="cuda")
    rr.rr_matvec(q, x.cuda(), out)
    P.check(out, *P.matvec(vals, x, False, "f32"))
    half = torch.empty(3, 64, dtype=torch.float16, device="cuda")
    rr.rr_matvec(q, x.cuda(), half)
    assert torch.equal(half.cpu(), out.half().cpu())


def test_matvec_streams_and_repeats():
    """The same bits from every call, on a side stream and in a CUDA graph."""
    gen = torch.Generator().manual_seed(31)
    q, vals = quantized(weights(gen, (1000, 2048), "bf16"), 128, "bf16")
    x = torch.randn(6, 2048, generator=gen).to(torch.bfloat16).cuda()
    first = torch.empty(6, 1000, dtype=torch.bfloat16, device="cuda")
    rr.rr_matvec(q, x, first)
    outs = [torch.empty_like(first) for _ in range(20)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i, o in enumerate(outs):
        rr.rr_matvec(q, x, o, stream=side if i % 2 else None)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)
    graph = torch.cuda.CUDAGraph()
    got = torch.zeros_like(first)
    with torch.cuda.graph(graph):
        rr.rr_matvec(q, x, got)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, first)


# ---------------------------------------------------------------------------
# Mixture of experts
# ---------------------------------------------------------------------------

def layer_of(gen, experts, hidden, inter, kind, group, top_k, first=0, local=None, norm=True,
             router=None):
    """(MoeLayer, router, w13 and w2 in 64 bits)."""
    local = experts if local is None else local
    router = P.grid_router(gen, experts, hidden, kind) if router is None else router
    w13 = weights(gen, (local, 2 * inter, hidden), kind)
    w2 = weights(gen, (local, hidden, inter), kind)
    if group:
        a, v13 = quantized(w13, group, kind, True)
        b, v2 = quantized(w2, group, kind)
    else:
        a, v13, b, v2 = w13.cuda(), w13.double(), w2.cuda(), w2.double()
    return rr.MoeLayer(router.cuda(), a, b, top_k, first, norm), router, v13, v2


def run_moe(layer, x, ws=None, stream=None):
    n = x.shape[0]
    ws = rr.MoeWorkspace(layer, max(1, n)) if ws is None else ws
    out = torch.full((n, layer.hidden), 5.0, dtype=layer.torch_dtype, device="cuda")
    ids = torch.full((n, layer.top_k), -7, dtype=torch.int32, device="cuda")
    c = torch.full((n, layer.top_k), -7.0, device="cuda")
    rr.rr_moe(layer, x.cuda(), out, ws, ids=ids, weights=c, stream=stream)
    rr.rr_moe_check(layer, ws, stream)
    return out, ids, c


# experts, hidden, inter, tokens, top_k, first, local, group, kind, norm
MOE = [(8, 128, 96, 1, 2, 0, 8, 0, "bf16", True), (8, 128, 96, 5, 2, 0, 8, 32, "bf16", True),
       (8, 128, 96, 64, 2, 0, 8, 0, "f16", False), (1, 64, 32, 3, 1, 0, 1, 0, "bf16", True),
       (16, 256, 64, 9, 16, 0, 16, 0, "f16", True), (16, 256, 64, 17, 3, 4, 4, 64, "f16", True),
       (32, 200, 72, 33, 4, 8, 8, 0, "bf16", False), (6, 75, 41, 7, 2, 0, 6, 0, "bf16", True),
       (6, 75, 41, 7, 2, 0, 6, 32, "f16", True), (5, 130, 33, 20, 3, 1, 3, 0, "f16", True),
       (512, 64, 16, 11, 16, 0, 512, 0, "bf16", True), (64, 512, 128, 64, 8, 0, 64, 0, "bf16", True),
       (64, 512, 128, 64, 8, 0, 64, 128, "bf16", True), (16, 1000, 520, 4, 4, 8, 8, 128, "bf16", True),
       (4, 2304, 800, 2, 2, 0, 4, 0, "bf16", True), (3, 1, 1, 2, 2, 0, 3, 0, "bf16", True),
       (3, 1, 1, 2, 2, 0, 3, 64, "f16", True), (4, 5000, 24, 20, 2, 0, 4, 0, "f16", True),
       (8, 40, 2600, 40, 4, 0, 8, 0, "bf16", True), (2, 9, 300, 64, 2, 1, 1, 0, "f16", False)]


@pytest.mark.parametrize("experts,hidden,inter,tokens,top_k,first,local,group,kind,norm", MOE)
def test_moe(experts, hidden, inter, tokens, top_k, first, local, group, kind, norm):
    gen = torch.Generator().manual_seed(experts + hidden + tokens)
    layer, router, v13, v2 = layer_of(gen, experts, hidden, inter, kind, group, top_k, first,
                                      local, norm)
    x = P.grid_tokens(gen, tokens, hidden, kind)
    out, ids, c = run_moe(layer, x)
    want_ids, want_c = P.route(x, router, top_k, norm)
    assert torch.equal(ids.cpu().long(), want_ids)
    P.check(c, want_c, 2.0 ** -18 * want_c)
    P.check(out, *P.moe(x, want_ids, want_c, v13, v2, first, kind))


@pytest.mark.parametrize("hidden,inter,tokens,group,kind", [
    (32768, 24, 5, 0, "bf16"), (32761, 16, 9, 0, "f16"), (32768, 40, 20, 32, "bf16"),
    (64, 16384, 6, 0, "f16"), (33, 16381, 18, 0, "bf16"), (64, 16384, 3, 64, "bf16")])
def test_moe_longest_rows(hidden, inter, tokens, group, kind):
    """The longest rows that are accepted: a block's shared memory holds one token's."""
    gen = torch.Generator().manual_seed(hidden + inter)
    layer, router, v13, v2 = layer_of(gen, 3, hidden, inter, kind, group, 2)
    x = P.grid_tokens(gen, tokens, hidden, kind)
    out, ids, c = run_moe(layer, x)
    want_ids, want_c = P.route(x, router, 2, True)
    assert torch.equal(ids.cpu().long(), want_ids)
    P.check(out, *P.moe(x, want_ids, want_c, v13, v2, 0, kind))
    with pytest.raises(rr.RRError, match="RR_ELAYOUT"):
        rr.MoeLayer(torch.zeros(2, 32769, dtype=torch.bfloat16), torch.zeros(2, 2, 32769, dtype=torch.bfloat16),
                    torch.zeros(2, 32769, 1, dtype=torch.bfloat16), 1)


def test_moe_ties_and_empty_tokens():
    """Equal logits go to the lowest index; a token whose experts are all elsewhere
    gets zeros."""
    gen = torch.Generator().manual_seed(41)
    router = P.grid_router(gen, 12, 64, "bf16")
    router[7] = router[2]
    router[11] = router[2]
    router[3] = -router[9]
    layer, _, v13, v2 = layer_of(gen, 12, 64, 32, "bf16", 0, 4, 2, 3, True, router)
    x = P.grid_tokens(gen, 30, 64, "bf16")
    x[4] = 0                       # every logit equal: experts 0..3
    out, ids, c = run_moe(layer, x)
    want_ids, want_c = P.route(x, router, 4, True)
    assert ids[4].tolist() == [0, 1, 2, 3] and torch.equal(ids.cpu().long(), want_ids)
    P.check(out, *P.moe(x, want_ids, want_c, v13, v2, 2, "bf16"))
    layer, _, v13, v2 = layer_of(gen, 12, 64, 32, "bf16", 0, 1, 5, 1, True, router)
    out, ids, c = run_moe(layer, x)
    empty = ids[:, 0].cpu() != 5
    assert bool(empty.any()) and bool((out.cpu()[empty] == 0).all())


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("tokens", [1, 16, 63])
def test_moe_all_tokens_on_one_expert(tokens, group):
    gen = torch.Generator().manual_seed(43)
    router = P.grid_router(gen, 16, 128, "bf16")
    router[9] = 0.25
    layer, _, v13, v2 = layer_of(gen, 16, 128, 64, "bf16", group, 1, 0, 16, False, router)
    x = P.grid_tokens(gen, tokens, 128, "bf16").abs()
    out, ids, c = run_moe(layer, x)
    assert bool((ids == 9).all())
    want_ids, want_c = P.route(x, router, 1, False)
    P.check(out, *P.moe(x, want_ids, want_c, v13, v2, 0, "bf16"))


def test_moe_not_finite():
    """A bad token stays to itself; its output is NaN and its experts are the first."""
    gen = torch.Generator().manual_seed(47)
    layer, router, v13, v2 = layer_of(gen, 8, 96, 40, "bf16", 0, 3)
    x = P.grid_tokens(gen, 6, 96, "bf16")
    good, ids_good, _ = run_moe(layer, x)
    bad = x.clone()
    bad[2, 50] = math.nan
    out, ids, c = run_moe(layer, bad)
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(out[keep], good[keep]) and torch.equal(ids[keep], ids_good[keep])
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(c[2]).all())
    assert ids[2].tolist() == [0, 1, 2]


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("tokens", [1, 3, 8, 20])
def test_moe_bad_expert(tokens, group):
    """An expert whose weights are not finite is felt by the tokens that chose it alone."""
    gen = torch.Generator().manual_seed(51)
    router = P.grid_router(gen, 8, 96, "bf16")
    w13, w2 = weights(gen, (8, 96, 96), "bf16"), weights(gen, (8, 96, 48), "bf16")
    x = P.grid_tokens(gen, tokens, 96, "bf16")
    ids, _ = P.route(x, router, 2, True)
    bad = int(ids[0, 0])
    outs = []
    for spoil in (False, True):
        if spoil:
            w2[bad] = math.nan
            w13[bad, 5] = math.inf
        a, b = (quantized(w13, group, "bf16", True)[0], quantized(w2, group, "bf16")[0]) if group \
            else (w13.cuda(), w2.cuda())
        outs.append(run_moe(rr.MoeLayer(router.cuda(), a, b, 2), x)[0].cpu())
    hit = (ids == bad).any(1)
    assert bool(torch.isnan(outs[1][hit]).all()) and bool(hit[0])
    assert torch.equal(outs[0][~hit], outs[1][~hit])
    assert tokens == 1 or bool((~hit).any())


def test_moe_large_hidden_values_f16():
    """silu(gate) * up past float16's range, and far below it, is held in 32 bits."""
    gen = torch.Generator().manual_seed(53)
    hidden, inter = 64, 48
    router = P.grid_router(gen, 4, hidden, "f16")
    w13 = weights(gen, (4, 2 * inter, hidden), "f16", 40.0)
    w13[1] = w13[1] / 4096
    w2 = weights(gen, (4, hidden, inter), "f16", 1e-3)
    layer = rr.MoeLayer(router.cuda(), w13.cuda(), w2.cuda(), 2)
    x = P.grid_tokens(gen, 9, hidden, "f16")
    ids, c = P.route(x, router, 2, True)
    h = torch.stack([P.silu(w13[e, :inter].double() @ x[0].double())
                     * (w13[e, inter:].double() @ x[0].double()) for e in range(4)])
    assert h.abs().max() > 65504
    out, got_ids, _ = run_moe(layer, x)
    assert torch.equal(got_ids.cpu().long(), ids)
    P.check(out, *P.moe(x, ids, c, w13.double(), w2.double(), 0, "f16"))


@pytest.mark.parametrize("group", [0, 32])
def test_moe_strides_and_reused_workspace(group):
    """Token rows at any alignment; one workspace for many calls of many sizes; the
    same bits each time; optional outputs left out; nothing written beside out."""
    gen = torch.Generator().manual_seed(59)
    layer, router, v13, v2 = layer_of(gen, 32, 176, 80, "bf16", group, 4)
    ws = rr.MoeWorkspace(layer, 64)
    seen = {}
    for n in (64, 1, 7, 33, 1, 64, 2, 7):
        x = P.grid_tokens(torch.Generator().manual_seed(n), n, 176, "bf16")
        store = torch.full((3 + n * 181,), math.nan, dtype=torch.bfloat16, device="cuda")
        view = store[3:].view(n, 181)[:, :176]
        view.copy_(x)
        out = torch.full((1 + n * 179,), 5.0, dtype=torch.bfloat16, device="cuda")
        to = out[1:].view(n, 179)
        rr.rr_moe(layer, view, to[:, :176], ws)
        assert bool((to[:, 176:] == 5).all()) and out[0].item() == 5
        got = to[:, :176].clone()
        if n in seen:
            assert torch.equal(seen[n], got)
        else:
            seen[n] = got
            ids, c = P.route(x, router, 4, True)
            P.check(got, *P.moe(x, ids, c, v13, v2, 0, "bf16"))
    rr.rr_moe(layer, torch.empty(0, 176, dtype=torch.bfloat16, device="cuda"),
              torch.empty(0, 176, dtype=torch.bfloat16, device="cuda"), ws)
    rr.rr_moe_check(layer, ws)


def test_moe_streams_and_graph():
    """Two streams with a workspace each, and replays of a captured call."""
    gen = torch.Generator().manual_seed(61)
    layer, router, v13, v2 = layer_of(gen, 16, 256, 128, "bf16", 0, 4)
    xs = [P.grid_tokens(gen, n, 256, "bf16").cuda() for n in (3, 20)]
    want = [run_moe(layer, x)[0] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    spaces = [rr.MoeWorkspace(layer, 20) for _ in xs]
    outs = [[torch.empty_like(w) for _ in range(30)] for w in want]
    torch.cuda.synchronize()
    for i in range(30):
        for k in range(2):
            rr.rr_moe(layer, xs[k], outs[k][i], spaces[k], stream=streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        rr.rr_moe_check(layer, spaces[k])
        for o in outs[k]:
            assert torch.equal(o, want[k])
    graph = torch.cuda.CUDAGraph()
    got = torch.zeros_like(want[1])
    x = xs[1].clone()
    with torch.cuda.graph(graph):
        rr.rr_moe(layer, x, got, spaces[1])
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[1])


def test_moe_a_wait_that_runs_out():
    """A count that can never be reached makes the blocks' wait run out (about two
    seconds): the call ends, rr_moe_check says so, and after it the workspace works
    again; until then calls on it do nothing."""
    gen = torch.Generator().manual_seed(71)
    layer, router, v13, v2 = layer_of(gen, 16, 512, 512, "bf16", 0, 4)
    x = P.grid_tokens(gen, 20, 512, "bf16")
    ws = rr.MoeWorkspace(layer, 20)
    want, _, _ = run_moe(layer, x, ws)
    # The count wraps round to below the number of blocks.
    ws.data[4:8] = torch.tensor([0xCD, 0xFF, 0xFF, 0xFF], dtype=torch.uint8, device="cuda")
    out = torch.empty_like(want)
    rr.rr_moe(layer, x.cuda(), out, ws)
    with pytest.raises(rr.RRError, match="RR_ECUDA"):
        rr.rr_moe_check(layer, ws)
    got, _, _ = run_moe(layer, x, ws)
    assert torch.equal(got, want)
    ws.data[0] = 1                 # an earlier call's mark
    out.fill_(5.0)
    rr.rr_moe(layer, x.cuda(), out, ws)
    with pytest.raises(rr.RRError, match="RR_ECUDA"):
        rr.rr_moe_check(layer, ws)
    assert bool((out == 5).all())
    got, _, _ = run_moe(layer, x, ws)
    assert torch.equal(got, want)


def test_offsets_past_32_bits():
    """Matrices of more than 2^31 elements: their last rows, and a stack's last expert."""
    gen = torch.Generator().manual_seed(73)
    rows, cols = 70000, 32768
    w = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = weights(gen, (48, cols), "bf16").cuda()
    w[-48:] = tail
    q = rr.Quantized(rows, cols, 128)
    rr.rr_quantize(q, w)
    small = rr.Quantized(48, cols, 128)
    rr.rr_quantize(small, tail)
    assert torch.equal(q.data[-small.nbytes:], small.data)
    x = torch.randn(3, cols, generator=gen).bfloat16().cuda()
    out, few = torch.empty(3, rows, device="cuda"), torch.empty(3, 48, device="cuda")
    rr.rr_matvec(q, x, out)
    rr.rr_matvec(small, x, few)
    vals = torch.empty(48, cols, device="cuda")
    rr.rr_dequantize(small, vals)
    want, tol = P.matvec(vals.cpu().double(), x.cpu(), False, "f32")
    P.check(few, want, tol)
    P.check(out[:, -48:], want, tol)
    assert bool((out[:, :-48] == 0).all())
    w.fill_(7.0)
    rr.rr_dequantize(q, w)
    back = torch.empty_like(tail)
    rr.rr_dequantize(small, back)
    assert torch.equal(w[-48:], back) and bool((w[:-48] == 0).all())
    del w, q, out
    experts, hidden, inter = 64, 8192, 2304
    router = P.grid_router(gen, experts, hidden, "bf16")
    router[experts - 1] = 0.25
    w13 = torch.zeros(experts, 2 * inter, hidden, dtype=torch.bfloat16, device="cuda")
    w2 = torch.zeros(experts, hidden, inter, dtype=torch.bfloat16, device="cuda")
    one13, one2 = weights(gen, (2 * inter, hidden), "bf16", 0.02), weights(gen, (hidden, inter), "bf16", 0.02)
    w13[-1], w2[-1] = one13.cuda(), one2.cuda()
    x = P.grid_tokens(gen, 2, hidden, "bf16").abs()
    layer = rr.MoeLayer(router.cuda(), w13, w2, 1)
    out, ids, c = run_moe(layer, x)
    assert bool((ids == experts - 1).all())
    zeros = torch.zeros(2, 1, dtype=torch.int64)
    P.check(out, *P.moe(x, zeros, torch.ones(2, 1, dtype=torch.float64), one13.unsqueeze(0).double(),
                        one2.unsqueeze(0).double(), 0, "bf16"))


# ---------------------------------------------------------------------------
# Refusals
# ---------------------------------------------------------------------------

def test_refusals_on_the_gpu():
    gen = torch.Generator().manual_seed(67)
    q, _ = quantized(weights(gen, (32, 128), "bf16"), 64, "bf16")
    x = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.full((2, 32), 3.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(rr.RRError, match="RR_EINVAL"):
        rr.rr_matvec(q, x.cpu(), out)
    with pytest.raises(rr.RRError, match="RR_EINVAL"):
        rr.rr_matvec(q, torch.zeros(17, 128, dtype=torch.bfloat16, device="cuda"),
                     torch.zeros(17, 32, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(rr.RRError, match="16-byte"):
        rr.rr_matvec(rr.Quantized(16, 128, data=torch.zeros(1064, dtype=torch.uint8,
                                                            device="cuda")[8:]),
                     x, torch.zeros(2, 16, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(rr.RRError, match="RR_EINVAL"):
        rr.rr_quantize(q, torch.zeros(32, 128, dtype=torch.bfloat16))
    stack = rr.Quantized(16, 128, count=2)
    with pytest.raises(rr.RRError, match="one matrix"):
        rr.rr_matvec(stack, x, torch.zeros(2, 16, dtype=torch.bfloat16, device="cuda"))
    layer, _, _, _ = layer_of(gen, 4, 64, 32, "bf16", 0, 2)
    ws = rr.MoeWorkspace(layer, 4)
    x = torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(rr.RRError, match="workspace"):
        rr.rr_moe(layer, x, torch.empty_like(x), ws)
    big = torch.zeros(65, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(rr.RRError, match="tokens"):
        rr.rr_moe(layer, big, torch.empty_like(big), ws)
    assert bool((out == 3).all())
