"""The values between a layer's two expert products, h = silu(gate) * up, enter
the second product as float32.

The layers are built so that every sum on the way is a float32 number, in any
order: gate is 28 * 2^k (silu leaves it as it is: exp(-28) is under 2^-24), up is
7/4 + b 2^-8 + c 2^-16 times 2^k with b and c multiples of 1/4 up to 7/4, so h has
22 bits; a row of w2 takes the difference of two adjacent h with the same b, times
7/8.  In 4 bits these weights are exact as well: each group's largest is 7 times
a power of two.  The output is the 16-bit type's nearest number to
7/8 * 28 * 2^(2 k - 16) (c - c')."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr

pytestmark = pytest.mark.gpu


def layer_of(w13, w2, group):
    """A layer of one expert, which every token takes with weight 1."""
    hidden, inter = w2.shape
    router = torch.zeros(1, hidden, dtype=w2.dtype, device="cuda")
    a, b = w13.unsqueeze(0).cuda(), w2.unsqueeze(0).cuda()
    if group:
        kind = "bf16" if w2.dtype == torch.bfloat16 else "f16"
        qa = rr.Quantized(2 * inter, hidden, group, kind, True)
        qb = rr.Quantized(hidden, inter, group, kind)
        rr.rr_quantize(qa, a)
        rr.rr_quantize(qb, b)
        a, b = qa, qb
    return rr.MoeLayer(router, a, b, 1)


def run(layer, x):
    ws = rr.MoeWorkspace(layer, x.shape[0])
    out = torch.full_like(x, 5.0)
    rr.rr_moe(layer, x, out, ws)
    rr.rr_moe_check(layer, ws)
    return out.cpu()


def exact_case(hidden, inter, tokens, dtype):
    gen = torch.Generator().manual_seed(hidden + inter + tokens)
    b = torch.randint(-7, 8, (inter,), generator=gen) / 4
    b[1::4] = b[0::4][:b[1::4].numel()]
    c = torch.randint(-7, 8, (inter,), generator=gen) / 4
    w13 = torch.zeros(2 * inter, hidden)
    w13[:inter, 0] = 28.0
    w13[inter:, 0] = 1.75
    w13[inter:, 1] = b
    w13[inter:, 2] = c
    w2 = torch.zeros(hidden, inter)
    m = 4 * (torch.arange(hidden) % ((inter + 2) // 4))
    w2[torch.arange(hidden), m] = 0.875
    w2[torch.arange(hidden), m + 1] = -0.875
    k = torch.arange(tokens) % 3
    x = torch.zeros(tokens, hidden)
    for i in range(3):
        x[:, i] = 2.0 ** (k - 8 * i)
    want = (0.875 * 28 * 2.0 ** -16) * torch.outer(4.0 ** k.double(), (c[m] - c[m + 1]).double())
    return w13.to(dtype), w2.to(dtype), x.to(dtype).cuda(), want.to(dtype)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("hidden,inter,tokens", [
    (64, 48, 1), (64, 48, 8), (64, 48, 20), (67, 42, 3), (67, 42, 17), (160, 1030, 1), (160, 1030, 30),
    (2048, 768, 1), (2048, 768, 40), (72, 16382, 2), (64, 8192, 40)])
def test_differences_of_hidden_values(hidden, inter, tokens, group):
    w13, w2, x, want = exact_case(hidden, inter, tokens, torch.bfloat16)
    got = run(layer_of(w13, w2, group), x)
    assert torch.equal(got, want)


@pytest.mark.parametrize("inter", [48, 45, 16384])
@pytest.mark.parametrize("tokens", [1, 9])
def test_hidden_values_at_the_top_of_float32(tokens, inter):
    """Finite in float32, past the largest bfloat16, and infinite ones: a row of w2
    that has one column of each kind gets its sign and no NaN."""
    hidden = 40
    w13 = torch.zeros(2 * inter, hidden)
    w13[:inter, 0] = 28.0
    w13[inter:, 0] = 1.140625
    w13[inter:, 1] = 0.25
    x = torch.zeros(tokens, hidden)
    x[:, 0], x[:, 1] = 2.0 ** 61, 2.0 ** 53
    # 56 * 2^61 * (1.140625 + 2^-10) * 2^61 = 0.9989 * 2^128.
    w13[:inter, 0] *= 2
    w2 = torch.zeros(hidden, inter)
    w2[:, 7] = 2.0 ** -10
    h = 56 * 2.0 ** 61 * (1.140625 + 2.0 ** -10) * 2.0 ** 61
    assert torch.finfo(torch.bfloat16).max * (1 + 2.0 ** -9) < h < torch.finfo(torch.float32).max
    got = run(layer_of(w13.bfloat16(), w2.bfloat16(), 0), x.bfloat16().cuda())
    want = torch.full_like(got, h * 2.0 ** -10)
    assert torch.equal(got, want)
    # Column 20's h is infinite: 8 times as large.
    w13[20, 0] *= 8
    w2[:, 20] = 0.5
    w2[::2, 20] = -0.5
    got = run(layer_of(w13.bfloat16(), w2.bfloat16(), 0), x.bfloat16().cuda())
    want = torch.full_like(got, math.inf)
    want[:, ::2] = -math.inf
    assert torch.equal(got, want)


@pytest.mark.parametrize("tokens", [1, 9])
def test_not_a_number_among_hidden_values(tokens):
    """A NaN in one column of h is NaN in every output; with weights of zero, too."""
    w13, w2, x, _ = exact_case(64, 48, tokens, torch.bfloat16)
    w13[30, 0] = math.nan
    assert bool(torch.isnan(run(layer_of(w13, w2, 0), x)).all())
