"""Products of the rollout's weights: sizes and refusals (no GPU), and the tests'
own restatement held against hand-worked numbers."""
import math

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P


def mem(n):
    return torch.zeros(n, dtype=torch.uint8)


@pytest.mark.parametrize("rows,cols,group,pair,count,want", [
    (16, 128, 128, False, 1, 1056), (17, 129, 32, False, 1, 4 * 1152), (1, 1, 64, False, 3, 3 * 1088),
    (16, 128, 128, True, 1, 1056), (18, 128, 128, True, 1, 2 * 1056),
    (151936, 4096, 128, False, 1, 9496 * 32 * 1056)])
def test_packed_sizes(rows, cols, group, pair, count, want):
    import ctypes
    from paper_2512_22492_gb300.products import _Quant
    from paper_2512_22492_gb300.rr import _lib
    c = _Quant(rows, cols, count, group, 0, int(pair))
    one, total = ctypes.c_int64(), ctypes.c_int64()
    assert _lib.rr_quant_bytes(ctypes.byref(c), ctypes.byref(one), ctypes.byref(total)) == 0
    assert total.value == want and one.value * count == want and one.value % 16 == 0


@pytest.mark.parametrize("kw", [dict(rows=0), dict(cols=0), dict(rows=-5), dict(cols=(1 << 24) + 1),
                                dict(rows=1 << 31), dict(group=16), dict(group=256), dict(group=0),
                                dict(count=0), dict(count=65536), dict(rows=15, pair=True)])
def test_shapes_refused(kw):
    args = dict(rows=16, cols=128, group=128, count=1, pair=False)
    args.update(kw)
    with pytest.raises(rr.RRError, match="RR_ELAYOUT"):
        rr.Quantized(data=mem(16), **args)


def test_bad_tensors_refused():
    q = rr.Quantized(32, 128, 64, "bf16", data=mem(2 * 1088))
    bf = torch.bfloat16
    with pytest.raises(ValueError):
        rr.Quantized(32, 128, 64, "f32", data=mem(2 * 1088))
    with pytest.raises(ValueError):
        rr.Quantized(32, 128, 64, "bf16", data=mem(2 * 1088 - 1))
    with pytest.raises(IndexError):
        q.matrix(1)
    for bad in (torch.zeros(32, 128), torch.zeros(32, 127, dtype=bf), torch.zeros(128, 32, dtype=bf).T,
                torch.zeros(4095, dtype=bf), torch.zeros(2, 32, 128, dtype=bf),
                torch.zeros(1, 128, dtype=bf).expand(32, 128)):
        with pytest.raises(ValueError):
            rr.rr_quantize(q, bad, stream=0)
    x, out = torch.zeros(3, 128, dtype=bf), torch.zeros(3, 32, dtype=bf)
    for a, b in ((x.float(), out), (x[:, :127], out), (x, out[:2]), (x, out.half()),
                 (x, torch.zeros(3, 31, dtype=bf)), (torch.zeros(128, 3, dtype=bf).T, out),
                 (x, torch.zeros(1, 32, dtype=bf).expand(3, 32))):
        with pytest.raises(ValueError):
            rr.rr_matvec(q, a, b, stream=0)


def test_layers_refused():
    bf = torch.bfloat16
    router, w13, w2 = torch.zeros(4, 32, dtype=bf), torch.zeros(4, 48, 32, dtype=bf), torch.zeros(4, 32, 24, dtype=bf)
    layer = rr.MoeLayer(router, w13, w2, 2)
    assert (layer.n_experts, layer.n_local, layer.hidden, layer.inter) == (4, 4, 32, 24)
    for kw in (dict(top_k=0), dict(top_k=5), dict(top_k=2, first_expert=1), dict(top_k=2, first_expert=-1)):
        with pytest.raises(rr.RRError, match="RR_ELAYOUT"):
            rr.MoeLayer(router, w13, w2, **kw)
    q13 = rr.Quantized(48, 32, 64, pair=True, count=4, data=mem(4 * 3 * 1088))
    q2 = rr.Quantized(32, 24, 64, count=4, data=mem(4 * 2 * 1088))
    assert rr.MoeLayer(router, q13, q2, 2).inter == 24
    unpaired = rr.Quantized(48, 32, 64, count=4, data=mem(4 * 3 * 1088))
    other = rr.Quantized(32, 24, 32, count=4, data=mem(4 * 2 * 1152))
    for a, b in ((w13, q2), (q13, w2), (unpaired, q2), (q13, other), (w13[:, :47], w2), (w13, w2[:3]),
                 (w13.half(), w2), (w13.transpose(1, 2).contiguous(), w2),
                 (torch.zeros(4, 48, 64, dtype=bf)[:, :, :32], w2)):
        with pytest.raises(ValueError):
            rr.MoeLayer(router, a, b, 2)
    with pytest.raises(rr.RRError):
        rr.MoeLayer(torch.zeros(513, 8, dtype=bf), torch.zeros(1, 16, 8, dtype=bf),
                    torch.zeros(1, 8, 8, dtype=bf), 1)
    for n in (0, 65):
        with pytest.raises(rr.RRError, match="tokens"):
            rr.MoeWorkspace(layer, n)


def test_restatement_by_hand():
    """Scales and codes worked out by hand: a group of 32 with maximum 3.5 has the
    scale 0.5, and 0.25 / 0.5 = 0.5 rounds to the even 0, 0.75 / 0.5 = 1.5 to 2."""
    w = torch.zeros(1, 40, dtype=torch.bfloat16)
    w[0, :5] = torch.tensor([3.5, -3.5, 0.25, 0.75, -1.0])
    w[0, 32:36] = torch.tensor([7.0, 1.0, -2.5, 0.0])
    q, s = P.quantize(w, 32)
    assert s.tolist() == [[0.5, 1.0]]
    assert q[0, :5].tolist() == [7, -7, 0, 2, -2] and q[0, 32:36].tolist() == [7, 1, -2, 0]
    assert P.values(q, s, 32)[0, :5].tolist() == [3.5, -3.5, 0.0, 1.0, -1.0]
    b = P.pack(q, s, 32, False)
    assert b.size == 1152
    # Columns 0..7 of row 0: word 0 of lane 0; codes 15, 1, 8, 10, 6, 8, 8, 8 with
    # even columns in the low half, odd ones in the high half.
    assert b[:4].tobytes().hex() == bytes([0x8F, 0x86, 0xA1, 0x88]).hex()
    # Scales 0.5 and 1.0 in bfloat16, of slot 0, then of slot 8 (zero): interleaved.
    assert b[1024:1032].tobytes().hex() == "003f0000803f0000"
    ids, c = P.route(torch.tensor([[1.0]]), torch.tensor([[0.0], [math.log(3.0)], [0.0]]), 2, True)
    assert ids.tolist() == [[1, 0]] and torch.allclose(c, torch.tensor([[0.75, 0.25]], dtype=torch.float64))
