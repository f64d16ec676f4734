"""How a mixture-of-experts layer is launched: in one cluster or on every SM, the mark
that a wait which ran out leaves, workspaces, and calls that overlap in time."""
import ctypes
import threading

import pytest
import torch

import paper_2512_22492_gb300 as rr
from tests import _products as P

pytestmark = pytest.mark.gpu


def layer_of(seed, experts, hidden, inter, top_k, first=0, local=None):
    gen = torch.Generator().manual_seed(seed)
    local = experts if local is None else local
    router = P.grid_router(gen, experts, hidden, "bf16")
    w13 = (torch.randn(local, 2 * inter, hidden, generator=gen) * 0.05).bfloat16()
    w2 = (torch.randn(local, hidden, inter, generator=gen) * 0.05).bfloat16()
    return rr.MoeLayer(router.cuda(), w13.cuda(), w2.cuda(), top_k, first), router, w13, w2


def tokens_of(seed, n, hidden):
    return P.grid_tokens(torch.Generator().manual_seed(seed), n, hidden, "bf16").cuda()


class _KernelParams(ctypes.Structure):       # CUDA_KERNEL_NODE_PARAMS of the driver API
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3),
                ("shared", ctypes.c_uint), ("params", ctypes.c_void_p), ("extra", ctypes.c_void_p),
                ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def blocks_of(layer, tokens):
    """The thread blocks of a call's one kernel, from a capture of it."""
    cu = ctypes.CDLL("libcuda.so.1")
    x = torch.zeros(tokens, layer.hidden, dtype=layer.torch_dtype, device="cuda")
    out, ws = torch.empty_like(x), rr.MoeWorkspace(layer, tokens)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    handle, graph, n = ctypes.c_void_p(stream.cuda_stream), ctypes.c_void_p(), ctypes.c_size_t(8)
    assert cu.cuStreamBeginCapture_v2(handle, 2) == 0
    try:
        rr.rr_moe(layer, x, out, ws, stream=stream)
    finally:
        assert cu.cuStreamEndCapture(handle, ctypes.byref(graph)) == 0
    nodes = (ctypes.c_void_p * 8)()
    assert cu.cuGraphGetNodes(graph, nodes, ctypes.byref(n)) == 0 and n.value == 1
    p = _KernelParams()
    assert cu.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(nodes[0]), ctypes.byref(p)) == 0
    assert cu.cuGraphDestroy(graph) == 0
    return p.grid[0]


# experts, hidden, inter, local, top_k, tokens
@pytest.mark.parametrize("shape,one", [
    ((8, 128, 96, 8, 2, 1), True), ((8, 128, 96, 8, 2, 20), True),
    ((256, 4096, 48, 1, 8, 64), False),        # a 2 MB router, read for every 16 tokens
    ((512, 4096, 16, 2, 4, 1), False), ((512, 8192, 16, 1, 1, 8), False),
    ((16, 512, 512, 16, 4, 20), False)])
def test_one_cluster_or_every_sm(shape, one):
    """A layer runs in one cluster where all that its call reads is little: the
    router and the tokens count, too."""
    experts, hidden, inter, local, top_k, tokens = shape
    layer, router, w13, w2 = layer_of(3, experts, hidden, inter, top_k, 0, local)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert blocks_of(layer, tokens) in ((8, 16) if one else (sms,))
    x = tokens_of(tokens, tokens, hidden)
    ws, out = rr.MoeWorkspace(layer, tokens), torch.empty_like(x)
    rr.rr_moe(layer, x, out, ws)
    rr.rr_moe_check(layer, ws)
    ids, c = P.route(x.cpu(), router, top_k, True)
    P.check(out, *P.moe(x.cpu(), ids, c, w13.double(), w2.double(), 0, "bf16"))


@pytest.mark.parametrize("experts,hidden,inter,tokens", [(8, 128, 96, 1), (8, 128, 96, 20), (16, 512, 512, 20)])
def test_a_marked_workspace_runs_nothing(experts, hidden, inter, tokens):
    """After a wait that ran out, calls of every size leave their outputs alone until
    rr_moe_check has reported it."""
    layer, _, _, _ = layer_of(5, experts, hidden, inter, 2)
    x = tokens_of(5, tokens, hidden)
    ws, want = rr.MoeWorkspace(layer, tokens), torch.empty_like(x)
    rr.rr_moe(layer, x, want, ws)
    rr.rr_moe_check(layer, ws)
    ws.data[0] = 1                 # the mark of an earlier call
    out = torch.full_like(x, 5.0)
    ids = torch.full((tokens, 2), -7, dtype=torch.int32, device="cuda")
    for _ in range(2):
        rr.rr_moe(layer, x, out, ws, ids=ids)
    with pytest.raises(rr.RRError, match="RR_ECUDA"):
        rr.rr_moe_check(layer, ws)
    assert bool((out == 5).all()) and bool((ids == -7).all())
    rr.rr_moe(layer, x, out, ws)
    rr.rr_moe_check(layer, ws)
    assert torch.equal(out, want)


def test_a_workspace_is_ready_when_it_is_there():
    """Its zeros have been written when the constructor returns, so that the first call
    may be on any stream."""
    layer, _, _, _ = layer_of(7, 8, 128, 96, 2)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)             # about a tenth of a second
    ws = rr.MoeWorkspace(layer, 4)
    assert torch.cuda.current_stream().query()
    x, side = tokens_of(7, 4, 128), torch.cuda.Stream()
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    rr.rr_moe(layer, x, out, ws, stream=side)
    rr.rr_moe_check(layer, ws, side)


def product_of(seed, rows, cols):
    gen = torch.Generator("cuda").manual_seed(seed)
    q = rr.Quantized(rows, cols, 128)
    rr.rr_quantize(q, (torch.randn(rows, cols, device="cuda", generator=gen) * 0.05).bfloat16())
    return q


def test_layers_on_every_sm_at_once():
    """Layers that fill every SM, on two streams, beside products and quantisations on
    a third: the results of calls one after another, and no wait that runs out."""
    layer, _, _, _ = layer_of(11, 16, 512, 512, 4)
    xs = [tokens_of(n, n, 512) for n in (3, 20)]
    spaces = [rr.MoeWorkspace(layer, 20) for _ in xs]
    want = [torch.empty_like(x) for x in xs]
    for x, ws, w in zip(xs, spaces, want):
        rr.rr_moe(layer, x, w, ws)
        rr.rr_moe_check(layer, ws)
    assert blocks_of(layer, 3) == blocks_of(layer, 20) == torch.cuda.get_device_properties(0).multi_processor_count
    q = product_of(1, 6144, 4096)
    token = torch.randn(2, 4096, device="cuda").bfloat16()
    product = torch.empty(2, 6144, device="cuda")
    rr.rr_matvec(q, token, product)
    raw = (torch.randn(512, 512, device="cuda") * 0.05).bfloat16()
    small = rr.Quantized(512, 512, 64)
    rr.rr_quantize(small, raw)
    packed, again = small.data.clone(), rr.Quantized(512, 512, 64)
    outs = [[torch.full_like(w, 9.0) for _ in range(50)] for w in want]
    products = [torch.full_like(product, 9.0) for _ in range(50)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for s in streams:              # until every call is queued
        with torch.cuda.stream(s):
            torch.cuda._sleep(40_000_000)
    for i in range(50):
        for k in range(2):
            rr.rr_moe(layer, xs[k], outs[k][i], spaces[k], stream=streams[k])
        rr.rr_matvec(q, token, products[i], stream=streams[2])
        rr.rr_quantize(again, raw, stream=streams[2])
    torch.cuda.synchronize()
    for k in range(2):
        rr.rr_moe_check(layer, spaces[k])
        assert all(torch.equal(o, want[k]) for o in outs[k])
    assert all(torch.equal(p, product) for p in products) and torch.equal(again.data, packed)


@pytest.mark.parametrize("inter", [32, 512])
def test_layers_and_products_from_several_threads(inter):
    """Four host threads, each with its own stream, workspace and outputs (32: in one
    cluster; 512: on every SM)."""
    layer, _, _, _ = layer_of(13, 8, 512, inter, 2)
    q = product_of(2, 2048, 512)
    xs = [tokens_of(30 + n, n, 512) for n in (1, 2, 9, 20)]
    want = []
    for x in xs:
        ws, out, product = rr.MoeWorkspace(layer, 20), torch.empty_like(x), torch.empty(min(16, len(x)), 2048, device="cuda")
        rr.rr_moe(layer, x, out, ws)
        rr.rr_matvec(q, x[:16], product)
        rr.rr_moe_check(layer, ws)
        want.append((out, product))
    torch.cuda.synchronize()
    errors = []

    def work(k):
        try:
            stream, x = torch.cuda.Stream(), xs[k]
            ws, out, product = rr.MoeWorkspace(layer, 20), torch.empty_like(x), torch.empty_like(want[k][1])
            torch.cuda.current_stream().synchronize()
            for _ in range(40):
                with torch.cuda.stream(stream):
                    out.fill_(9.0)
                    product.fill_(9.0)
                rr.rr_moe(layer, x, out, ws, stream=stream)
                rr.rr_matvec(q, x[:16], product, stream=stream)
                stream.synchronize()
                assert torch.equal(out, want[k][0]) and torch.equal(product, want[k][1])
            rr.rr_moe_check(layer, ws, stream)
        except BaseException as e:
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
