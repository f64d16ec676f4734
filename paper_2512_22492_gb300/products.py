"""Products of the rollout's weights: the binding of that part of include/rr.h.

After a sync, a rollout quantises the matrices it serves from (``rr_quantize``:
4 bits with group scales) and runs its token step's products on them:
``rr_matvec`` and, for a mixture-of-experts layer, ``rr_moe`` on the stacked
experts (as ``rr_unpack`` writes them, or quantised).  As in ``rr.py``, every
step runs in the CUDA library; this module checks and marshals arguments.
Descriptions are marshalled once, in ``Quantized``, ``MoeLayer`` and
``MoeWorkspace``; a call then checks its own tensors only.
"""
from __future__ import annotations

import ctypes

from .rr import RR_OK, _check, _DST_DTYPES, _lib, _sig, _stream, _vp

RR_MATVEC_MAX_TOKENS = 16
RR_MOE_MAX_TOKENS = 64

_i32, _i64 = ctypes.c_int32, ctypes.c_int64


class _Quant(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("count", _i32), ("group", _i32),
                ("dtype", _i32), ("pair", _i32)]


class _Moe(ctypes.Structure):
    _fields_ = [("n_experts", _i32), ("first_expert", _i32), ("n_local", _i32), ("top_k", _i32),
                ("hidden", _i64), ("inter", _i64), ("dtype", _i32), ("group", _i32),
                ("norm_topk", _i32), ("reserved", _i32)]


_PQ, _PM, _P64 = ctypes.POINTER(_Quant), ctypes.POINTER(_Moe), ctypes.POINTER(_i64)

_sig("rr_quant_bytes", [_PQ, _P64, _P64])
_sig("rr_quantize", [_PQ, _vp, _i64, _vp, _vp])
_sig("rr_dequantize", [_PQ, _vp, _vp, _i64, _i32, _vp])
_sig("rr_matvec", [_PQ, _vp, _vp, _i64, _i32, _vp, _i64, _i32, _vp])
_sig("rr_moe_workspace", [_PM, _i32, _P64])
_sig("rr_moe", [_PM, _vp, _vp, _vp, _vp, _i64, _i32, _vp, _i64, _vp, _vp, _vp, _i64, _vp])
_sig("rr_moe_check", [_PM, _i32, _vp, _vp])


def _type_name(torch_dtype) -> str:
    import torch
    for name, t in (("bf16", torch.bfloat16), ("f16", torch.float16)):
        if torch_dtype == t:
            return name
    raise ValueError(f"elements must be bfloat16 or float16, not {torch_dtype}")


def _torch_type(name: str):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def _rows(x, cols: int, dtype, what: str):
    """(rows, row stride) of a token tensor [rows, cols] (or [cols]) of `dtype`."""
    if x.dtype is not dtype:
        raise ValueError(f"{what}: elements of {x.dtype}, expected {dtype}")
    dim = x.dim()
    if dim == 2 and x.size(1) == cols:
        n = x.size(0)
        if x.is_contiguous():
            return n, cols
        ld = x.stride(0) if n > 1 else cols
        if ld < cols:
            raise ValueError(f"{what}: rows overlap")
    elif dim == 1 and x.size(0) == cols:
        n, ld = 1, cols
    else:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected [n, {cols}]")
    if cols > 1 and x.stride(-1) != 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    return n, ld


_raw_stream = None


def _stream_of(x, stream) -> int:
    """The stream's handle; None: the current one of x's device."""
    global _raw_stream
    if stream is not None or not x.is_cuda:
        return _stream(stream)
    if _raw_stream is None:
        # The call that torch's own code generators use; it is not public.
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda device: int(torch.cuda.current_stream(device).cuda_stream))
    return _raw_stream(x.get_device())


class Quantized:
    """A stack of `count` matrices [rows, cols] in 4 bits with group scales.

    pair: the rows are [gate; up], as a fused gate_up_proj or an expert's w13.
    `data`: the packed bytes (a contiguous uint8 device tensor of ``nbytes``);
    allocated on the current device if not given.  ``matrix_bytes`` is one
    matrix's share of them; ``matrix(i)`` is matrix i of the stack, on the same
    memory."""

    def __init__(self, rows: int, cols: int, group: int = 128, dtype: str = "bf16",
                 pair: bool = False, count: int = 1, data=None):
        if dtype not in _DST_DTYPES:
            raise ValueError(f"dtype must be one of {sorted(_DST_DTYPES)}, not {dtype!r}")
        self._c = _Quant(rows, cols, count, group, _DST_DTYPES[dtype], int(pair))
        self._ref = ctypes.byref(self._c)
        one, total = _i64(), _i64()
        _check(_lib.rr_quant_bytes(self._ref, ctypes.byref(one), ctypes.byref(total)),
               "rr_quant_bytes")
        self.rows, self.cols, self.group, self.count = rows, cols, group, count
        self.dtype, self.pair = dtype, bool(pair)
        self.torch_dtype = _torch_type(dtype)
        self.n_out = rows // 2 if pair else rows
        self.matrix_bytes, self.nbytes = one.value, total.value
        if data is None:
            import torch
            data = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")
        if data.numel() * data.element_size() < self.nbytes or not data.is_contiguous():
            raise ValueError(f"data: needs {self.nbytes} contiguous bytes")
        self.data = data
        self._p = data.data_ptr()

    def matrix(self, i: int) -> "Quantized":
        if not 0 <= i < self.count:
            raise IndexError(f"matrix {i} of {self.count}")
        flat = self.data.view(-1).view(_uint8())
        return Quantized(self.rows, self.cols, self.group, self.dtype, self.pair, 1,
                         flat[i * self.matrix_bytes:(i + 1) * self.matrix_bytes])


def _uint8():
    import torch
    return torch.uint8


def _matrices(q: Quantized, w, dtypes, what: str) -> int:
    """The row stride of a tensor [rows, cols] or [count, rows, cols] (a flat
    tensor of as many elements, as the sync's destination tensors are, too)."""
    if w.dtype not in dtypes:
        raise ValueError(f"{what}: elements of {w.dtype}, expected one of {dtypes}")
    shape = tuple(w.shape)
    if shape == (q.count * q.rows * q.cols,):
        if not w.is_contiguous():
            raise ValueError(f"{what}: not contiguous")
        return q.cols
    if shape == (q.rows, q.cols) and q.count == 1:
        ld = w.stride(0) if q.rows > 1 else q.cols
    elif shape == (q.count, q.rows, q.cols):
        ld = w.stride(1) if q.rows > 1 else \
            w.stride(0) if q.count > 1 else q.cols
        if q.count > 1 and w.stride(0) != q.rows * ld:
            raise ValueError(f"{what}: the matrices must follow one another")
    else:
        raise ValueError(f"{what}: shape {shape}, expected {(q.count, q.rows, q.cols)}")
    if (q.cols > 1 and w.stride(-1) != 1) or ld < q.cols:
        raise ValueError(f"{what}: the elements of a row must be contiguous, and rows must not "
                         f"overlap")
    return ld


def rr_quantize(q: Quantized, w, stream=None) -> None:
    """16-bit matrices -> q (asynchronous on `stream`)."""
    ld = _matrices(q, w, (q.torch_dtype,), "w")
    _check(_lib.rr_quantize(q._ref, w.data_ptr(), ld, q._p, _stream_of(w, stream)), "rr_quantize")


def rr_dequantize(q: Quantized, out, stream=None) -> None:
    """The values that q stands for, into `out`: of q's 16-bit type (rounded
    once), or float32 (exact).  Asynchronous on `stream`."""
    import torch
    ld = _matrices(q, out, (q.torch_dtype, torch.float32), "out")
    _check(_lib.rr_dequantize(q._ref, q._p, out.data_ptr(), ld,
                              int(out.dtype == torch.float32), _stream_of(out, stream)), "rr_dequantize")


def rr_matvec(q: Quantized, x, out, stream=None) -> None:
    """out[t] = W x[t] for up to 16 rows of x (asynchronous on `stream`); with
    q.pair, silu(gate) * up.  `out` is of q's 16-bit type or float32."""
    n, ldx = _rows(x, q.cols, q.torch_dtype, "x")
    f32 = out.dtype is not q.torch_dtype
    if f32 and out.dtype is not _f32():
        raise ValueError(f"out: elements of {out.dtype}, expected {q.torch_dtype} or float32")
    m, ldo = _rows(out, q.n_out, out.dtype, "out")
    if m != n:
        raise ValueError(f"out: {m} rows, x has {n}")
    st = _lib.rr_matvec(q._ref, q._p, x.data_ptr(), ldx, n, out.data_ptr(), ldo, f32,
                        _stream_of(x, stream))
    if st != RR_OK:
        _check(st, "rr_matvec")


def _f32():
    import torch
    return torch.float32


class MoeLayer:
    """A mixture-of-experts layer's weights, checked and marshalled once.

    router: [n_experts, hidden].  w13 and w2: the 16-bit stacks [n_local,
    2 inter, hidden] and [n_local, hidden, inter] as ``rr_unpack`` writes them,
    or both ``Quantized`` (w13 with pair=True).  first_expert: the first of the
    n_local experts held here (expert parallelism).  The layer holds references
    to the tensors; they must not be resized or freed while it is in use."""

    def __init__(self, router, w13, w2, top_k: int, first_expert: int = 0,
                 norm_topk: bool = True):
        if len(router.shape) != 2 or not router.is_contiguous():
            raise ValueError("router: expected a contiguous [n_experts, hidden]")
        n_experts, hidden = router.shape
        dtype = _type_name(router.dtype)
        packed = isinstance(w13, Quantized)
        if packed != isinstance(w2, Quantized):
            raise ValueError("w13 and w2 must both be 16-bit tensors or both Quantized")
        if packed:
            n_local, inter, group = w13.count, w13.rows // 2, w13.group
            if not w13.pair or w2.pair:
                raise ValueError("w13 must be quantised with pair=True, w2 without")
            if (w13.cols, w2.rows, w2.cols, w2.count, w2.group) != \
                    (hidden, hidden, inter, n_local, group):
                raise ValueError(f"w2 [{w2.count}, {w2.rows}, {w2.cols}] (group {w2.group}) does "
                                 f"not fit w13 [{n_local}, {2 * inter}, {w13.cols}] (group "
                                 f"{group}) and the router's {hidden} columns")
            if w13.dtype != dtype or w2.dtype != dtype:
                raise ValueError("router, w13 and w2 must have one element type")
        else:
            if len(w13.shape) != 3 or len(w2.shape) != 3:
                raise ValueError("w13 and w2: expected [n_local, 2 inter, hidden] and "
                                 "[n_local, hidden, inter]")
            n_local, inter, group = w13.shape[0], w13.shape[1] // 2, 0
            if tuple(w13.shape) != (n_local, 2 * inter, hidden) or \
                    tuple(w2.shape) != (n_local, hidden, inter):
                raise ValueError(f"w13 {tuple(w13.shape)} and w2 {tuple(w2.shape)} do not fit "
                                 f"the router's {hidden} columns")
            if w13.dtype != router.dtype or w2.dtype != router.dtype:
                raise ValueError("router, w13 and w2 must have one element type")
            if not (w13.is_contiguous() and w2.is_contiguous()):
                raise ValueError("w13 and w2 must be contiguous")
        self._c = _Moe(n_experts, first_expert, n_local, top_k, hidden, inter,
                       _DST_DTYPES[dtype], group, int(norm_topk), 0)
        self._ref = ctypes.byref(self._c)
        need = _i64()
        _check(_lib.rr_moe_workspace(self._ref, 1, ctypes.byref(need)), "rr_moe_workspace")
        self.n_experts, self.n_local, self.top_k = n_experts, n_local, top_k
        self.first_expert, self.hidden, self.inter = first_expert, hidden, inter
        self.dtype, self.torch_dtype = dtype, router.dtype
        self._keep = (router, w13, w2)
        self._p = (router.data_ptr(), w13._p if packed else w13.data_ptr(),
                   w2._p if packed else w2.data_ptr())


class MoeWorkspace:
    """Device workspace of ``rr_moe`` for up to max_tokens (1..64) tokens of a
    layer, or of any layer of the same shape, ready on every stream (the constructor
    waits for its zeros; within a graph capture it cannot, and calls belong to
    the captured stream).  Calls that overlap in time need one each.  A call whose blocks wait for one another in vain (two seconds) marks
    its workspace; later calls there leave their outputs as they are until
    ``rr_moe_check`` has raised."""

    def __init__(self, layer: MoeLayer, max_tokens: int):
        import torch
        need = _i64()
        _check(_lib.rr_moe_workspace(layer._ref, max_tokens, ctypes.byref(need)),
               "rr_moe_workspace")
        self.nbytes, self.max_tokens = need.value, max_tokens
        self.data = torch.zeros(self.nbytes, dtype=torch.uint8, device="cuda")
        # The first call may come on another stream than the zeros.
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()
        self._p = self.data.data_ptr()


def rr_moe(layer: MoeLayer, x, out, workspace: MoeWorkspace, ids=None, weights=None,
           stream=None) -> None:
    """One mixture-of-experts layer for up to 64 rows of x (asynchronous on
    `stream`).  `ids` (int32) and `weights` (float32), both [n, top_k], receive
    the chosen experts and their weights.  Outputs hold once ``rr_moe_check`` has
    found no wait that ran out."""
    n, ldx = _rows(x, layer.hidden, layer.torch_dtype, "x")
    m, ldo = _rows(out, layer.hidden, layer.torch_dtype, "out")
    if m != n:
        raise ValueError(f"out: {m} rows, x has {n}")
    pi = pw = None
    if ids is not None:
        pi = _choice(ids, n, layer.top_k, "ids", 0)
    if weights is not None:
        pw = _choice(weights, n, layer.top_k, "weights", 1)
    r, w13, w2 = layer._p
    st = _lib.rr_moe(layer._ref, r, w13, w2, x.data_ptr(), ldx, n, out.data_ptr(), ldo, pi, pw,
                     workspace._p, workspace.nbytes, _stream_of(x, stream))
    if st != RR_OK:
        _check(st, "rr_moe")


def _choice(t, n: int, k: int, what: str, floating: int) -> int:
    import torch
    want = torch.float32 if floating else torch.int32
    if t.dtype != want or t.numel() != n * k or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {want} tensor of [{n}, {k}]")
    return t.data_ptr()


def rr_moe_check(layer: MoeLayer, workspace: MoeWorkspace, stream=None) -> None:
    """Raise if a call on this workspace gave up a bounded wait (waits for `stream`):
    the outputs since the last check that passed may then be incomplete or unwritten."""
    _check(_lib.rr_moe_check(layer._ref, workspace.max_tokens, workspace._p, _stream(stream)),
           "rr_moe_check")
