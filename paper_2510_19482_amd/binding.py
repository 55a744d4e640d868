"""Thin ctypes binding over libhlq.so: argument marshalling only.

Every step of the path (pack, tables, lookups, scaling, reduction) runs inside the HIP
library; torch is used for device memory and the current stream.  There is no fallback: if
the library has not been built, importing this module raises."""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("HLQ_LIB", os.path.join(_PKG, "libhlq.so"))

HLQ_OK = 0
HLQ_OUT_F16 = 0
HLQ_OUT_F32 = 1


class HlqDesc(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("N", ctypes.c_int32), ("q", ctypes.c_int32),
                ("G", ctypes.c_int32), ("layout", ctypes.c_uint32)]


class GemvPlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("formulation", "waves_per_workgroup", "waves_per_tile", "chunks_per_slice",
                                              "slices", "tile_groups", "first_block", "blocks")]


class Mx4PlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("kernel", "tile_rows", "tile_cols", "k_parts", "quantizes", "reserved")] + [("workspace_bytes", ctypes.c_int64)]


class HlqError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {status_string(status)} (status {status})")


_vp, _sz, _i64, _i32, _int = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int32, ctypes.c_int
_szp = ctypes.POINTER(ctypes.c_size_t)
_MX4_ARGS = {
    "hlq_mx4_bytes": [_i64, _i32, _szp],
    "hlq_mx4_quantize": [_i64, _i32, _vp, _int, _i64, _vp, _sz, _vp],
    "hlq_mx4_dequantize": [_i64, _i32, _vp, _vp, _int, _i64, _vp],
    "hlq_mx4_pack": [_i64, _i32, _vp, _i64, _vp, _i64, _vp, _sz, _vp],
    "hlq_mx4_unpack": [_i64, _i32, _vp, _vp, _vp, _vp],
    "hlq_mx4_workspace_bytes": [_i64, _i32, _i32, _i64, _i64, _szp],
    "hlq_mx4_plan_query": [_i64, _i32, _i32, _i64, _i64, _int, _int, ctypes.POINTER(Mx4PlanInfo)],
    "hlq_mx4_gemm": [_i64, _i32, _vp, _i64, _vp, _int, _i64, _vp, _int, _i64, _int, _vp, _sz, _vp],
    "hlq_route_workspace_bytes": [_i64, _i32, _i32, _szp],
    "hlq_route": [_i64, _i32, _i32, _vp, _int, _i64, _int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "hlq_expert_gemm": [_i32, _i64, _i32, _vp, _vp, _vp, _i64, _i64, _vp, _int, _i64, _vp, _int, _i64, _int, _vp, _sz, _vp],
    "hlq_expert_combine": [_i64, _i32, _i32, _i64, _vp, _int, _i64, _vp, _vp, _vp, _int, _i64, _vp],
}


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2510_19482_amd.build` "
            "(there is no CPU fallback)")
    # torch ships its own copy of the HIP runtime (same SONAME as the system one).  It has to be
    # loaded first: libhlq then binds to that copy, and both sides share one runtime, one device
    # context and the same stream handles.  Loaded the other way round the process ends up with
    # two runtimes and launches fail with "no ROCm-capable device".
    global torch
    import torch
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, i64, u32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_uint32
    dp = ctypes.POINTER(HlqDesc)
    szp = ctypes.POINTER(ctypes.c_size_t)
    lib.hlq_status_string.restype = ctypes.c_char_p
    lib.hlq_status_string.argtypes = [ctypes.c_int]
    lib.hlq_layout_version.restype = u32
    lib.hlq_layout_version.argtypes = []
    lib.hlq_packed_bytes.restype = ctypes.c_int
    lib.hlq_packed_bytes.argtypes = [dp, szp, szp, szp]
    lib.hlq_workspace_bytes.restype = ctypes.c_int
    lib.hlq_workspace_bytes.argtypes = [dp, i64, szp]
    lib.hlq_pack.restype = ctypes.c_int
    lib.hlq_pack.argtypes = [dp, vp, vp, vp, vp, sz, vp]
    lib.hlq_unpack.restype = ctypes.c_int
    lib.hlq_unpack.argtypes = [dp, vp, vp, vp, vp, vp]
    lib.hlq_lut_gemv.restype = ctypes.c_int
    lib.hlq_lut_gemv.argtypes = [dp, vp, vp, vp, ctypes.c_int, vp, sz, vp]
    lib.hlq_lut_gemv_static.restype = ctypes.c_int
    lib.hlq_lut_gemv_static.argtypes = [dp, vp, vp, vp, ctypes.c_int, vp]
    lib.hlq_batch_workspace_bytes.restype = ctypes.c_int
    lib.hlq_batch_workspace_bytes.argtypes = [ctypes.c_int, dp, szp]
    lib.hlq_workspace_init.restype = ctypes.c_int
    lib.hlq_workspace_init.argtypes = [vp, sz, vp]
    lib.hlq_quantize.restype = ctypes.c_int
    lib.hlq_quantize.argtypes = [dp, vp, ctypes.c_int, vp, vp, vp, vp, vp]
    lib.hlq_gemm_batch_workspace_bytes.restype = ctypes.c_int
    lib.hlq_gemm_batch_workspace_bytes.argtypes = [ctypes.c_int, dp, ctypes.c_int64, szp]
    lib.hlq_lut_gemm_batch.restype = ctypes.c_int
    lib.hlq_lut_gemm_batch.argtypes = [ctypes.c_int, dp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.c_int64,
                                       ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(vp),
                                       ctypes.POINTER(ctypes.c_int64), ctypes.c_int, vp, ctypes.c_size_t, vp]
    lib.hlq_lut_gemv_batch.restype = ctypes.c_int
    lib.hlq_lut_gemv_batch.argtypes = [ctypes.c_int, dp, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                       ctypes.POINTER(vp), ctypes.c_int, vp, sz, vp]
    lib.hlq_gemv_plan_query.restype = ctypes.c_int
    lib.hlq_gemv_plan_query.argtypes = [ctypes.c_int, dp, i64, ctypes.POINTER(GemvPlanInfo)]
    lib.hlq_set_gemv_plan.restype = ctypes.c_int
    lib.hlq_set_gemv_plan.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int]
    lib.hlq_set_gemm_path.restype = ctypes.c_int
    lib.hlq_set_gemm_path.argtypes = [ctypes.c_int]
    lib.hlq_set_gemv_path.restype = ctypes.c_int
    lib.hlq_set_gemv_path.argtypes = [ctypes.c_int]
    lib.hlq_stream_read.restype = ctypes.c_int
    lib.hlq_stream_read.argtypes = [vp, sz, ctypes.c_int, vp, sz, vp]
    lib.hlq_mfma_probe.restype = ctypes.c_int
    lib.hlq_mfma_probe.argtypes = [ctypes.c_int, vp, sz, ctypes.c_int, ctypes.c_int, vp, sz, ctypes.POINTER(ctypes.c_double), vp]
    lib.hlq_stream_read_shaped.restype = ctypes.c_int
    lib.hlq_stream_read_shaped.argtypes = [vp, sz, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, sz, vp]
    for name, args in _MX4_ARGS.items():
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = args
    lib.hlq_lut_gemm.restype = ctypes.c_int
    lib.hlq_lut_gemm.argtypes = [dp, vp, vp, i64, i64, vp, i64, ctypes.c_int, vp, sz, vp]
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.hlq_status_string(int(status)).decode()


def layout_version() -> int:
    return int(lib.hlq_layout_version())


def make_desc(K: int, N: int, q: int, G: int, layout: int | None = None) -> HlqDesc:
    return HlqDesc(K, N, q, G, layout_version() if layout is None else layout)


def _check(fn: str, status: int) -> None:
    if status != HLQ_OK:
        raise HlqError(fn, status)


def set_gemv_plan(tiles_per_wave: int = 0, waves_per_workgroup: int = 0, chunks_per_wave: int = 0) -> None:
    _check("hlq_set_gemv_plan", lib.hlq_set_gemv_plan(tiles_per_wave, waves_per_workgroup, chunks_per_wave))


def gemv_plan_query(descs, M: int = 1):
    """Work split of a grouped GEMV / few-rows launch over `descs` (host arithmetic, no GPU needed)."""
    n = len(descs)
    arr = (HlqDesc * n)(*descs)
    out = (GemvPlanInfo * n)()
    _check("hlq_gemv_plan_query", lib.hlq_gemv_plan_query(n, arr, M, out))
    return list(out)


GEMM_AUTO, GEMM_LUT, GEMM_MFMA, GEMM_MFMA_FP16, GEMM_ROWS16 = 0, 1, 2, 3, 4


def set_gemm_path(path: int = 0) -> None:
    _check("hlq_set_gemm_path", lib.hlq_set_gemm_path(path))


GEMV_AUTO, GEMV_LUT, GEMV_MX = 0, 1, 2
GEMV_TABLE_F32, GEMV_TABLE_MIRROR, GEMV_TABLE_F16, GEMV_TABLE_I8 = 3, 4, 5, 6


def set_gemv_path(path: int = 0) -> None:
    _check("hlq_set_gemv_path", lib.hlq_set_gemv_path(path))


def packed_bytes(desc: HlqDesc):
    """(total, bits, meta) byte counts of the packed blob."""
    t, b, m = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check("hlq_packed_bytes", lib.hlq_packed_bytes(ctypes.byref(desc), ctypes.byref(t), ctypes.byref(b), ctypes.byref(m)))
    return t.value, b.value, m.value


def workspace_bytes(desc: HlqDesc, M: int) -> int:
    w = ctypes.c_size_t()
    _check("hlq_workspace_bytes", lib.hlq_workspace_bytes(ctypes.byref(desc), M, ctypes.byref(w)))
    return w.value


# ---- torch-facing helpers (device tensors in, device tensors out) -------------------------
def _stream_ptr(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    if not torch.cuda.is_initialized():
        return int(torch.cuda.current_stream().cuda_stream)
    # the handle of the calling thread's current stream on its current device, without the Stream object around it:
    # a one-row call of a small matrix spends 3 us on the GPU, and building that object took 1.5 us of the host's time
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def hlq_pack(desc: HlqDesc, codes, scales, zeros, packed=None, stream=None):
    """codes u8 [K,N], scales fp16 [q,K/G,N], zeros fp16 [K/G,N] (cuda tensors) -> packed u8 blob."""
    total, _, _ = packed_bytes(desc)
    if packed is None:
        packed = torch.empty(total, dtype=torch.uint8, device=codes.device)
    _check("hlq_pack", lib.hlq_pack(ctypes.byref(desc), _ptr(codes), _ptr(scales), _ptr(zeros),
                                    _ptr(packed), packed.numel() * packed.element_size(), _stream_ptr(stream)))
    return packed


def hlq_unpack(desc: HlqDesc, packed, stream=None):
    K, N, q, G = desc.K, desc.N, desc.q, desc.G
    codes = torch.empty((K, N), dtype=torch.uint8, device=packed.device)
    scales = torch.empty((q, K // G, N), dtype=torch.float16, device=packed.device)
    zeros = torch.empty((K // G, N), dtype=torch.float16, device=packed.device)
    _check("hlq_unpack", lib.hlq_unpack(ctypes.byref(desc), _ptr(packed), _ptr(codes), _ptr(scales),
                                        _ptr(zeros), _stream_ptr(stream)))
    return codes, scales, zeros


def batch_workspace_bytes(descs) -> int:
    arr = (HlqDesc * len(descs))(*descs)
    w = ctypes.c_size_t()
    _check("hlq_batch_workspace_bytes", lib.hlq_batch_workspace_bytes(len(descs), arr, ctypes.byref(w)))
    return w.value


def _new_workspace(nbytes: int, device, stream=None):
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _check("hlq_workspace_init", lib.hlq_workspace_init(_ptr(ws), ws.numel(), _stream_ptr(stream)))
    return ws


def alloc_workspace(desc: HlqDesc, M: int, device="cuda", stream=None):
    """Allocate and initialise a workspace for GEMV/GEMM calls on `desc` with up to M rows."""
    return _new_workspace(workspace_bytes(desc, M), device, stream)


def alloc_batch_workspace(descs, device="cuda", stream=None):
    return _new_workspace(batch_workspace_bytes(descs), device, stream)


def hlq_quantize(desc: HlqDesc, W, t_max: int = 10, with_err: bool = False, stream=None):
    """Alg. 1 on W fp32 cuda [K, N] -> codes u8 [K, N], scales fp16 [q, K/G, N], zeros fp16 [K/G, N]
    (and the per-group squared error fp32 [K/G, N] with with_err=True)."""
    assert W.dtype == torch.float32 and W.is_contiguous() and tuple(W.shape) == (desc.K, desc.N)
    dev = W.device
    codes = torch.empty((desc.K, desc.N), dtype=torch.uint8, device=dev)
    scales = torch.empty((desc.q, desc.K // desc.G, desc.N), dtype=torch.float16, device=dev)
    zeros = torch.empty((desc.K // desc.G, desc.N), dtype=torch.float16, device=dev)
    err = torch.empty((desc.K // desc.G, desc.N), dtype=torch.float32, device=dev) if with_err else None
    _check("hlq_quantize", lib.hlq_quantize(ctypes.byref(desc), _ptr(W), t_max, _ptr(codes), _ptr(scales), _ptr(zeros),
                                            _ptr(err) if with_err else None, _stream_ptr(stream)))
    return (codes, scales, zeros, err) if with_err else (codes, scales, zeros)


def hlq_stream_read(src, nbytes: int, sink, blocks: int = 0, offset: int = 0, stream=None):
    """Measurement helper: read nbytes of `src` (a cuda tensor) from byte `offset` on, once."""
    _check("hlq_stream_read", lib.hlq_stream_read(_ptr(src) + offset, nbytes, blocks, _ptr(sink),
                                                  sink.numel() * sink.element_size(), _stream_ptr(stream)))


def hlq_stream_read_shaped(src, nbytes: int, sink, blocks: int = 0, unroll: int = 4, temporal: bool = False,
                           offset: int = 0, stream=None):
    """hlq_stream_read with its loop shape and cache policy as arguments (for sweeps)."""
    _check("hlq_stream_read_shaped", lib.hlq_stream_read_shaped(_ptr(src) + offset, nbytes, blocks, unroll, int(temporal),
                                                                _ptr(sink), sink.numel() * sink.element_size(),
                                                                _stream_ptr(stream)))


def hlq_mfma_probe(operands, iters: int, blocks: int, sink, kind: int = 0, stream=None) -> float:
    """Launch the matrix-core-only measurement loop (kind 0: fp16 32x32x16, 1: bf8 x fp4 16x16x128); returns the
    floating-point operations of the launch."""
    flop = ctypes.c_double(0.0)
    _check("hlq_mfma_probe", lib.hlq_mfma_probe(kind, _ptr(operands), operands.numel() * operands.element_size(), iters, blocks,
                                                _ptr(sink), sink.numel() * sink.element_size(), ctypes.byref(flop),
                                                _stream_ptr(stream)))
    return flop.value


class GemvBatch:
    """Pre-marshalled arguments of one hlq_lut_gemv_batch call (host arrays built once)."""

    def __init__(self, descs, packed, xs, ys, out_f32=False, ws=None):
        n = len(descs)
        self.n = n
        self.descs = (HlqDesc * n)(*descs)
        self.packed = (ctypes.c_void_p * n)(*[_ptr(p) for p in packed])
        self.xs = (ctypes.c_void_p * n)(*[_ptr(x) for x in xs])
        self.ys = (ctypes.c_void_p * n)(*[_ptr(y) for y in ys])
        self.out = HLQ_OUT_F32 if out_f32 else HLQ_OUT_F16
        self.ws = ws if ws is not None else alloc_batch_workspace(list(descs), xs[0].device)
        self._keep = (list(packed), list(xs), list(ys))

    def launch(self, stream=None):
        _check("hlq_lut_gemv_batch", lib.hlq_lut_gemv_batch(
            self.n, self.descs, self.packed, self.xs, self.ys, self.out, _ptr(self.ws),
            self.ws.numel(), _stream_ptr(stream)))


class GemmBatch:
    """Pre-marshalled arguments of one hlq_lut_gemm_batch call: Y_i[M, N_i] = X_i[M, K_i] @ W^_i."""

    def __init__(self, descs, packed, Xs, Ys, out_f32=False, ws=None):
        n = len(descs)
        self.n = n
        self.M = int(Xs[0].shape[0])
        self.descs = (HlqDesc * n)(*descs)
        self.packed = (ctypes.c_void_p * n)(*[_ptr(p) for p in packed])
        self.Xs = (ctypes.c_void_p * n)(*[_ptr(x) for x in Xs])
        self.Ys = (ctypes.c_void_p * n)(*[_ptr(y) for y in Ys])
        self.ldx = (ctypes.c_int64 * n)(*[max(int(x.stride(0)), d.K) for x, d in zip(Xs, descs)])
        self.ldy = (ctypes.c_int64 * n)(*[max(int(y.stride(0)), d.N) for y, d in zip(Ys, descs)])
        self.out = HLQ_OUT_F32 if out_f32 else HLQ_OUT_F16
        if ws is None:
            w = ctypes.c_size_t()
            _check("hlq_gemm_batch_workspace_bytes",
                   lib.hlq_gemm_batch_workspace_bytes(n, self.descs, self.M, ctypes.byref(w)))
            ws = _new_workspace(w.value, Xs[0].device)
        self.ws = ws
        self._keep = (list(packed), list(Xs), list(Ys))

    def launch(self, stream=None):
        _check("hlq_lut_gemm_batch", lib.hlq_lut_gemm_batch(
            self.n, self.descs, self.packed, self.Xs, self.M, self.ldx, self.Ys, self.ldy, self.out,
            _ptr(self.ws), self.ws.numel(), _stream_ptr(stream)))


def hlq_lut_gemv(desc: HlqDesc, packed, x, y=None, out_f32: bool = False, ws=None, stream=None):
    """y[N] = x[K] @ W^ ; x fp16 cuda tensor."""
    if y is None:
        y = torch.empty(desc.N, dtype=torch.float32 if out_f32 else torch.float16, device=x.device)
    if ws is None:
        ws = alloc_workspace(desc, 1, x.device)
    status = lib.hlq_lut_gemv(desc, _ptr(packed), _ptr(x), _ptr(y), HLQ_OUT_F32 if out_f32 else HLQ_OUT_F16, _ptr(ws), ws.numel(),
                              _stream_ptr(stream))
    if status != HLQ_OK:
        raise HlqError("hlq_lut_gemv", status)
    return y


STATIC_SCRATCH_BYTES = 131072 + (4 << 20)


def hlq_lut_gemv_static(desc: HlqDesc, packed, x, y, out_f32: bool = False, stream=None):
    """hlq_lut_gemv without a workspace argument (scratch in a fixed array of the library); `y` is
    the caller's output tensor: this call allocates nothing."""
    _check("hlq_lut_gemv_static", lib.hlq_lut_gemv_static(ctypes.byref(desc), _ptr(packed), _ptr(x), _ptr(y),
                                                          HLQ_OUT_F32 if out_f32 else HLQ_OUT_F16, _stream_ptr(stream)))
    return y


def hlq_lut_gemm(desc: HlqDesc, packed, X, Y=None, out_f32: bool = False, ws=None, stream=None):
    """Y[M,N] = X[M,K] @ W^ ; X fp16 cuda tensor, row-major (stride(1) == 1)."""
    M = X.shape[0]
    if Y is None:
        Y = torch.empty((M, desc.N), dtype=torch.float32 if out_f32 else torch.float16, device=X.device)
    if ws is None:
        ws = alloc_workspace(desc, M, X.device)
    ldx = X.stride(0) if M > 1 else max(X.stride(0), desc.K)
    ldy = Y.stride(0) if M > 1 else max(Y.stride(0), desc.N)
    _check("hlq_lut_gemm", lib.hlq_lut_gemm(ctypes.byref(desc), _ptr(packed), _ptr(X), M, ldx, _ptr(Y), ldy,
                                            HLQ_OUT_F32 if out_f32 else HLQ_OUT_F16, _ptr(ws), ws.numel(),
                                            _stream_ptr(stream)))
    return Y


# ---- microscaled 4-bit matrices and the expert block ----------------------------------------------------------------
HLQ_F16, HLQ_F32, HLQ_BF16, HLQ_MX4 = 0, 1, 2, 3
_DTYPES = {torch.float16: HLQ_F16, torch.float32: HLQ_F32, torch.bfloat16: HLQ_BF16}


def _matrix(t):
    """(rows, columns, pointer, type, leading dimension) of a matrix whose rows are contiguous; one row's leading dimension is its length.
    Called several times for an operator whose kernel takes a few microseconds: each attribute of a tensor costs a tenth of one."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise TypeError(f"expected a float16, bfloat16 or float32 tensor, got {t.dtype}")
    try:
        rows, cols = t.shape
        ld, one = t.stride()
    except ValueError:
        raise ValueError(f"expected a matrix, got shape {tuple(t.shape)}") from None
    if (one != 1 and cols > 1) or (rows > 1 and ld < cols):
        raise ValueError(f"expected a matrix whose rows are contiguous, got shape {tuple(t.shape)} with strides {t.stride()}")
    return rows, cols, t.data_ptr(), dtype, ld if rows > 1 else cols


def _not_on_gpu(*tensors):
    return ValueError(f"expected tensors on the GPU, all on one GPU, got {', '.join(str(t.device) for t in tensors)}")


_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # of a device, its handle


def _stream_of(stream, device: int) -> int:
    """Handle of the stream that a call on this device runs on."""
    if stream is None:
        return _current_stream(device)
    if stream.device_index != device:
        raise ValueError(f"the tensors are on cuda:{device}, the stream is of cuda:{stream.device_index}")
    return int(stream.cuda_stream)


def _there(device: int, call, *args):
    """The call with its operands' device as the current one, which the library launches on."""
    with torch.cuda.device(device):
        return call(*args)


def _empty(shape, dtype, device, stream):
    """A new tensor of the stream that the call runs on: memory that another stream still uses is not handed out for it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def mx4_bytes(rows: int, K: int) -> int:
    n = ctypes.c_size_t()
    _check("hlq_mx4_bytes", lib.hlq_mx4_bytes(rows, K, ctypes.byref(n)))
    return n.value


class Mx4:
    """A microscaled 4-bit matrix [rows, K]: the blob (u8) in the library's layout.  Another blob may be put in its place."""

    __slots__ = ("blob", "rows", "K", "_need", "_kept", "_ptr", "_size", "_device")

    def __init__(self, blob, rows: int, K: int):
        put = object.__setattr__
        put(self, "rows", int(rows))
        put(self, "K", int(K))
        put(self, "_need", mx4_bytes(rows, K))
        self.blob = blob

    def __setattr__(self, name, value):
        if name != "blob":
            raise AttributeError(f"{name} of a matrix stays as it was made")
        self._take(value)
        object.__setattr__(self, name, value)

    def _take(self, blob) -> None:
        size, ptr, put = blob.numel(), blob.data_ptr(), object.__setattr__
        if blob.dtype != torch.uint8 or size < self._need or not blob.is_contiguous() or (ptr == 0 and self._need):
            raise ValueError(f"a blob of {self._need} bytes is needed for {self.rows} x {self.K}")
        put(self, "_kept", blob.detach())
        put(self, "_ptr", ptr)
        put(self, "_size", size)
        put(self, "_device", blob.get_device())

    is_cuda = property(lambda self: self.blob.is_cuda)
    device = property(lambda self: self.blob.device)

    def get_device(self) -> int:
        return self.blob.get_device()

    def __reduce__(self):
        return Mx4, (self.blob, self.rows, self.K)


def _blob(m: Mx4):
    """Address, size and device of a matrix's blob as it is now.  Its data may have been replaced since the last call; at the address that was
    taken then it has not been, since that memory is kept and nothing else can be there."""
    if m.blob.data_ptr() != m._ptr:
        m._take(m.blob)
    return m._ptr, m._size, m._device


def alloc_mx4(rows: int, K: int, device="cuda", stream=None) -> Mx4:
    return Mx4(_empty(mx4_bytes(rows, K), torch.uint8, device, stream), rows, K)


def _mx4_out(out, rows: int, K: int, device, stream) -> Mx4:
    if out is None:
        return alloc_mx4(rows, K, device, stream)
    if out.rows != rows or out.K != K:
        raise ValueError(f"the output is a matrix of {out.rows} x {out.K}, not {rows} x {K}")
    return out


def hlq_mx4_quantize(x, out: Mx4 | None = None, stream=None) -> Mx4:
    """Rows of x [rows, K] (f16, bf16 or f32) in 4-bit floats, a power-of-two scale for each 32 of a row."""
    rows, K, ptr, dtype, ld = _matrix(x)
    out = _mx4_out(out, rows, K, x.device, stream)
    blob, size, at = _blob(out)
    device = x.get_device()
    if device < 0 or at != device:
        raise _not_on_gpu(x, out.blob)
    if device != _current_device():
        return _there(device, hlq_mx4_quantize, x, out, stream)
    status = lib.hlq_mx4_quantize(rows, K, ptr, dtype, ld, blob, size, _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_mx4_quantize", status)
    return out


def hlq_mx4_dequantize(m: Mx4, y=None, dtype=None, stream=None):
    """The values [rows, K] that a matrix stands for, in y or a new tensor of `dtype` (f32 by default)."""
    if y is None:
        y = _empty((m.rows, m.K), dtype or torch.float32, m.blob.device, stream)
    rows, K, ptr, dtype, ld = _matrix(y)
    if rows != m.rows or K != m.K:
        raise ValueError(f"y has shape {tuple(y.shape)}, the matrix is {m.rows} x {m.K}")
    blob, _, device = _blob(m)
    if device < 0 or y.get_device() != device:
        raise _not_on_gpu(y, m.blob)
    if device != _current_device():
        return _there(device, hlq_mx4_dequantize, m, y, None, stream)
    status = lib.hlq_mx4_dequantize(rows, K, blob, ptr, dtype, ld, _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_mx4_dequantize", status)
    return y


def hlq_mx4_pack(codes, scales, K: int, out: Mx4 | None = None, stream=None) -> Mx4:
    """codes u8 [rows, (K + 1) // 2 or more] (the even k in the low half of a byte), scales u8 [rows, (K + 31) // 32 or more] -> matrix."""
    rows = codes.shape[0]
    for name, t, least in (("codes", codes, (K + 1) // 2), ("scales", scales, (K + 31) // 32)):
        if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[0] != rows or t.shape[1] < least or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError(f"{name}: expected uint8 of shape ({rows}, at least {least}), rows contiguous, got {t.dtype} {tuple(t.shape)}")
    out = _mx4_out(out, rows, K, codes.device, stream)
    blob, size, device = _blob(out)
    if device < 0 or codes.get_device() != device or scales.get_device() != device:
        raise _not_on_gpu(codes, scales, out.blob)
    if device != _current_device():
        return _there(device, hlq_mx4_pack, codes, scales, K, out, stream)
    _check("hlq_mx4_pack", lib.hlq_mx4_pack(rows, K, _ptr(codes), codes.stride(0), _ptr(scales), scales.stride(0), blob, size, _stream_of(stream, device)))
    return out


def hlq_mx4_unpack(m: Mx4, stream=None):
    blob, _, device = _blob(m)
    if device < 0:
        raise _not_on_gpu(m.blob)
    if device != _current_device():
        return _there(device, hlq_mx4_unpack, m, stream)
    codes = _empty((m.rows, (m.K + 1) // 2), torch.uint8, m.blob.device, stream)
    scales = _empty((m.rows, (m.K + 31) // 32), torch.uint8, m.blob.device, stream)
    _check("hlq_mx4_unpack", lib.hlq_mx4_unpack(m.rows, m.K, blob, _ptr(codes), _ptr(scales), _stream_of(stream, device)))
    return codes, scales


def mx4_workspace_bytes(N: int, K: int, experts: int, x_rows: int, rows: int) -> int:
    n = ctypes.c_size_t()
    _check("hlq_mx4_workspace_bytes", lib.hlq_mx4_workspace_bytes(N, K, experts, x_rows, rows, ctypes.byref(n)))
    return n.value


def mx4_plan_query(N: int, K: int, rows: int, experts: int = 1, x_rows: int | None = None, xtype: int = HLQ_MX4, gated: bool = False) -> Mx4PlanInfo:
    """The kernel that a product goes to (host arithmetic, no GPU needed)."""
    out = Mx4PlanInfo()
    _check("hlq_mx4_plan_query", lib.hlq_mx4_plan_query(N, K, experts, rows if x_rows is None else x_rows, rows, xtype, 1 if gated else 0, ctypes.byref(out)))
    return out


def alloc_mx4_workspace(W: Mx4, x_rows: int, rows: int | None = None, experts: int = 1, stream=None):
    """Workspace for products with W of up to x_rows activation rows and `rows` result rows (the same if not given)."""
    device = W.blob.get_device()
    if device < 0:
        raise _not_on_gpu(W.blob)
    if device != _current_device():
        return _there(device, alloc_mx4_workspace, W, x_rows, rows, experts, stream)
    ws = _empty(mx4_workspace_bytes(W.rows // experts, W.K, experts, x_rows, x_rows if rows is None else rows), torch.uint8, W.blob.device, stream)
    _check("hlq_workspace_init", lib.hlq_workspace_init(_ptr(ws), ws.numel(), _stream_of(stream, device)))
    return ws


def _operand(X: Mx4):
    """As _matrix, of activations that are quantized already."""
    return X.rows, X.K, _blob(X)[0], HLQ_MX4, 0


def _product_out(W: Mx4, X, R: int, cols: int, out_dtype, stream):
    if out_dtype is None:
        out_dtype = torch.float32 if type(X) is Mx4 else X.dtype
    return _empty((R, cols), out_dtype, W.blob.device, stream)


def hlq_mx4_gemm(W: Mx4, X, Y=None, gated: bool = False, out_dtype=None, ws=None, stream=None):
    """Y = Q(X) W^T, or with `gated` silu of its first half of columns times the second; X [M, K] f16, bf16 or f32, or Mx4."""
    M, K, x, xtype, ldx = _operand(X) if type(X) is Mx4 else _matrix(X)
    blob, _, device = _blob(W)
    N = W.rows
    cols = N // 2 if gated else N
    if Y is None:
        Y = _product_out(W, X, M, cols, out_dtype, stream)
    y_rows, y_cols, y, ytype, ldy = _matrix(Y)
    if K != W.K or y_rows != M or y_cols != cols:
        raise ValueError(f"X is {M} x {K}, W {N} x {W.K}, Y {y_rows} x {y_cols}{' (gated)' if gated else ''}")
    if ws is None:
        ws = alloc_mx4_workspace(W, M, stream=stream)
    if device < 0 or X.get_device() != device or Y.get_device() != device or ws.get_device() != device:
        raise _not_on_gpu(W.blob, X, Y, ws)
    if device != _current_device():
        return _there(device, hlq_mx4_gemm, W, X, Y, gated, None, ws, stream)
    status = lib.hlq_mx4_gemm(N, K, blob, M, x, xtype, ldx, y, ytype, ldy, 1 if gated else 0, ws.data_ptr(), ws.numel(), _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_mx4_gemm", status)
    return Y


class Route:
    """What hlq_route writes: ids, weights, slots [T, k], offsets [E + 1], rows [T k], and its workspace; views of memory that lives as long
    as this does."""

    __slots__ = ("ids", "weights", "offsets", "rows", "slots", "ws", "T", "E", "k", "_device", "_memory", "_args")

    def __init__(self, T: int, E: int, k: int, device="cuda", stream=None):
        n = ctypes.c_size_t()
        _check("hlq_route_workspace_bytes", lib.hlq_route_workspace_bytes(T, E, k, ctypes.byref(n)))
        pairs, room = T * k, (T * k + 3) // 4 * 4                # in words; parts begin at multiples of 16 bytes
        offsets, ws = 4 * room, 4 * room + (E + 4) // 4 * 4
        memory = _empty(ws + (n.value + 3) // 4, torch.int32, device, stream)
        base, bytes_ = memory.data_ptr(), memory.view(torch.uint8)
        for name, value in (("T", T), ("E", E), ("k", k), ("_memory", bytes_), ("_device", memory.get_device()),
                            ("ids", memory.as_strided((T, k), (k, 1), 0)), ("slots", memory.as_strided((T, k), (k, 1), room)), ("rows", memory.as_strided((pairs,), (1,), 2 * room)),
                            ("weights", memory.view(torch.float32).as_strided((T, k), (k, 1), 3 * room)), ("offsets", memory.as_strided((E + 1,), (1,), offsets)),
                            ("ws", bytes_.as_strided((n.value,), (1,), 4 * ws)),
                            ("_args", (base, base + 12 * room, base + 4 * offsets, base + 8 * room, base + 4 * room, base + 4 * ws, n.value))):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):
        raise AttributeError(f"{name} of a route stays as it was made")

    def __reduce__(self):
        return _route_of, (self.T, self.E, self.k, self._memory)


def _route_of(T: int, E: int, k: int, memory) -> Route:
    route = Route(T, E, k, memory.device)
    route._memory.copy_(memory)
    return route


def alloc_route(T: int, E: int, k: int, device="cuda", stream=None) -> Route:
    return Route(T, E, k, device, stream)


def hlq_route(logits, k: int, renorm: bool = True, out: Route | None = None, stream=None) -> Route:
    """The k experts of each token by its logits [T, E], their weights, and the tokens grouped by expert."""
    T, E, ptr, dtype, ld = _matrix(logits)
    if out is None:
        out = Route(T, E, k, logits.device, stream)
    elif out.T != T or out.E != E or out.k != k:
        raise ValueError(f"the output is for {out.T} tokens, {out.E} experts, {out.k} each")
    device = logits.get_device()
    if device < 0 or out._device != device:
        raise _not_on_gpu(logits, out._memory)
    if device != _current_device():
        return _there(device, hlq_route, logits, k, renorm, out, stream)
    status = lib.hlq_route(T, E, k, ptr, dtype, ld, 1 if renorm else 0, *out._args, _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_route", status)
    return out


def hlq_expert_gemm(W: Mx4, offsets, X, Y=None, rows=None, gated: bool = False, out_dtype=None, ws=None, stream=None):
    """Y[r] = Q(X[rows[r]]) W_e^T for the rows offsets[e] <= r < offsets[e + 1] of each expert e, or of X[r] without `rows`;
    W holds the experts' matrices one after the other."""
    E = offsets.numel() - 1
    if E < 1 or W.rows % E or offsets.dtype != torch.int32 or not offsets.is_contiguous():
        raise ValueError(f"offsets: int32, one more than experts; {offsets.numel()} of {offsets.dtype} for {W.rows} rows of weights")
    x_rows, K, x, xtype, ldx = _operand(X) if type(X) is Mx4 else _matrix(X)
    if rows is None:
        R, rows_ptr = x_rows, None
    else:
        if rows.dtype != torch.int32 or not rows.is_contiguous():
            raise ValueError(f"rows: contiguous int32, got {rows.dtype}")
        R, rows_ptr = rows.numel(), rows.data_ptr()
    blob, _, device = _blob(W)
    N = W.rows // E
    cols = N // 2 if gated else N
    if Y is None:
        Y = _product_out(W, X, R, cols, out_dtype, stream)
    y_rows, y_cols, y, ytype, ldy = _matrix(Y)
    if K != W.K or y_rows != R or y_cols != cols:
        raise ValueError(f"X is {x_rows} x {K}, a matrix of W {N} x {W.K}, Y {y_rows} x {y_cols} for {R} rows{' (gated)' if gated else ''}")
    if ws is None:
        ws = alloc_mx4_workspace(W, x_rows, R, E, stream)
    if (device < 0 or offsets.get_device() != device or X.get_device() != device or Y.get_device() != device or ws.get_device() != device
            or (rows is not None and rows.get_device() != device)):
        raise _not_on_gpu(W.blob, offsets, X, Y, ws, *([] if rows is None else [rows]))
    if device != _current_device():
        return _there(device, hlq_expert_gemm, W, offsets, X, Y, rows, gated, None, ws, stream)
    status = lib.hlq_expert_gemm(E, N, K, blob, offsets.data_ptr(), rows_ptr, R, x_rows, x, xtype, ldx, y, ytype, ldy, 1 if gated else 0,
                                 ws.data_ptr(), ws.numel(), _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_expert_gemm", status)
    return Y


def hlq_expert_combine(Y, slots, weights, out=None, out_dtype=None, stream=None):
    """out[t] = sum_i weights[t, i] Y[slots[t, i]] (slot -1: nothing)."""
    T, k = slots.shape
    R, D, y, ytype, ldy = _matrix(Y)
    if slots.dtype != torch.int32 or weights.dtype != torch.float32 or weights.shape != slots.shape or not (slots.is_contiguous() and weights.is_contiguous()):
        raise ValueError(f"slots and weights: contiguous int32 and float32 of one shape, got {slots.dtype} {tuple(slots.shape)} and {weights.dtype} {tuple(weights.shape)}")
    if out is None:
        out = _empty((T, D), out_dtype or Y.dtype, Y.device, stream)
    o_rows, o_cols, o, otype, ldo = _matrix(out)
    if o_rows != T or o_cols != D:
        raise ValueError(f"out has shape {tuple(out.shape)}, the result is {T} x {D}")
    device = Y.get_device()
    if device < 0 or slots.get_device() != device or weights.get_device() != device or out.get_device() != device:
        raise _not_on_gpu(Y, slots, weights, out)
    if device != _current_device():
        return _there(device, hlq_expert_combine, Y, slots, weights, out, None, stream)
    status = lib.hlq_expert_combine(T, k, D, R, y, ytype, ldy, slots.data_ptr(), weights.data_ptr(), o, otype, ldo, _stream_of(stream, device))
    if status != HLQ_OK:
        raise HlqError("hlq_expert_combine", status)
    return out
