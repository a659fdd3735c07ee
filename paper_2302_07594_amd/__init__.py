"""Python binding for libigemm (integer GEMM C += A.B on MI355X / gfx950).

The functions here marshal arguments into the C ABI of ``include/igemm.h``
with ctypes; every step of the computation runs in the HIP library. PyTorch
is used only to hand over device pointers and the current HIP stream. The
tensor calls below go through a compiled binding (``_igemm_torch``) in the
plain case: checks, plan, workspace and call in one step. There is no CPU
fallback: the libraries are loaded at the first call, and that call raises
ImportError if they are not built (``build`` is importable without them).

Same names as the C ABI:
    igemm_i16(m, n, k, A, lda, B, ldb, C, ldc, stream=None)
    igemm_i8 (m, n, k, A, lda, B, ldb, C, ldc, stream=None)
    igemm_i16_ex / igemm_i8_ex(..., kernel=-1, split=-1)
    igemm_i16_ws / igemm_i8_ws(..., kernel=-1, split=-1, workspace=None,
                               workspace_bytes=0)
    igemm_i16_noalloc(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1,
                      split=-1)
    igemm_pack_i16 / igemm_pack_i8(m, n, k, A, lda, B, ldb, kernel=-1,
                                   workspace, workspace_bytes, stream=None)
    igemm_i16_prepacked / igemm_i8_prepacked(m, n, k, A, lda, C, ldc, kernel=-1,
                                             workspace, workspace_bytes, stream=None)
    igemm_pack_b_i16 / igemm_pack_b_i8(n, k, B, ldb, kernel=-1, packed_b,
                                       packed_b_bytes, stream=None)
    igemm_i16_packed_b / igemm_i8_packed_b(m, n, k, A, lda, packed_b, packed_b_bytes,
                                           C, ldc, kernel=-1, workspace=None,
                                           workspace_bytes=0, stream=None)
    igemm_query_plan(elem_bytes, m, n, k, A, lda, B, ldb, C, ldc, num_cu=0,
                     kernel=-1, split=-1) -> dict
    igemm_conv2d_i16 / igemm_conv2d_i8(desc, X, W, Y, stream=None)
    igemm_conv2d_ex(elem_bytes, desc, X, W, Y, stream=None, kernel=-1, split=-1)
    igemm_conv2d_query_plan(elem_bytes, desc, X=None, W=None, Y=None, num_cu=0,
                            kernel=-1, split=-1) -> dict
    igemm_conv2d_out_dim(in, f, stride, pad, dil)
    igemm_i16_srs / igemm_i8_srs(m, n, k, A, lda, B, ldb, C, ldc, kc=0, shift=0,
                                 round_half_up=0, stream=None)
    igemm_srs_ex(elem_bytes, ..., stream=None, kernel=-1)
    igemm_srs_query(elem_bytes, m, n, k, A, lda, B, ldb, C, ldc, kc=0, num_cu=0,
                    kernel=-1) -> workspace bytes
    igemm_srs_ws(elem_bytes, ..., stream=None, kernel=-1, workspace=None,
                 workspace_bytes=0)
    igemm_strerror(status), igemm_kernel_name(i), igemm_num_kernels(),
    igemm_version()
and of include/igemm_rows.h (RouteDesc, GroupedDesc, AdaptersDesc for its
descriptors):
    igemm_route_query(desc), igemm_i8_grouped_query(desc, num_cu=0),
    igemm_i8_adapters_query(desc, num_cu=0) -> workspace bytes
    igemm_route(desc, logits, ld, bias, ids, weights, offsets, order,
                workspace=None, workspace_bytes=0, stream=None)
    igemm_i8_grouped(desc, offsets, order, A, lda, scale_a, B, ldb, stride_b, scale_b,
                     out, ldo, workspace=None, workspace_bytes=0, stream=None)
    igemm_combine(tokens, top_k, n, type, Z, ldz, weights, ids, base, ld_base, out,
                  ldo, stream=None)
    igemm_i8_adapters(desc, A, lda, scale_a, B, ldb, scale_b, ids, down, ld_down,
                      stride_down, up, ld_up, stride_up, ranks, scaling, out, ldo,
                      workspace=None, workspace_bytes=0, stream=None)
A, B, C may be integer device addresses or torch tensors (their data_ptr()).
Tensor conveniences: gemm_i16(A, B, C) and gemm_i8(A, B, C) take 2-D CUDA
tensors with unit stride along rows and update C in place; gemm_srs(A, B, C,
kc, shift, round_half_up) the same with an int16 C; conv2d(X, W, Y,
stride, pad, dil) takes contiguous NHWC / (r, s, c, k) / NHWC tensors; route,
grouped_i8 and combine are a sparse layer's routing, its experts' products and
the sum of a token's results, adapters_i8 a projection with the low-rank
adapters of many requests; a workspace the
call needs is taken from torch's caching allocator (so the calls can be
captured into a torch CUDA graph) and recorded on the stream the call runs
on; the library itself allocates nothing.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libigemm.so")

IGEMM_OK = 0
IGEMM_EINVAL = -1
IGEMM_EHIP = -2
IGEMM_ENOTSUP = -3
IGEMM_ENOMEM = -4
IGEMM_ESCRATCH = -5
IGEMM_NOALLOC_SCRATCH_BYTES = 72 << 20


class IgemmError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {igemm_strerror(status)} (status {status})")
        self.status = status


class _Plan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int), ("elem_bytes", ctypes.c_int),
                ("bm", ctypes.c_int), ("bn", ctypes.c_int), ("bk", ctypes.c_int),
                ("split", ctypes.c_int), ("k_chunk", ctypes.c_int64),
                ("tiles", ctypes.c_int64), ("grid", ctypes.c_int64),
                ("threads", ctypes.c_int), ("vec_a", ctypes.c_int), ("vec_b", ctypes.c_int),
                ("limb_products", ctypes.c_int), ("packed", ctypes.c_int),
                ("workspace_bytes", ctypes.c_int64), ("packed_a_bytes", ctypes.c_int64),
                ("packed_b_bytes", ctypes.c_int64)]


class ConvDesc(ctypes.Structure):
    """igemm_conv2d_desc: input n x h x w x c (NHWC), k output channels,
    r x s filters, strides, zero padding and dilations."""
    _fields_ = [(f, ctypes.c_int64) for f in
                ("n", "h", "w", "c", "k", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w",
                 "dil_h", "dil_w")]


class RouteDesc(ctypes.Structure):
    """igemm_route_desc."""
    _fields_ = [("tokens", ctypes.c_int64)] + \
        [(f, ctypes.c_int) for f in ("experts", "top_k", "groups", "top_groups", "group_best",
                                     "score", "renormalise")] + \
        [("scale", ctypes.c_float), ("type", ctypes.c_int)]


class GroupedDesc(ctypes.Structure):
    """igemm_grouped_desc."""
    _fields_ = [(f, ctypes.c_int64) for f in ("rows", "n", "k", "groups", "a_rows", "out_rows",
                                              "slots")] + \
        [("scatter", ctypes.c_int), ("type", ctypes.c_int)]


class AdaptersDesc(ctypes.Structure):
    """igemm_adapters_desc."""
    _fields_ = [(f, ctypes.c_int64) for f in ("m", "n", "k", "adapters", "rank")] + \
        [("type", ctypes.c_int), ("weight_type", ctypes.c_int)]


def conv_desc(n, h, w, c, k, r, s, stride=(1, 1), pad=(0, 0), dil=(1, 1)) -> ConvDesc:
    return ConvDesc(int(n), int(h), int(w), int(c), int(k), int(r), int(s), int(stride[0]),
                    int(stride[1]), int(pad[0]), int(pad[1]), int(dil[0]), int(dil[1]))


def _load():
    # torch ships its own HIP runtime whose DT_NEEDED name differs from the
    # soname this library links against; loading torch first lets the dynamic
    # linker bind both to that one runtime, so torch's streams and allocations
    # are valid handles for this library's launches.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "or `python -m paper_2302_07594_amd.build` (the HIP library has no fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    gemm_args = [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp]
    for name in ("igemm_i16", "igemm_i8"):
        getattr(lib, name).argtypes = gemm_args
        getattr(lib, name).restype = ci
        getattr(lib, name + "_ex").argtypes = gemm_args + [ci, ci]
        getattr(lib, name + "_ex").restype = ci
        getattr(lib, name + "_ws").argtypes = gemm_args + [ci, ci, vp, i64]
        getattr(lib, name + "_ws").restype = ci
    lib.igemm_i16_noalloc.argtypes = gemm_args + [ci, ci]
    lib.igemm_i16_noalloc.restype = ci
    for name in ("igemm_pack_i16", "igemm_pack_i8"):
        getattr(lib, name).argtypes = [i64, i64, i64, vp, i64, vp, i64, ci, vp, i64, vp]
        getattr(lib, name).restype = ci
    for name in ("igemm_i16_prepacked", "igemm_i8_prepacked"):
        getattr(lib, name).argtypes = [i64, i64, i64, vp, i64, vp, i64, ci, vp, i64, vp]
        getattr(lib, name).restype = ci
    for name in ("igemm_pack_b_i16", "igemm_pack_b_i8"):
        getattr(lib, name).argtypes = [i64, i64, vp, i64, ci, vp, i64, vp]
        getattr(lib, name).restype = ci
    for name in ("igemm_i16_packed_b", "igemm_i8_packed_b"):
        getattr(lib, name).argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, ci, vp, i64, vp]
        getattr(lib, name).restype = ci
    cd = ctypes.POINTER(ConvDesc)
    lib.igemm_conv2d_i16.argtypes = [cd, vp, vp, vp, vp]
    lib.igemm_conv2d_i16.restype = ci
    lib.igemm_conv2d_i8.argtypes = [cd, vp, vp, vp, vp]
    lib.igemm_conv2d_i8.restype = ci
    lib.igemm_conv2d_ex.argtypes = [ci, cd, vp, vp, vp, vp, ci, ci]
    lib.igemm_conv2d_ex.restype = ci
    lib.igemm_conv2d_query_plan.argtypes = [ci, cd, vp, vp, vp, ci, ci, ci,
                                            ctypes.POINTER(_Plan)]
    lib.igemm_conv2d_query_plan.restype = ci
    for name in ("igemm_i16_srs", "igemm_i8_srs"):
        getattr(lib, name).argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i64, ci, ci, vp]
        getattr(lib, name).restype = ci
    lib.igemm_srs_ex.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, vp, i64, i64, ci, ci, vp,
                                 ci]
    lib.igemm_srs_ex.restype = ci
    lib.igemm_srs_query.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, vp, i64, i64, ci, ci,
                                    ctypes.POINTER(i64)]
    lib.igemm_srs_query.restype = ci
    lib.igemm_srs_ws.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, vp, i64, i64, ci, ci, vp,
                                 ci, vp, i64]
    lib.igemm_srs_ws.restype = ci
    rd, gd = ctypes.POINTER(RouteDesc), ctypes.POINTER(GroupedDesc)
    ad = ctypes.POINTER(AdaptersDesc)
    for name, args in (
            ("igemm_route_query", [rd, ctypes.POINTER(i64)]),
            ("igemm_route", [rd, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp]),
            ("igemm_i8_grouped_query", [gd, ci, ctypes.POINTER(i64)]),
            ("igemm_i8_grouped", [gd, vp, vp, vp, i64, vp, vp, i64, i64, vp, vp, i64, vp, i64,
                                  vp]),
            ("igemm_combine", [i64, i64, i64, ci, vp, i64, vp, vp, vp, i64, vp, i64, vp]),
            ("igemm_i8_adapters_query", [ad, ci, ctypes.POINTER(i64)]),
            ("igemm_i8_adapters", [ad, vp, i64, vp, vp, i64, vp, vp, vp, i64, i64, vp, i64, i64,
                                   vp, vp, vp, i64, vp, i64, vp])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ci
    lib.igemm_conv2d_out_dim.argtypes = [i64] * 5
    lib.igemm_conv2d_out_dim.restype = i64
    lib.igemm_query_plan.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, vp, i64, ci, ci, ci,
                                     ctypes.POINTER(_Plan)]
    lib.igemm_query_plan.restype = ci
    lib.igemm_strerror.argtypes = [ci]
    lib.igemm_strerror.restype = ctypes.c_char_p
    lib.igemm_kernel_name.argtypes = [ci]
    lib.igemm_kernel_name.restype = ctypes.c_char_p
    lib.igemm_num_kernels.argtypes = []
    lib.igemm_num_kernels.restype = ci
    lib.igemm_version.argtypes = []
    lib.igemm_version.restype = ci
    return lib


class _Lazy:
    """Loads libigemm.so on first attribute access."""
    _handle = None

    def __getattr__(self, name):
        if _Lazy._handle is None:
            _Lazy._handle = _load()
        return getattr(_Lazy._handle, name)


_lib = _Lazy()


def load() -> None:
    """Load the HIP library now (raises ImportError if it is not built)."""
    if _Lazy._handle is None:
        _Lazy._handle = _load()


_native = None  # the compiled binding of the tensor calls, loaded at the first one


def _load_native():
    """binding/igemm_torch.cpp: the plain case of the tensor calls in one step
    (checks, plan, workspace, call). Its functions return None for anything
    else, which the Python code below then handles."""
    global _native
    load()  # first, so that both bind to the library and runtime loaded there
    try:
        from . import _igemm_torch
    except ImportError as e:
        raise ImportError(f"{HERE}/_igemm_torch.so is not built or does not load ({e}); run "
                          "`python -m paper_2302_07594_amd.build`") from e
    _native = _igemm_torch
    return _native


def library_path() -> str:
    return LIB_PATH


def _addr(x) -> int:
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    raise TypeError(f"expected a device address or a tensor, got {type(x).__name__}")


def _stream(stream) -> int:
    if stream is None:
        import torch
        return int(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return stream
    if hasattr(stream, "cuda_stream"):
        return int(stream.cuda_stream)
    raise TypeError("stream must be None, an int handle or a torch stream")


def _call(name, m, n, k, A, lda, B, ldb, C, ldc, stream, *extra) -> int:
    fn = getattr(_lib, name)
    st = fn(int(m), int(n), int(k), _addr(A), int(lda), _addr(B), int(ldb), _addr(C), int(ldc),
            _stream(stream), *extra)
    return int(st)


def igemm_i16(m, n, k, A, lda, B, ldb, C, ldc, stream=None) -> int:
    """C += A.B, int16 operands, int32 wraparound C. Returns the status."""
    return _call("igemm_i16", m, n, k, A, lda, B, ldb, C, ldc, stream)


def igemm_i8(m, n, k, A, lda, B, ldb, C, ldc, stream=None) -> int:
    """C += A.B, int8 operands, int32 wraparound C. Returns the status."""
    return _call("igemm_i8", m, n, k, A, lda, B, ldb, C, ldc, stream)


def igemm_i16_ex(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1, split=-1) -> int:
    return _call("igemm_i16_ex", m, n, k, A, lda, B, ldb, C, ldc, stream, int(kernel), int(split))


def igemm_i8_ex(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1, split=-1) -> int:
    return _call("igemm_i8_ex", m, n, k, A, lda, B, ldb, C, ldc, stream, int(kernel), int(split))


def igemm_i16_ws(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1, split=-1,
                 workspace=None, workspace_bytes=0) -> int:
    return _call("igemm_i16_ws", m, n, k, A, lda, B, ldb, C, ldc, stream, int(kernel),
                 int(split), _addr(workspace), int(workspace_bytes))


def igemm_i8_ws(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1, split=-1,
                workspace=None, workspace_bytes=0) -> int:
    return _call("igemm_i8_ws", m, n, k, A, lda, B, ldb, C, ldc, stream, int(kernel),
                 int(split), _addr(workspace), int(workspace_bytes))


def igemm_i16_noalloc(m, n, k, A, lda, B, ldb, C, ldc, stream=None, kernel=-1,
                      split=-1) -> int:
    """igemm_i16_ws with the library's static scratch array as the workspace
    (no allocation; calls that overlap on one GPU race). Returns the status."""
    return _call("igemm_i16_noalloc", m, n, k, A, lda, B, ldb, C, ldc, stream, int(kernel),
                 int(split))


def igemm_pack_i16(m, n, k, A, lda, B, ldb, kernel=-1, workspace=None, workspace_bytes=0,
                   stream=None) -> int:
    return int(_lib.igemm_pack_i16(int(m), int(n), int(k), _addr(A), int(lda), _addr(B),
                                   int(ldb), int(kernel), _addr(workspace), int(workspace_bytes),
                                   _stream(stream)))


def igemm_pack_i8(m, n, k, A, lda, B, ldb, kernel=-1, workspace=None, workspace_bytes=0,
                  stream=None) -> int:
    return int(_lib.igemm_pack_i8(int(m), int(n), int(k), _addr(A), int(lda), _addr(B),
                                  int(ldb), int(kernel), _addr(workspace), int(workspace_bytes),
                                  _stream(stream)))


def igemm_i16_prepacked(m, n, k, A, lda, C, ldc, kernel=-1, workspace=None, workspace_bytes=0,
                        stream=None) -> int:
    return int(_lib.igemm_i16_prepacked(int(m), int(n), int(k), _addr(A), int(lda), _addr(C),
                                        int(ldc), int(kernel), _addr(workspace),
                                        int(workspace_bytes), _stream(stream)))


def igemm_i8_prepacked(m, n, k, A, lda, C, ldc, kernel=-1, workspace=None, workspace_bytes=0,
                       stream=None) -> int:
    return int(_lib.igemm_i8_prepacked(int(m), int(n), int(k), _addr(A), int(lda), _addr(C),
                                       int(ldc), int(kernel), _addr(workspace),
                                       int(workspace_bytes), _stream(stream)))


def igemm_pack_b_i16(n, k, B, ldb, kernel=-1, packed_b=None, packed_b_bytes=0,
                     stream=None) -> int:
    return int(_lib.igemm_pack_b_i16(int(n), int(k), _addr(B), int(ldb), int(kernel),
                                     _addr(packed_b), int(packed_b_bytes), _stream(stream)))


def igemm_pack_b_i8(n, k, B, ldb, kernel=-1, packed_b=None, packed_b_bytes=0,
                    stream=None) -> int:
    return int(_lib.igemm_pack_b_i8(int(n), int(k), _addr(B), int(ldb), int(kernel),
                                    _addr(packed_b), int(packed_b_bytes), _stream(stream)))


def igemm_i16_packed_b(m, n, k, A, lda, packed_b, packed_b_bytes, C, ldc, kernel=-1,
                       workspace=None, workspace_bytes=0, stream=None) -> int:
    return int(_lib.igemm_i16_packed_b(int(m), int(n), int(k), _addr(A), int(lda),
                                       _addr(packed_b), int(packed_b_bytes), _addr(C), int(ldc),
                                       int(kernel), _addr(workspace), int(workspace_bytes),
                                       _stream(stream)))


def igemm_i8_packed_b(m, n, k, A, lda, packed_b, packed_b_bytes, C, ldc, kernel=-1,
                      workspace=None, workspace_bytes=0, stream=None) -> int:
    return int(_lib.igemm_i8_packed_b(int(m), int(n), int(k), _addr(A), int(lda),
                                      _addr(packed_b), int(packed_b_bytes), _addr(C), int(ldc),
                                      int(kernel), _addr(workspace), int(workspace_bytes),
                                      _stream(stream)))


_PLACEHOLDER = 1 << 12  # aligned, non-NULL; the planner never dereferences it


def igemm_query_plan(elem_bytes, m, n, k, A=None, lda=None, B=None, ldb=None, C=None,
                     ldc=None, num_cu=0, kernel=-1, split=-1):
    """The launch the library would make (host-only). Returns a dict, or
    raises IgemmError for invalid arguments. Omitted pointers stand for
    16-byte aligned buffers."""
    A = _PLACEHOLDER if A is None else A
    B = _PLACEHOLDER if B is None else B
    C = _PLACEHOLDER if C is None else C
    lda = k if lda is None else lda
    ldb = n if ldb is None else ldb
    ldc = n if ldc is None else ldc
    p = _Plan()
    st = _lib.igemm_query_plan(int(elem_bytes), int(m), int(n), int(k), _addr(A), int(lda),
                               _addr(B), int(ldb), _addr(C), int(ldc), int(num_cu), int(kernel),
                               int(split), ctypes.byref(p))
    if st != IGEMM_OK:
        raise IgemmError(st, "igemm_query_plan")
    d = {f: getattr(p, f) for f, _ in _Plan._fields_}
    d["kernel_name"] = igemm_kernel_name(p.kernel) if p.kernel >= 0 else None
    return d


def igemm_strerror(status: int) -> str:
    return _lib.igemm_strerror(int(status)).decode()


def igemm_kernel_name(kernel: int):
    r = _lib.igemm_kernel_name(int(kernel))
    return r.decode() if r is not None else None


def igemm_num_kernels() -> int:
    return int(_lib.igemm_num_kernels())


def igemm_version() -> int:
    return int(_lib.igemm_version())


def kernels_for(elem_bytes: int):
    """Indices of the kernels that take operands of ``elem_bytes`` bytes."""
    out = []
    for i in range(igemm_num_kernels()):
        nm = igemm_kernel_name(i)
        if (elem_bytes == 2) == nm.startswith("i16"):
            out.append(i)
    return out


def _check_tensors(A, B, C, torch_dtype, name):
    import torch
    if A.dtype != torch_dtype or B.dtype != torch_dtype:
        raise TypeError(f"{name}: A and B must be {torch_dtype}")
    if C.dtype != torch.int32:
        raise TypeError(f"{name}: C must be torch.int32")
    if A.dim() != 2 or B.dim() != 2 or C.dim() != 2:
        raise ValueError(f"{name}: A, B and C must be 2-D")
    m, k = A.shape
    k2, n = B.shape
    if k2 != k or tuple(C.shape) != (m, n):
        raise ValueError(f"{name}: shapes {tuple(A.shape)} x {tuple(B.shape)} -> {tuple(C.shape)}")
    for t, nm in ((A, "A"), (B, "B"), (C, "C")):
        if not t.is_cuda:
            raise ValueError(f"{name}: {nm} must be a CUDA (HIP) tensor")
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: {nm} must have unit stride along rows")

    def ld(t):
        return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)
    return m, n, k, ld(A), ld(B), ld(C)


_num_cu_cache = {}


def _num_cu(device) -> int:
    import torch
    idx = device.index if device.index is not None else torch.cuda.current_device()
    if idx not in _num_cu_cache:
        _num_cu_cache[idx] = torch.cuda.get_device_properties(idx).multi_processor_count
    return _num_cu_cache[idx]


def _aligned_workspace(nbytes, device, stream=None):
    """A uint8 device tensor of nbytes from torch's caching allocator,
    256-byte aligned. It is allocated on torch's current stream and recorded
    on `stream` when the call runs elsewhere (a torch stream, or a raw HIP
    stream handle, wrapped as an external stream), so that the allocator does
    not hand its memory to other work before the call's kernels are done."""
    import torch
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    if stream is not None:
        if isinstance(stream, int):
            if stream != int(torch.cuda.current_stream(device).cuda_stream):
                ws.record_stream(torch.cuda.ExternalStream(stream, device=device))
        elif hasattr(stream, "cuda_stream"):
            ws.record_stream(stream)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + nbytes]


def _gemm(es, A, B, C, stream, kernel, split, workspace, name):
    import torch
    m, n, k, lda, ldb, ldc = _check_tensors(A, B, C, torch.int16 if es == 2 else torch.int8, name)
    fn = igemm_i16_ws if es == 2 else igemm_i8_ws
    ws, ws_bytes = None, 0
    if workspace is None or workspace == "torch":
        if m and n and k:
            plan = igemm_query_plan(es, m, n, k, A, lda, B, ldb, C, ldc, _num_cu(C.device),
                                    kernel, split)
            if plan["workspace_bytes"] > 0:
                ws_bytes = plan["workspace_bytes"]
                ws = _aligned_workspace(ws_bytes, C.device, stream)
    elif workspace == "none":
        pass
    elif hasattr(workspace, "data_ptr"):
        ws, ws_bytes = workspace, workspace.numel() * workspace.element_size()
    else:
        raise ValueError(f"{name}: workspace must be None, 'torch', 'none' or a tensor")
    st = fn(m, n, k, A, lda, B, ldb, C, ldc, stream, kernel, split, ws, ws_bytes)
    if st != IGEMM_OK:
        raise IgemmError(st, name)
    return C


class Packed:
    """Packed operands of C += A.B (pack once, multiply many times).

    Holds the device workspace written by igemm_pack_*, the shape and the A
    it was packed with (int8 plans may read A in place)."""

    def __init__(self, es, m, n, k, A, lda, kernel, workspace, nbytes):
        self.es, self.m, self.n, self.k = es, m, n, k
        self.A, self.lda, self.kernel = A, lda, kernel
        self.workspace, self.nbytes = workspace, nbytes


def _packed_kernel(es):
    want = "i16_packed_128x128" if es == 2 else "i8_packed_256x256"
    return [i for i in range(igemm_num_kernels()) if igemm_kernel_name(i) == want][0]


def pack(A, B, stream=None):
    """Pack the operands of C += A.B (2-D torch.int16 or torch.int8 CUDA
    tensors, unit stride along rows). Returns a Packed object for
    gemm_prepacked; A must stay alive and unchanged while it is used."""
    import torch
    if A.dtype not in (torch.int16, torch.int8) or B.dtype != A.dtype:
        raise TypeError("pack: A and B must both be torch.int16 or both torch.int8")
    es = 2 if A.dtype == torch.int16 else 1
    if A.dim() != 2 or B.dim() != 2 or A.shape[1] != B.shape[0]:
        raise ValueError(f"pack: shapes {tuple(A.shape)} x {tuple(B.shape)}")
    for t, nm in ((A, "A"), (B, "B")):
        if not t.is_cuda:
            raise ValueError(f"pack: {nm} must be a CUDA (HIP) tensor")
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"pack: {nm} must have unit stride along rows")
    m, k = A.shape
    n = B.shape[1]
    lda = A.stride(0) if m > 1 else max(k, 1)
    ldb = B.stride(0) if k > 1 else max(n, 1)
    kid = _packed_kernel(es)
    nbytes = 0
    if m and n and k:
        plan = igemm_query_plan(es, m, n, k, A, lda, B, ldb, None, n, _num_cu(A.device), kid)
        nbytes = plan["workspace_bytes"]
    ws = _aligned_workspace(max(nbytes, 1), A.device, stream)
    fn = igemm_pack_i16 if es == 2 else igemm_pack_i8
    st = fn(m, n, k, A, lda, B, ldb, kid, ws, nbytes, stream)
    if st != IGEMM_OK:
        raise IgemmError(st, "pack")
    return Packed(es, m, n, k, A, lda, kid, ws, nbytes)


def gemm_prepacked(P, C, stream=None):
    """C += A.B from operands packed by pack(); C is a torch.int32 CUDA
    tensor of shape (m, n) with unit stride along rows. Returns C."""
    import torch
    if C.dtype != torch.int32 or C.dim() != 2 or tuple(C.shape) != (P.m, P.n) or not C.is_cuda:
        raise ValueError("gemm_prepacked: C must be an int32 CUDA tensor of shape (m, n)")
    if C.shape[1] > 1 and C.stride(1) != 1:
        raise ValueError("gemm_prepacked: C must have unit stride along rows")
    ldc = C.stride(0) if C.shape[0] > 1 else max(C.shape[1], 1)
    fn = igemm_i16_prepacked if P.es == 2 else igemm_i8_prepacked
    st = fn(P.m, P.n, P.k, P.A, P.lda, C, ldc, P.kernel, P.workspace, P.nbytes, stream)
    if st != IGEMM_OK:
        raise IgemmError(st, "gemm_prepacked")
    return C


class PackedB:
    """The fixed operand B of C += A.B in packed form (pack once, multiply
    with any A of k columns). Holds the device buffer igemm_pack_b_* wrote."""

    def __init__(self, es, n, k, kernel, buf, nbytes):
        self.es, self.n, self.k, self.kernel = es, n, k, kernel
        self.buf, self.nbytes = buf, nbytes


def pack_b(B, stream=None):
    """Pack a 2-D torch.int16 or torch.int8 CUDA tensor B (k x n, unit stride
    along rows) for gemm_packed_b. Returns a PackedB."""
    import torch
    if B.dtype not in (torch.int16, torch.int8) or B.dim() != 2 or not B.is_cuda:
        raise TypeError("pack_b: B must be a 2-D torch.int16 or torch.int8 CUDA tensor")
    if B.shape[1] > 1 and B.stride(1) != 1:
        raise ValueError("pack_b: B must have unit stride along rows")
    es = 2 if B.dtype == torch.int16 else 1
    k, n = B.shape
    ldb = B.stride(0) if k > 1 else max(n, 1)
    kid = _packed_kernel(es)
    nbytes = 0
    if n and k:
        nbytes = igemm_query_plan(es, 1, n, k, None, k, B, ldb, None, n, _num_cu(B.device),
                                  kid)["packed_b_bytes"]
    buf = _aligned_workspace(max(nbytes, 1), B.device, stream)
    fn = igemm_pack_b_i16 if es == 2 else igemm_pack_b_i8
    st = fn(n, k, B, ldb, kid, buf, nbytes, stream)
    if st != IGEMM_OK:
        raise IgemmError(st, "pack_b")
    return PackedB(es, n, k, kid, buf, nbytes)


def gemm_packed_b(A, PB, C, stream=None):
    """C += A.B with B packed by pack_b: A is an m x k CUDA tensor of B's
    type, C an m x n torch.int32 CUDA tensor (unit stride along rows).
    A's packed copy takes memory from torch's caching allocator. Returns C."""
    if stream is None:
        st = (_native or _load_native()).packed_b(PB.es, A, PB.buf, PB.nbytes, PB.n, PB.k, C,
                                                  PB.kernel)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "gemm_packed_b")
            return C
    import torch
    want = torch.int16 if PB.es == 2 else torch.int8
    if A.dtype != want or A.dim() != 2 or A.shape[1] != PB.k or not A.is_cuda:
        raise ValueError(f"gemm_packed_b: A must be a {want} CUDA tensor with {PB.k} columns")
    m = A.shape[0]
    if C.dtype != torch.int32 or C.dim() != 2 or tuple(C.shape) != (m, PB.n) or not C.is_cuda:
        raise ValueError("gemm_packed_b: C must be an int32 CUDA tensor of shape (m, n)")
    for t, nm in ((A, "A"), (C, "C")):
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"gemm_packed_b: {nm} must have unit stride along rows")
    lda = A.stride(0) if m > 1 else max(PB.k, 1)
    ldc = C.stride(0) if m > 1 else max(PB.n, 1)
    ws, ws_bytes = None, 0
    if m and PB.n and PB.k:
        ws_bytes = igemm_query_plan(PB.es, m, PB.n, PB.k, A, lda, None, PB.n, C, ldc,
                                    _num_cu(C.device), PB.kernel)["packed_a_bytes"]
        if ws_bytes > 0:
            ws = _aligned_workspace(ws_bytes, C.device, stream)
    fn = igemm_i16_packed_b if PB.es == 2 else igemm_i8_packed_b
    st = fn(m, PB.n, PB.k, A, lda, PB.buf, PB.nbytes, C, ldc, PB.kernel, ws, ws_bytes, stream)
    if st != IGEMM_OK:
        raise IgemmError(st, "gemm_packed_b")
    return C


def gemm_i16(A, B, C, stream=None, kernel=-1, split=-1, workspace=None):
    """C += A.B for 2-D torch.int16 CUDA tensors A (m x k), B (k x n) and a
    torch.int32 C (m x n). Returns C. Raises IgemmError on a bad status.
    workspace: None / "torch" (a workspace from torch's allocator when the
    plan packs the operands), "none" (no workspace: the in-place kernels
    only) or a uint8 CUDA tensor (256-byte aligned) to use as is."""
    if stream is None and workspace is None:
        st = (_native or _load_native()).gemm(2, A, B, C, kernel, split)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "gemm_i16")
            return C
    return _gemm(2, A, B, C, stream, kernel, split, workspace, "gemm_i16")


def gemm_i8(A, B, C, stream=None, kernel=-1, split=-1, workspace=None):
    """C += A.B for 2-D torch.int8 CUDA tensors; see gemm_i16."""
    if stream is None and workspace is None:
        st = (_native or _load_native()).gemm(1, A, B, C, kernel, split)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "gemm_i8")
            return C
    return _gemm(1, A, B, C, stream, kernel, split, workspace, "gemm_i8")


# ---- int16-output update (shift-round-saturate per k block) -----------------

def igemm_i16_srs(m, n, k, A, lda, B, ldb, C, ldc, kc=0, shift=0, round_half_up=0,
                  stream=None) -> int:
    """int16 C += srs(A B) per k block (see include/igemm.h). Returns the status."""
    return int(_lib.igemm_i16_srs(m, n, k, _addr(A), lda, _addr(B), ldb, _addr(C), ldc, kc,
                                  int(shift), int(round_half_up), _stream(stream)))


def igemm_i8_srs(m, n, k, A, lda, B, ldb, C, ldc, kc=0, shift=0, round_half_up=0,
                 stream=None) -> int:
    return int(_lib.igemm_i8_srs(m, n, k, _addr(A), lda, _addr(B), ldb, _addr(C), ldc, kc,
                                 int(shift), int(round_half_up), _stream(stream)))


def igemm_srs_ex(elem_bytes, m, n, k, A, lda, B, ldb, C, ldc, kc=0, shift=0, round_half_up=0,
                 stream=None, kernel=-1) -> int:
    return int(_lib.igemm_srs_ex(int(elem_bytes), m, n, k, _addr(A), lda, _addr(B), ldb,
                                 _addr(C), ldc, kc, int(shift), int(round_half_up),
                                 _stream(stream), int(kernel)))


def igemm_srs_query(elem_bytes, m, n, k, A, lda, B, ldb, C, ldc, kc=0, num_cu=0,
                    kernel=-1) -> int:
    """Workspace bytes igemm_srs_ws asks for with these arguments (0: it has no
    packed path). Host only. Raises IgemmError for invalid arguments."""
    out = ctypes.c_int64(0)
    st = int(_lib.igemm_srs_query(int(elem_bytes), m, n, k, _addr(A), lda, _addr(B), ldb,
                                  _addr(C), ldc, kc, int(num_cu), int(kernel), ctypes.byref(out)))
    if st != IGEMM_OK:
        raise IgemmError(st, "igemm_srs_query")
    return int(out.value)


def igemm_srs_ws(elem_bytes, m, n, k, A, lda, B, ldb, C, ldc, kc=0, shift=0, round_half_up=0,
                 stream=None, kernel=-1, workspace=None, workspace_bytes=0) -> int:
    return int(_lib.igemm_srs_ws(int(elem_bytes), m, n, k, _addr(A), lda, _addr(B), ldb,
                                 _addr(C), ldc, kc, int(shift), int(round_half_up),
                                 _stream(stream), int(kernel),
                                 _addr(workspace) if workspace is not None else None,
                                 int(workspace_bytes)))


def gemm_srs(A, B, C, kc=0, shift=0, round_half_up=False, stream=None, kernel=-1,
             workspace=None):
    """int16 C += srs(A B) for 2-D CUDA tensors: A (m x k) and B (k x n) both
    torch.int16 or both torch.int8, C (m x n) torch.int16, rows with unit
    stride. Per block of kc k indices (0: all of k) the exact product is
    shifted right by `shift` (floor, or round-half-up), saturated to int16
    and added to C modulo 2^16. `workspace` as for gemm_i16: None or 'torch'
    (a workspace from torch's allocator when the packed path is taken, so the
    call may be captured into a graph), 'none' (A and B in place) or a
    uint8 tensor. Returns C."""
    if stream is None and workspace is None:
        st = (_native or _load_native()).srs(A, B, C, kc, shift, round_half_up, kernel)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "gemm_srs")
            return C
    import torch
    if A.dtype not in (torch.int16, torch.int8) or B.dtype != A.dtype:
        raise TypeError("gemm_srs: A and B must both be torch.int16 or both torch.int8")
    if C.dtype != torch.int16:
        raise TypeError("gemm_srs: C must be torch.int16")
    # the shared checks expect an int32 C: check a stand-in of C's shape
    stand_in = torch.empty_strided(C.shape, C.stride(), dtype=torch.int32, device=C.device)
    m, n, k, lda, ldb, ldc = _check_tensors(A, B, stand_in, A.dtype, "gemm_srs")
    es = 2 if A.dtype == torch.int16 else 1
    ws, ws_bytes = None, 0
    if workspace is None or workspace == "torch":
        if m and n and k:
            ws_bytes = igemm_srs_query(es, m, n, k, A, lda, B, ldb, C, ldc, kc,
                                       _num_cu(C.device), kernel)
            if ws_bytes > 0:
                ws = _aligned_workspace(ws_bytes, C.device, stream)
    elif workspace == "none":
        pass
    elif hasattr(workspace, "data_ptr"):
        ws, ws_bytes = workspace, workspace.numel() * workspace.element_size()
    else:
        raise ValueError("gemm_srs: workspace must be None, 'torch', 'none' or a tensor")
    st = igemm_srs_ws(es, m, n, k, A, lda, B, ldb, C, ldc, kc, shift,
                      1 if round_half_up else 0, stream, kernel, ws, ws_bytes)
    if st != IGEMM_OK:
        raise IgemmError(st, "gemm_srs")
    return C


# ---- convolution through its IM2ROW lowering --------------------------------

def igemm_conv2d_out_dim(size, f, stride=1, pad=0, dil=1) -> int:
    return int(_lib.igemm_conv2d_out_dim(int(size), int(f), int(stride), int(pad), int(dil)))


def igemm_conv2d_i16(desc, X, W, Y, stream=None) -> int:
    """Y += conv(X, W), int16 operands (see include/igemm.h). Returns the status."""
    return int(_lib.igemm_conv2d_i16(ctypes.byref(desc), _addr(X), _addr(W), _addr(Y),
                                     _stream(stream)))


def igemm_conv2d_i8(desc, X, W, Y, stream=None) -> int:
    return int(_lib.igemm_conv2d_i8(ctypes.byref(desc), _addr(X), _addr(W), _addr(Y),
                                    _stream(stream)))


def igemm_conv2d_ex(elem_bytes, desc, X, W, Y, stream=None, kernel=-1, split=-1) -> int:
    return int(_lib.igemm_conv2d_ex(int(elem_bytes), ctypes.byref(desc), _addr(X), _addr(W),
                                    _addr(Y), _stream(stream), int(kernel), int(split)))


def igemm_conv2d_query_plan(elem_bytes, desc, X=None, W=None, Y=None, num_cu=0, kernel=-1,
                            split=-1) -> dict:
    """Plan of the lowered GEMM (host-only); omitted pointers stand for
    16-byte aligned buffers."""
    p = _Plan()
    st = _lib.igemm_conv2d_query_plan(
        int(elem_bytes), ctypes.byref(desc), _addr(_PLACEHOLDER if X is None else X),
        _addr(_PLACEHOLDER if W is None else W), _addr(_PLACEHOLDER if Y is None else Y),
        int(num_cu), int(kernel), int(split), ctypes.byref(p))
    if st != IGEMM_OK:
        raise IgemmError(st, "igemm_conv2d_query_plan")
    d = {f: getattr(p, f) for f, _ in _Plan._fields_}
    d["kernel_name"] = igemm_kernel_name(p.kernel) if p.kernel >= 0 else None
    return d


def conv2d(X, W, Y, stride=(1, 1), pad=(0, 0), dil=(1, 1), stream=None, kernel=-1, split=-1):
    """Y += conv(X, W) on contiguous CUDA tensors: X n x h x w x c and W
    r x s x c x k (both torch.int16 or both torch.int8), Y n x oh x ow x k
    torch.int32. Returns Y; raises IgemmError on a bad status."""
    if stream is None:
        st = (_native or _load_native()).conv2d(X, W, Y, stride, pad, dil, kernel, split)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "conv2d")
            return Y
    import torch
    if X.dtype not in (torch.int16, torch.int8) or W.dtype != X.dtype:
        raise TypeError("conv2d: X and W must both be torch.int16 or both torch.int8")
    if Y.dtype != torch.int32:
        raise TypeError("conv2d: Y must be torch.int32")
    for t, nm in ((X, "X"), (W, "W"), (Y, "Y")):
        if t.dim() != 4 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"conv2d: {nm} must be a contiguous 4-D CUDA tensor")
    n, h, w, c = X.shape
    r, s, c2, k = W.shape
    oh = igemm_conv2d_out_dim(h, r, stride[0], pad[0], dil[0])
    ow = igemm_conv2d_out_dim(w, s, stride[1], pad[1], dil[1])
    if c2 != c or tuple(Y.shape) != (n, oh, ow, k):
        raise ValueError(f"conv2d: X {tuple(X.shape)}, W {tuple(W.shape)} need Y "
                         f"{(n, oh, ow, k)}, got {tuple(Y.shape)}")
    d = conv_desc(n, h, w, c, k, r, s, stride, pad, dil)
    st = igemm_conv2d_ex(2 if X.dtype == torch.int16 else 1, d, X, W, Y, stream, kernel, split)
    if st != IGEMM_OK:
        raise IgemmError(st, "conv2d")
    return Y


# ---- products whose rows choose their weights ----------------------------------

IGEMM_F32, IGEMM_BF16, IGEMM_F16 = 0, 1, 2
IGEMM_SOFTMAX, IGEMM_SIGMOID = 0, 1


def _query(name, desc, *args) -> int:
    out = ctypes.c_int64(0)
    st = int(getattr(_lib, name)(None if desc is None else ctypes.byref(desc), *args,
                                 ctypes.byref(out)))
    if st != IGEMM_OK:
        raise IgemmError(st, name)
    return int(out.value)


def igemm_route_query(desc) -> int:
    """Workspace bytes igemm_route needs. Host only; raises IgemmError for an
    invalid descriptor, as the two queries below."""
    return _query("igemm_route_query", desc)


def igemm_i8_grouped_query(desc, num_cu=0) -> int:
    return _query("igemm_i8_grouped_query", desc, int(num_cu))


def igemm_i8_adapters_query(desc, num_cu=0) -> int:
    return _query("igemm_i8_adapters_query", desc, int(num_cu))


def igemm_route(desc, logits, ld, bias, ids, weights, offsets, order, workspace=None,
                workspace_bytes=0, stream=None) -> int:
    """Routing (see include/igemm_rows.h). Returns the status."""
    return int(_lib.igemm_route(ctypes.byref(desc), _addr(logits), int(ld), _addr(bias),
                                _addr(ids), _addr(weights), _addr(offsets), _addr(order),
                                _addr(workspace), int(workspace_bytes), _stream(stream)))


def igemm_i8_grouped(desc, offsets, order, A, lda, scale_a, B, ldb, stride_b, scale_b, out, ldo,
                     workspace=None, workspace_bytes=0, stream=None) -> int:
    """The experts' products (see include/igemm_rows.h). Returns the status."""
    return int(_lib.igemm_i8_grouped(ctypes.byref(desc), _addr(offsets), _addr(order), _addr(A),
                                     int(lda), _addr(scale_a), _addr(B), int(ldb), int(stride_b),
                                     _addr(scale_b), _addr(out), int(ldo), _addr(workspace),
                                     int(workspace_bytes), _stream(stream)))


def igemm_combine(tokens, top_k, n, type, Z, ldz, weights, ids, base, ld_base, out, ldo,
                  stream=None) -> int:
    """The weighted sum of each token's slots. Returns the status."""
    return int(_lib.igemm_combine(int(tokens), int(top_k), int(n), int(type), _addr(Z), int(ldz),
                                  _addr(weights), _addr(ids), _addr(base), int(ld_base),
                                  _addr(out), int(ldo), _stream(stream)))


def igemm_i8_adapters(desc, A, lda, scale_a, B, ldb, scale_b, ids, down, ld_down, stride_down,
                      up, ld_up, stride_up, ranks, scaling, out, ldo, workspace=None,
                      workspace_bytes=0, stream=None) -> int:
    """A projection with adapters (see include/igemm_rows.h). Returns the status."""
    return int(_lib.igemm_i8_adapters(ctypes.byref(desc), _addr(A), int(lda), _addr(scale_a),
                                      _addr(B), int(ldb), _addr(scale_b), _addr(ids),
                                      _addr(down), int(ld_down), int(stride_down), _addr(up),
                                      int(ld_up), int(stride_up), _addr(ranks), _addr(scaling),
                                      _addr(out), int(ldo), _addr(workspace),
                                      int(workspace_bytes), _stream(stream)))


def _type_of(dtype, name, what):
    import torch
    types = {torch.float32: IGEMM_F32, torch.bfloat16: IGEMM_BF16, torch.float16: IGEMM_F16}
    if dtype not in types:
        raise TypeError(f"{name}: {what} must be torch.float32, bfloat16 or float16")
    return types[dtype]


@contextlib.contextmanager
def _on(device, stream):
    """The device of the tensors made current, and the stream the call runs on:
    the device's current one, or `stream` (a torch stream or a raw handle), made
    current too, so that what the call allocates and fills belongs to it."""
    import torch
    with torch.cuda.device(device):
        if stream is None:
            yield int(torch.cuda.current_stream().cuda_stream)
            return
        if not hasattr(stream, "cuda_stream") and not isinstance(stream, int):
            raise TypeError("stream must be None, an int handle or a torch stream")
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=device)
        if stream.device != device:
            raise ValueError("stream must be one of the tensors' device")
        with torch.cuda.stream(stream):
            yield int(stream.cuda_stream)


def _expect(name, what, t, dtypes, shape, device, rows=True):
    """Type, shape (None: any) and device of a tensor whose rows have unit stride;
    rows=False: it is dense. Returns the leading dimension of its last two."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError(f"{name}: {what} must be a tensor of {' or '.join(map(str, dtypes))}")
    if t.dim() != len(shape) or any(w is not None and s != w for s, w in zip(t.shape, shape)):
        want = ", ".join("any" if w is None else str(w) for w in shape)
        raise ValueError(f"{name}: {what} must have shape ({want}), got {tuple(t.shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name}: {what} must be a CUDA (HIP) tensor on the operands' device")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} has no backward pass: call it under torch.no_grad() or detach "
                         f"{what}")
    if t.is_floating_point() and \
            torch.autograd.forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has no forward-mode derivative: detach {what}")
    if t.numel() == 0:
        return max(t.shape[-1], 1)
    if not rows:
        if not t.is_contiguous():
            raise ValueError(f"{name}: {what} must be contiguous")
        return max(t.shape[-1], 1)
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: {what} must have unit stride along rows")
    ld = t.stride(-2) if t.dim() > 1 and t.shape[-2] > 1 else max(t.shape[-1], 1)
    return ld


def _wrote(t):
    """Autograd's note that t has been written (what it saved of t is out of date)."""
    import torch
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


def _c_int(name, x) -> int:
    """An argument that the C call takes as an int (ctypes would wrap a larger one)."""
    if not -2 ** 31 <= int(x) < 2 ** 31:
        raise ValueError(f"{name}: {x} does not fit a C int")
    return int(x)


def _space(name, workspace, nbytes, device):
    """(workspace, bytes): the caller's, or one from torch's caching allocator."""
    if workspace is None:
        return (_aligned_workspace(nbytes, device), nbytes) if nbytes > 0 else (None, 0)
    import torch
    if not isinstance(workspace, torch.Tensor) or workspace.device != device or \
            not workspace.is_contiguous():
        raise ValueError(f"{name}: workspace must be None or a contiguous tensor on the "
                         "operands' device")
    return workspace, workspace.numel() * workspace.element_size()


def route(logits, top_k, bias=None, groups=1, top_groups=1, group_best=1, score="softmax",
          renormalise=True, scale=1.0, plan=True, stream=None, workspace=None):
    """Choose top_k experts for every row of logits (tokens x experts, a CUDA tensor
    of float32, bfloat16 or float16 with unit stride along rows).

    score: "softmax" or "sigmoid"; bias: float32, one an expert, added to the scores
    for the choice only; groups, top_groups, group_best: the experts form `groups`
    runs, of which the top_groups with the largest sum of their group_best (1 or
    2) best stay; renormalise: the weights of a token add up to scale. Experts
    whose logit is -inf or NaN are not chosen; ties go to the lower index.

    Returns (ids, weights, offsets, order): int32 and float32 (tokens, top_k), with
    id -1 and weight 0 where no expert is left, and the plan that grouped_i8
    takes, int32 (experts + 1) and (tokens * top_k); plan=False leaves the plan
    out (None, None). workspace: None, or a contiguous tensor on the same device."""
    if stream is None and workspace is None and score in ("softmax", "sigmoid"):
        r = (_native or _load_native()).route(
            logits, top_k, bias, groups, top_groups, group_best, 1 if score == "sigmoid" else 0,
            1 if renormalise else 0, scale, 1 if plan else 0)
        if r is not None:
            if not isinstance(r, tuple):
                raise IgemmError(r, "route")
            return r
    import torch
    f = (torch.float32, torch.bfloat16, torch.float16)
    ld = _expect("route", "logits", logits, f, (None, None), None)
    tokens, experts = logits.shape
    if bias is not None:
        _expect("route", "bias", bias, (torch.float32,), (experts,), logits.device, rows=False)
    if score not in ("softmax", "sigmoid"):
        raise ValueError("route: score must be 'softmax' or 'sigmoid'")
    top_k, groups, top_groups, group_best = \
        (_c_int("route", x) for x in (top_k, groups, top_groups, group_best))
    desc = RouteDesc(tokens, experts, top_k, groups, top_groups, group_best,
                     IGEMM_SIGMOID if score == "sigmoid" else IGEMM_SOFTMAX,
                     1 if renormalise else 0, float(scale),
                     _type_of(logits.dtype, "route", "logits"))
    nbytes = igemm_route_query(desc)
    with _on(logits.device, stream) as s:
        new = dict(device=logits.device, dtype=torch.int32)
        ids = torch.empty((tokens, top_k), **new)
        weights = torch.empty((tokens, top_k), dtype=torch.float32, device=logits.device)
        offsets = torch.empty(experts + 1, **new) if plan else None
        order = torch.empty(tokens * top_k, **new) if plan else None
        ws, ws_bytes = _space("route", workspace, nbytes, logits.device)
        st = igemm_route(desc, logits, ld, bias, ids, weights, offsets, order, ws, ws_bytes, s)
    if st != IGEMM_OK:
        raise IgemmError(st, "route")
    return ids, weights, offsets, order


def grouped_i8(A, B, offsets, order=None, scale_a=None, scale_b=None, slots=0, scatter=False,
               rows=None, out=None, out_dtype=None, stream=None, workspace=None):
    """The experts' products: position i of group g (offsets[g] <= i < offsets[g + 1])
    multiplies a row of A with B[g].

    A: a_rows x k int8, B: groups x k x n int8 (each group's matrix with unit stride
    along rows), offsets: int32 (groups + 1), order: int32 (rows) or None (the
    positions themselves); scale_a float32 (a_rows), scale_b float32 (groups, n),
    or None. The row of A is the position, or order[i] // slots for slots > 0 (slots
    = top_k: the token); the row of out is the position, or order[i] with scatter.
    rows: the number of positions, if order is None (default: A's rows).

    out: (out_rows, n) float32, bfloat16 or float16 with unit stride along rows,
    overwritten where a position leads; None: a zeroed (rows, n) tensor of out_dtype
    (default bfloat16). Returns out. Raises IgemmError on a bad status."""
    if out is not None and out_dtype is None and rows is None and stream is None and \
            workspace is None:
        st = (_native or _load_native()).grouped(A, B, offsets, order, scale_a, scale_b, slots,
                                                 1 if scatter else 0, out)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "grouped_i8")
            return out
    import torch
    i8, i32, f32 = (torch.int8,), (torch.int32,), (torch.float32,)
    lda = _expect("grouped_i8", "A", A, i8, (None, None), None)
    a_rows, k = A.shape
    ldb = _expect("grouped_i8", "B", B, i8, (None, k, None), A.device)
    groups, _, n = B.shape
    stride_b = B.stride(0) if groups > 1 and B.numel() > 0 else 0
    _expect("grouped_i8", "offsets", offsets, i32, (groups + 1,), A.device, rows=False)
    if order is not None:
        _expect("grouped_i8", "order", order, i32, (rows,), A.device, rows=False)
        rows = order.shape[0]
    elif rows is None:
        rows = a_rows
    if scale_a is not None:
        _expect("grouped_i8", "scale_a", scale_a, f32, (a_rows,), A.device, rows=False)
    if scale_b is not None:
        _expect("grouped_i8", "scale_b", scale_b, f32, (groups, n), A.device, rows=False)
    f = (torch.float32, torch.bfloat16, torch.float16)
    if out is not None:
        _expect("grouped_i8", "out", out, f if out_dtype is None else (out_dtype,), (None, n),
                A.device)
    dtype = out.dtype if out is not None else (out_dtype or torch.bfloat16)
    with _on(A.device, stream) as s:
        if out is None:
            _type_of(dtype, "grouped_i8", "out_dtype")
            out = torch.zeros((rows, n), dtype=dtype, device=A.device)
        ldo = out.stride(0) if out.shape[0] > 1 and out.numel() > 0 else max(n, 1)
        desc = GroupedDesc(rows, n, k, groups, a_rows, out.shape[0], int(slots),
                           1 if scatter else 0, _type_of(dtype, "grouped_i8", "out"))
        nbytes = igemm_i8_grouped_query(desc, _num_cu(A.device))
        ws, ws_bytes = _space("grouped_i8", workspace, nbytes, A.device)
        st = igemm_i8_grouped(desc, offsets, order, A, lda, scale_a, B, ldb, stride_b, scale_b,
                              out, ldo, ws, ws_bytes, s)
    if st != IGEMM_OK:
        raise IgemmError(st, "grouped_i8")
    _wrote(out)
    return out


def combine(Z, weights, ids=None, base=None, out=None, stream=None):
    """out[t] = base[t] + the sum over j of weights[t, j] * Z[t * top_k + j], slots with
    ids[t, j] < 0 left out. Z: (tokens * top_k, n) float32, bfloat16 or float16, unit
    stride along rows; weights: float32 (tokens, top_k), contiguous; ids: int32 of
    that shape or None; base and out: (tokens, n) of Z's type (out may be base; None:
    a new tensor). Returns out."""
    if out is not None and stream is None:
        st = (_native or _load_native()).combine(Z, weights, ids, base, out)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "combine")
            return out
    import torch
    f = (torch.float32, torch.bfloat16, torch.float16)
    _expect("combine", "weights", weights, (torch.float32,), (None, None), None, rows=False)
    tokens, top_k = weights.shape
    dev = weights.device
    ldz = _expect("combine", "Z", Z, f, (tokens * top_k, None), dev)
    n = Z.shape[1]
    if ids is not None:
        _expect("combine", "ids", ids, (torch.int32,), (tokens, top_k), dev, rows=False)
    ld_base = 0
    if base is not None:
        ld_base = _expect("combine", "base", base, (Z.dtype,), (tokens, n), dev)
    if out is not None:
        _expect("combine", "out", out, (Z.dtype,), (tokens, n), dev)
    with _on(dev, stream) as s:
        if out is None:
            out = torch.empty((tokens, n), dtype=Z.dtype, device=dev)
        ldo = out.stride(0) if tokens > 1 and n > 0 else max(n, 1)
        st = igemm_combine(tokens, top_k, n, _type_of(Z.dtype, "combine", "Z"), Z, ldz, weights,
                           ids, base, ld_base, out, ldo, s)
    if st != IGEMM_OK:
        raise IgemmError(st, "combine")
    _wrote(out)
    return out


def adapters_i8(A, B, ids=None, down=None, up=None, scale_a=None, scale_b=None, ranks=None,
                scaling=None, out=None, out_dtype=None, stream=None, workspace=None):
    """The projection scale_a * scale_b * (A.B) of int8 A (m x k) and B (k x n) and, beside
    it, for row i with adapter a = ids[i] (-1: none),
    scaling[a] * (scale_a[i] * A[i] . down[a]^T) . up[a]^T.

    down: (adapters, rank, k) and up: (adapters, n, rank), both bfloat16 or both
    float16, unit stride along rows; ids: int32 (m); ranks: int32 (adapters) or
    None; scale_a float32 (m), scale_b float32 (n), scaling float32 (adapters), or
    None. ids, down and up are given together; without them: the projection alone.
    out: (m, n) float32, bfloat16 or float16 with unit stride along rows; None: a new
    tensor of out_dtype (default bfloat16). Returns out."""
    if out is not None and out_dtype is None and stream is None and workspace is None:
        st = (_native or _load_native()).adapters(A, B, ids, down, up, scale_a, scale_b, ranks,
                                                  scaling, out)
        if st is not None:
            if st != IGEMM_OK:
                raise IgemmError(st, "adapters_i8")
            return out
    import torch
    i8, i32, f32 = (torch.int8,), (torch.int32,), (torch.float32,)
    name = "adapters_i8"
    lda = _expect(name, "A", A, i8, (None, None), None)
    m, k = A.shape
    dev = A.device
    ldb = _expect(name, "B", B, i8, (k, None), dev)
    n = B.shape[1]
    if scale_a is not None:
        _expect(name, "scale_a", scale_a, f32, (m,), dev, rows=False)
    if scale_b is not None:
        _expect(name, "scale_b", scale_b, f32, (n,), dev, rows=False)
    given = [x is not None for x in (ids, down, up)]
    if any(given) != all(given):
        raise ValueError(f"{name}: ids, down and up are given together")
    adapters = rank = ld_down = ld_up = stride_down = stride_up = 0
    wt = IGEMM_BF16
    if all(given):
        h = (torch.bfloat16, torch.float16)
        ld_down = _expect(name, "down", down, h, (None, None, k), dev)
        adapters, rank, _ = down.shape
        ld_up = _expect(name, "up", up, (down.dtype,), (adapters, n, rank), dev)
        _expect(name, "ids", ids, i32, (m,), dev, rows=False)
        stride_down = down.stride(0) if adapters > 1 and down.numel() > 0 else 0
        stride_up = up.stride(0) if adapters > 1 and up.numel() > 0 else 0
        wt = _type_of(down.dtype, name, "down")
        if ranks is not None:
            _expect(name, "ranks", ranks, i32, (adapters,), dev, rows=False)
        if scaling is not None:
            _expect(name, "scaling", scaling, f32, (adapters,), dev, rows=False)
    f = (torch.float32, torch.bfloat16, torch.float16)
    if out is not None:
        _expect(name, "out", out, f if out_dtype is None else (out_dtype,), (m, n), dev)
    dtype = out.dtype if out is not None else (out_dtype or torch.bfloat16)
    desc = AdaptersDesc(m, n, k, adapters, rank, _type_of(dtype, name, "out_dtype"), wt)
    nbytes = igemm_i8_adapters_query(desc, _num_cu(dev))
    with _on(dev, stream) as s:
        if out is None:
            out = torch.empty((m, n), dtype=dtype, device=dev)
        ldo = out.stride(0) if m > 1 and n > 0 else max(n, 1)
        ws, ws_bytes = _space(name, workspace, nbytes, dev)
        st = igemm_i8_adapters(desc, A, lda, scale_a, B, ldb, scale_b, ids, down, ld_down,
                               stride_down, up, ld_up, stride_up, ranks, scaling, out, ldo, ws,
                               ws_bytes, s)
    if st != IGEMM_OK:
        raise IgemmError(st, name)
    _wrote(out)
    return out
