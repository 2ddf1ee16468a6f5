"""ctypes binding of libspmi.so.  Same names as the C ABI; argument marshalling only."""
import ctypes
import os
import struct

import torch

from . import build as _build

SP_DENSE, SP_COMPRESSED = 0, 1
SP_F32, SP_F64, SP_F16, SP_BF16 = 0, 1, 2, 3
SP_TUNE_SPMV_KERNEL, SP_TUNE_CSC_MODE, SP_TUNE_SPMM_KERNEL, SP_TUNE_PROFILE, SP_TUNE_SPGEMM_KERNEL = 1, 2, 3, 4, 5
SP_MAX_RANK = 8

STATUS_NAMES = ["SP_OK", "SP_ERR_NULL", "SP_ERR_RANK", "SP_ERR_LEVEL_TYPE", "SP_ERR_ORDERING", "SP_ERR_WIDTH",
                "SP_ERR_COORD_RANGE", "SP_ERR_DUPLICATE", "SP_ERR_SHAPE", "SP_ERR_DTYPE", "SP_ERR_UNSUPPORTED",
                "SP_ERR_TOO_LARGE", "SP_ERR_ALLOC", "SP_ERR_HIP"]

EXPORTS = ["sp_encode", "sp_encoding_free", "sp_pack", "sp_tensor_free", "sp_prepare", "sp_matmul", "sp_matmul_noalloc", "sp_pos", "sp_crd", "sp_values",
           "sp_unpack", "sp_convert", "sp_sddmm", "sp_prepare_attention", "sp_attention_workspace", "sp_attention", "sp_attention_grad", "sp_rotary", "sp_rotary_grad", "sp_rotary_frequencies",
           "sp_cache_bytes", "sp_cache_map", "sp_cache_store", "sp_cache_load", "sp_cache_attention_workspace", "sp_cache_attention", "sp_mttkrp", "sp_spgemm", "sp_add", "sp_tensor_info", "sp_tensor_tune", "sp_profile_read", "sp_stream_copy", "sp_stream_read", "sp_pack_sort_mode", "sp_status_str", "sp_last_hip_error"]

_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class SpInfo(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int), ("levelTypes", ctypes.c_int * SP_MAX_RANK), ("dimOrdering", ctypes.c_int * SP_MAX_RANK),
                ("posWidth", ctypes.c_int), ("crdWidth", ctypes.c_int), ("dtype", ctypes.c_int),
                ("shape", ctypes.c_int64 * SP_MAX_RANK), ("nnz", ctypes.c_int64), ("nvalues", ctypes.c_int64),
                ("maxSegment", ctypes.c_int64), ("storageBytes", ctypes.c_int64), ("derivedBytes", ctypes.c_int64),
                ("spmvKernel", ctypes.c_int), ("lazyPrepares", ctypes.c_int)]


class SpAttentionProblem(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("heads", ctypes.c_int), ("kvHeads", ctypes.c_int), ("headDim", ctypes.c_int), ("causal", ctypes.c_int),
                ("buckets", ctypes.c_int), ("maxDistance", ctypes.c_int), ("bidirectional", ctypes.c_int), ("scale", ctypes.c_double),
                ("Q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("hdq", ctypes.c_int64),
                ("K", ctypes.c_void_p), ("ldk", ctypes.c_int64), ("hdk", ctypes.c_int64),
                ("V", ctypes.c_void_p), ("ldv", ctypes.c_int64), ("hdv", ctypes.c_int64),
                ("qpos", ctypes.c_void_p), ("kpos", ctypes.c_void_p), ("table", ctypes.c_void_p), ("ldt", ctypes.c_int64)]


class SpAttentionGrads(ctypes.Structure):
    _fields_ = [("O", ctypes.c_void_p), ("ldo", ctypes.c_int64), ("hdo", ctypes.c_int64), ("lse", ctypes.c_void_p),
                ("dO", ctypes.c_void_p), ("lddo", ctypes.c_int64), ("hddo", ctypes.c_int64),
                ("dQ", ctypes.c_void_p), ("lddq", ctypes.c_int64), ("hddq", ctypes.c_int64),
                ("dK", ctypes.c_void_p), ("lddk", ctypes.c_int64), ("hddk", ctypes.c_int64),
                ("dV", ctypes.c_void_p), ("lddv", ctypes.c_int64), ("hddv", ctypes.c_int64),
                ("dTable", ctypes.c_void_p), ("lddt", ctypes.c_int64)]


class SpRotaryProblem(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("headDim", ctypes.c_int), ("rotDim", ctypes.c_int), ("interleaved", ctypes.c_int), ("scale", ctypes.c_double),
                ("tokens", ctypes.c_int64), ("position", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("heads", ctypes.c_int), ("kvHeads", ctypes.c_int),
                ("Q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("hdq", ctypes.c_int64),
                ("K", ctypes.c_void_p), ("ldk", ctypes.c_int64), ("hdk", ctypes.c_int64),
                ("Qout", ctypes.c_void_p), ("ldqo", ctypes.c_int64), ("hdqo", ctypes.c_int64),
                ("Kout", ctypes.c_void_p), ("ldko", ctypes.c_int64), ("hdko", ctypes.c_int64)]


class SpCache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("pageTokens", ctypes.c_int), ("kvHeads", ctypes.c_int), ("headDim", ctypes.c_int)]


class SpCacheStep(ctypes.Structure):
    _fields_ = [("requests", ctypes.c_int64), ("tokens", ctypes.c_int64), ("pages", ctypes.c_int64), ("pageTokens", ctypes.c_int),
                ("length", ctypes.c_void_p), ("added", ctypes.c_void_p), ("freePages", ctypes.c_void_p), ("freeCount", ctypes.c_int64),
                ("taken", ctypes.c_void_p), ("table", ctypes.c_void_p), ("ldt", ctypes.c_int64), ("width", ctypes.c_int64),
                ("lengthOut", ctypes.c_void_p), ("start", ctypes.c_void_p), ("position", ctypes.c_void_p), ("slot", ctypes.c_void_p), ("takenOut", ctypes.c_void_p)]


class SpCacheProblem(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("heads", ctypes.c_int), ("causal", ctypes.c_int), ("scale", ctypes.c_double),
                ("requests", ctypes.c_int64), ("tokens", ctypes.c_int64), ("Q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("hdq", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("ldt", ctypes.c_int64), ("width", ctypes.c_int64), ("length", ctypes.c_void_p), ("start", ctypes.c_void_p)]


class SpError(RuntimeError):
    def __init__(self, code, what=""):
        name = STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES) else str(code)
        extra = ""
        if code == 13 and _lib is not None:
            extra = " (hipError %d)" % _lib.sp_last_hip_error()
        super().__init__("%s%s %s" % (name, extra, what))
        self.code = code


_lib = None


def load_library():
    """Loads libspmi.so; builds it first when there is none or when a source or header is newer than it.  Fails loudly
    when it can neither be loaded nor built: there is no other path."""
    global _lib
    if _lib is not None:
        return _lib
    if _build.is_stale():
        _build.build()
    L = ctypes.CDLL(_build.LIB)
    vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    L.sp_encode.restype = ci
    L.sp_encode.argtypes = [ci, vp, vp, ci, ci, ctypes.POINTER(vp)]
    L.sp_encoding_free.restype = None
    L.sp_encoding_free.argtypes = [vp]
    L.sp_pack.restype = ci
    L.sp_pack.argtypes = [vp, vp, i64, vp, vp, ci, _ALLOC_FN, _FREE_FN, vp, vp, ctypes.POINTER(vp)]
    L.sp_tensor_free.restype = None
    L.sp_tensor_free.argtypes = [vp]
    L.sp_matmul.restype = ci
    L.sp_matmul.argtypes = [vp, vp, i64, i64, vp, i64, ci, vp]
    L.sp_matmul_noalloc.restype = ci
    L.sp_matmul_noalloc.argtypes = [vp, vp, i64, i64, vp, i64, ci, vp]
    L.sp_prepare.restype = ci
    L.sp_prepare.argtypes = [vp, i64, vp]
    for f in (L.sp_pos, L.sp_crd):
        f.restype = ci
        f.argtypes = [vp, ci, ctypes.POINTER(vp), ctypes.POINTER(i64)]
    L.sp_values.restype = ci
    L.sp_values.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(i64)]
    L.sp_unpack.restype = ci
    L.sp_unpack.argtypes = [vp, vp, vp, vp]
    L.sp_add.restype = ci
    L.sp_add.argtypes = [vp, vp, vp, vp, ctypes.POINTER(vp)]
    L.sp_spgemm.restype = ci
    L.sp_spgemm.argtypes = [vp, vp, vp, vp, ctypes.POINTER(vp)]
    L.sp_mttkrp.restype = ci
    L.sp_mttkrp.argtypes = [vp, vp, i64, vp, i64, i64, vp, i64, ci, vp]
    L.sp_sddmm.restype = ci
    L.sp_sddmm.argtypes = [vp, vp, i64, vp, i64, ci, i64, vp, vp]
    problem, grads, size = ctypes.POINTER(SpAttentionProblem), ctypes.POINTER(SpAttentionGrads), ctypes.c_size_t
    L.sp_prepare_attention.restype = ci
    L.sp_prepare_attention.argtypes = [vp, ci, vp]
    L.sp_attention_workspace.restype = ci
    L.sp_attention_workspace.argtypes = [vp, problem, ci, ctypes.POINTER(size)]
    L.sp_attention.restype = ci
    L.sp_attention.argtypes = [vp, problem, vp, i64, i64, vp, vp, size, vp]
    L.sp_attention_grad.restype = ci
    L.sp_attention_grad.argtypes = [vp, problem, grads, vp, size, vp]
    L.sp_rotary_frequencies.restype = ci
    L.sp_rotary_frequencies.argtypes = [ci, ctypes.c_double, ctypes.c_double, i64, ctypes.c_double, ctypes.c_double, vp]
    for f in (L.sp_rotary, L.sp_rotary_grad):
        f.restype = ci
        f.argtypes = [vp, vp]                # structures, or their bytes
    cache = ctypes.POINTER(SpCache)
    L.sp_cache_bytes.restype = ci
    L.sp_cache_bytes.argtypes = [cache, ctypes.POINTER(size)]
    L.sp_cache_map.restype = ci
    L.sp_cache_map.argtypes = [vp, vp]
    for f in (L.sp_cache_store, L.sp_cache_load):
        f.restype = ci
        f.argtypes = [cache, ci, i64, vp, vp, i64, i64, vp, i64, i64, vp]
    L.sp_cache_attention_workspace.restype = ci
    L.sp_cache_attention_workspace.argtypes = [cache, vp, ctypes.POINTER(size)]
    L.sp_cache_attention.restype = ci
    L.sp_cache_attention.argtypes = [cache, vp, vp, i64, i64, vp, vp, size, vp]
    L.sp_convert.restype = ci
    L.sp_convert.argtypes = [vp, vp, vp, ctypes.POINTER(vp)]
    L.sp_tensor_info.restype = ci
    L.sp_tensor_info.argtypes = [vp, ctypes.POINTER(SpInfo)]
    L.sp_tensor_tune.restype = ci
    L.sp_tensor_tune.argtypes = [vp, ci, i64]
    L.sp_profile_read.restype = ci
    L.sp_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    L.sp_stream_copy.restype = ci
    L.sp_stream_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
    L.sp_pack_sort_mode.restype = ci
    L.sp_pack_sort_mode.argtypes = [ci]
    L.sp_stream_read.restype = ci
    L.sp_stream_read.argtypes = [vp, ctypes.c_size_t, vp, vp]
    L.sp_status_str.restype = ctypes.c_char_p
    L.sp_status_str.argtypes = [ci]
    L.sp_last_hip_error.restype = ci
    L.sp_last_hip_error.argtypes = []
    _lib = L
    return L


def _check(code, what=""):
    if code != 0:
        raise SpError(code, what)


# torch's own names for the current device and the handle of its current stream; not part of its documented interface
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr():
    """The current stream of the current device, as torch.cuda.current_stream() has it, without building a Stream object for it
    where torch lets one (0.2 against 2.8 us; a small product's whole call 7.5 -> 4.4 us)."""
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return _raw_stream(_raw_device())


class _TorchAllocator:
    """Backs the library's allocator callbacks with torch's caching allocator (uint8 tensors kept alive by address)."""

    def __init__(self, device):
        self.device = device
        self.live = {}
        self.alloc_cb = _ALLOC_FN(self._alloc)
        self.free_cb = _FREE_FN(self._free)

    def _alloc(self, nbytes, _ctx):
        try:
            t = torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=self.device)
        except Exception:          # out of memory: the library turns NULL into SP_ERR_ALLOC
            return None
        self.live[t.data_ptr()] = t
        return t.data_ptr()

    def _free(self, ptr, _ctx):
        self.live.pop(ptr, None)


class Encoding:
    def __init__(self, handle, rank):
        self._h, self.rank = handle, rank

    def __del__(self):
        if self._h and _lib is not None:
            _lib.sp_encoding_free(self._h)
            self._h = None


class Tensor:
    def __init__(self, handle, allocator, dtype, device):
        self._h, self._allocator, self.dtype, self.device = handle, allocator, dtype, device
        self._sizes = None               # (rank, m, n), once asked for
        self._workspaces = {}            # bytes of workspace of the attention problems met so far

    def free(self):
        if self._h and _lib is not None:
            _lib.sp_tensor_free(self._h)
            self._h = None

    def __del__(self):
        self.free()


def sp_encode(level_types, dim_ordering=None, pos_width=0, crd_width=0, rank=None):
    L = load_library()
    rank = len(level_types) if rank is None else rank
    lt = (ctypes.c_int * max(len(level_types), 1))(*[int(x) for x in level_types])
    order = None
    if dim_ordering is not None:
        order = (ctypes.c_int * max(len(dim_ordering), 1))(*[int(x) for x in dim_ordering])
    h = ctypes.c_void_p()
    _check(L.sp_encode(rank, lt, order, pos_width, crd_width, ctypes.byref(h)), "in sp_encode")
    return Encoding(h, rank)


def _dt(t):
    if t.dtype == torch.float64:
        return SP_F64
    if t.dtype == torch.float32:
        return SP_F32
    return -1


def sp_pack(enc, shape, coords, values, allocator=None):
    """coords: one int64 device tensor per dimension; values: device tensor (f32/f64).  allocator: an object with
    alloc_cb / free_cb (ctypes callbacks) that outlives the tensor; default: torch's caching allocator."""
    L = load_library()
    assert values.is_cuda and all(c.is_cuda and c.dtype == torch.int64 and c.is_contiguous() for c in coords)
    assert values.is_contiguous()
    nnz = int(values.shape[0])
    shp = (ctypes.c_int64 * max(len(shape), 1))(*[int(s) for s in shape])
    carr = (ctypes.c_void_p * max(len(coords), 1))(*[c.data_ptr() for c in coords])
    allocator = allocator or _TorchAllocator(values.device)
    h = ctypes.c_void_p()
    code = L.sp_pack(enc._h, shp, nnz, carr, values.data_ptr(), _dt(values), allocator.alloc_cb, allocator.free_cb, None,
                     _stream_ptr(), ctypes.byref(h))
    _check(code, "in sp_pack")
    return Tensor(h, allocator, values.dtype, values.device)


def sp_prepare(A, N=1):
    """The inspector step: builds and keeps whatever a product of A with N columns needs (synchronises)."""
    L = load_library()
    _check(L.sp_prepare(A._h, int(N), _stream_ptr()), "in sp_prepare")
    return A


def sp_matmul(A, B, C, accumulate=False, N=None, ldb=None, ldc=None):
    """C = A.B (or C += A.B).  B: (n, N) or (n,), C: (m, N) or (m,), row-major device tensors of A's dtype."""
    L = load_library()
    assert B.is_cuda and C.is_cuda and B.dtype == A.dtype and C.dtype == A.dtype
    if N is None:
        N = 1 if B.dim() == 1 else int(B.shape[1])
    if ldb is None:
        ldb = 1 if B.dim() == 1 else int(B.stride(0))
    if ldc is None:
        ldc = 1 if C.dim() == 1 else int(C.stride(0))
    _check(L.sp_matmul(A._h, B.data_ptr(), N, ldb, C.data_ptr(), ldc, int(bool(accumulate)), _stream_ptr()), "in sp_matmul")
    return C


def sp_matmul_noalloc(A, B, C, accumulate=False):
    """sp_matmul through the entry point that allocates nothing (SpMM of a CSR / DCSR tensor, scratch inside the library)."""
    L = load_library()
    assert B.is_cuda and C.is_cuda and B.dtype == A.dtype and C.dtype == A.dtype and B.dim() == 2 and C.dim() == 2
    _check(L.sp_matmul_noalloc(A._h, B.data_ptr(), int(B.shape[1]), int(B.stride(0)), C.data_ptr(), int(C.stride(0)), int(bool(accumulate)),
                               _stream_ptr()), "in sp_matmul_noalloc")
    return C


_INT = {8: torch.int8, 16: torch.int16, 32: torch.int32, 64: torch.int64}


def sp_tensor_info(A):
    L = load_library()
    info = SpInfo()
    _check(L.sp_tensor_info(A._h, ctypes.byref(info)))
    return info


def _view(A, ptr, length, dtype):
    """Borrowed torch view of an array the library allocated through the tensor's allocator (valid until A is freed)."""
    if length == 0:
        return torch.empty(0, dtype=dtype, device=A.device)
    owner = A._allocator.live[ptr]
    return owner[: length * torch.empty(0, dtype=dtype).element_size()].view(dtype)


def sp_pos(A, level):
    """pos[level] as a borrowed device tensor (int32/int64)."""
    L = load_library()
    p, n = ctypes.c_void_p(), ctypes.c_int64()
    _check(L.sp_pos(A._h, level, ctypes.byref(p), ctypes.byref(n)), "in sp_pos")
    return _view(A, p.value, n.value, _INT[sp_tensor_info(A).posWidth])


def sp_crd(A, level):
    L = load_library()
    p, n = ctypes.c_void_p(), ctypes.c_int64()
    _check(L.sp_crd(A._h, level, ctypes.byref(p), ctypes.byref(n)), "in sp_crd")
    return _view(A, p.value, n.value, _INT[sp_tensor_info(A).crdWidth])


def sp_values(A):
    L = load_library()
    p, n = ctypes.c_void_p(), ctypes.c_int64()
    _check(L.sp_values(A._h, ctypes.byref(p), ctypes.byref(n)), "in sp_values")
    return _view(A, p.value, n.value, A.dtype)


def sp_unpack(A):
    """(coords per dimension, values): every stored position in storage order, as device tensors."""
    L = load_library()
    info = sp_tensor_info(A)
    n = info.nvalues
    coords = [torch.empty(n, dtype=torch.int64, device=A.device) for _ in range(info.rank)]
    vals = torch.empty(n, dtype=A.dtype, device=A.device)
    carr = (ctypes.c_void_p * info.rank)(*[c.data_ptr() for c in coords])
    _check(L.sp_unpack(A._h, carr, vals.data_ptr(), _stream_ptr()), "in sp_unpack")
    return coords, vals


def sp_sddmm(S, A, B, X=None, b_is_transposed=False):
    """X[p] = S.values[p] * (A @ B)[i, j] for every stored position p = (i, j) of S.  A: (m, K); B: (K, n), or (n, K) when
    b_is_transposed.  Returns X (storage order)."""
    L = load_library()
    assert A.is_cuda and B.is_cuda and A.dtype == S.dtype and B.dtype == S.dtype and A.dim() == 2 and B.dim() == 2
    K = int(A.shape[1])
    if X is None:
        X = torch.empty(sp_tensor_info(S).nvalues, dtype=S.dtype, device=S.device)
    _check(L.sp_sddmm(S._h, A.data_ptr(), int(A.stride(0)), B.data_ptr(), int(B.stride(0)), int(bool(b_is_transposed)), K,
                      X.data_ptr(), _stream_ptr()), "in sp_sddmm")
    return X


_ATTENTION_DT = {torch.float32: SP_F32, torch.float16: SP_F16, torch.bfloat16: SP_BF16}


def sp_prepare_attention(S, grad=False):
    """The inspector step of sp_attention (grad: and of sp_attention_grad) on the pattern of S; synchronises."""
    L = load_library()
    _attention_call(S, lambda: _check(L.sp_prepare_attention(S._h, int(bool(grad)), _stream_ptr()), "in sp_prepare_attention"))
    return S


def _rows_of_heads(t, name, S, dtype):
    """The address and strides of a (tokens, heads, d) tensor: the last dimension is contiguous, the other two are free."""
    st = t.stride()
    if len(st) != 3 or t.dtype != dtype or t.device != S.device or (st[2] != 1 and t.shape[2] > 1):
        raise ValueError("%s: a (tokens, heads, d) tensor of %s on %s with a contiguous last dimension, not %s %s strides %s on %s" % (
            name, dtype, S.device, t.dtype, tuple(t.shape), tuple(t.stride()), t.device))
    return t.data_ptr(), st[0], st[1]


def _attention_problem(S, Q, K, V, scale, causal, qpos, kpos, bias, max_distance, bidirectional):
    if S._sizes is None:
        info = sp_tensor_info(S)
        S._sizes = info.rank, info.shape[0], info.shape[1] if info.rank > 1 else 0
    rank, m, n = S._sizes
    if rank != 2:
        raise SpError(2, "in sp_attention")
    dtype = Q.dtype
    if dtype not in _ATTENTION_DT:
        raise SpError(9, "in sp_attention: %s" % dtype)
    q, k, v = _rows_of_heads(Q, "Q", S, dtype), _rows_of_heads(K, "K", S, dtype), _rows_of_heads(V, "V", S, dtype)
    (rows, heads, d), (cols, kv, dk) = Q.shape, K.shape
    if rows != m or cols != n or V.shape != K.shape or dk != d:
        raise ValueError("Q %s, K %s, V %s for a pattern of %d x %d" % (tuple(Q.shape), tuple(K.shape), tuple(V.shape), m, n))
    at, table = (None, None), (None, 0)
    buckets = 0
    if causal or bias is not None:
        for name, t, size in (("qpos", qpos, m), ("kpos", kpos, n)):
            if t is None or t.dtype != torch.int32 or t.device != S.device or tuple(t.shape) != (size,) or not t.is_contiguous():
                raise ValueError("%s: %d contiguous int32 positions on %s" % (name, size, S.device))
        at = qpos.data_ptr(), kpos.data_ptr()
    if bias is not None:
        if bias.dim() != 2 or bias.dtype != dtype or bias.device != S.device or bias.shape[1] != heads or (heads > 1 and bias.stride(1) != 1):
            raise ValueError("bias: a (buckets, heads) tensor of %s on %s" % (dtype, S.device))
        buckets = int(bias.shape[0])
        if buckets == 0:
            raise SpError(8, "in sp_attention: no buckets")
        table = bias.data_ptr(), max(bias.stride(0), heads) if buckets == 1 else bias.stride(0)
    return SpAttentionProblem(_ATTENTION_DT[dtype], heads, kv, d, 1 if causal else 0, buckets, int(max_distance), 1 if bidirectional else 0,
                              (float(d) ** -0.5 if d else 1.0) if scale is None else float(scale), *q, *k, *v, *at, *table)


def _attention_call(S, f):
    """f() with S's device current: the stream, the workspace and the launches are that device's."""
    if S.device.index is None or S.device.index == torch.cuda.current_device():
        return f()
    with torch.cuda.device(S.device):
        return f()


def _attention_workspace(L, S, p, grad):
    key = (grad, p.dtype, p.heads, p.kvHeads, p.headDim, p.buckets, p.bidirectional, p.maxDistance)
    size = S._workspaces.get(key)
    if size is None:
        need = ctypes.c_size_t()
        _check(L.sp_attention_workspace(S._h, ctypes.byref(p), grad, ctypes.byref(need)), "in sp_attention_workspace")
        size = S._workspaces[key] = need.value
    return torch.empty(size, dtype=torch.uint8, device=S.device) if size else None, size


def _attention_output(t, like, name):
    """An output of `like`'s shape: a new one, or the caller's (its rows must not overlap)."""
    if t is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    if t.shape != like.shape:
        raise ValueError("%s: shape %s, not %s" % (name, tuple(like.shape), tuple(t.shape)))
    return t


def sp_attention(S, Q, K, V, scale=None, causal=False, qpos=None, kpos=None, bias=None, max_distance=128, bidirectional=True, O=None, lse=None):
    """Attention of the rows of S (queries) to the columns each stores (keys).  Q: (m, heads, d); K, V: (n, kv heads, d), f32, f16 or bf16;
    scale: 1 / sqrt(d) unless given.  bias: (buckets, heads), the learned relative position bias; qpos (m), kpos (n): int32 positions,
    for the bias and for causal (only keys at positions up to the query's).  Returns O (m, heads, d) and lse (heads, m) f32."""
    L = load_library()

    def call():
        p = _attention_problem(S, Q, K, V, scale, causal, qpos, kpos, bias, max_distance, bidirectional)
        out = _attention_output(O, Q, "O")
        logs = torch.empty((Q.shape[1], Q.shape[0]), dtype=torch.float32, device=S.device) if lse is None else lse
        if tuple(logs.shape) != (Q.shape[1], Q.shape[0]) or logs.dtype != torch.float32 or not logs.is_contiguous() or logs.device != S.device:
            raise ValueError("lse: a contiguous f32 tensor of (heads, m)")
        o, ldo, hdo = _rows_of_heads(out, "O", S, Q.dtype)
        work, size = _attention_workspace(L, S, p, 0)
        _check(L.sp_attention(S._h, ctypes.byref(p), o, ldo, hdo, logs.data_ptr(), work.data_ptr() if size else None, size, _stream_ptr()), "in sp_attention")
        return out, logs
    return _attention_call(S, call)


def sp_attention_grad(S, Q, K, V, O, lse, dO, scale=None, causal=False, qpos=None, kpos=None, bias=None, max_distance=128, bidirectional=True,
                      dQ=None, dK=None, dV=None):
    """Gradients (dQ, dK, dV, dBias) for dO, the gradient with respect to O; O and lse are sp_attention's for the same arguments.
    dBias is None without a bias."""
    L = load_library()

    def call():
        p = _attention_problem(S, Q, K, V, scale, causal, qpos, kpos, bias, max_distance, bidirectional)
        if O.shape != Q.shape or dO.shape != Q.shape or tuple(lse.shape) != (Q.shape[1], Q.shape[0]) or lse.dtype != torch.float32 or \
                not lse.is_contiguous() or lse.device != S.device:
            raise ValueError("O and dO: Q's shape; lse: a contiguous f32 tensor of (heads, m)")
        g = SpAttentionGrads()
        out = [_attention_output(t, like, name) for t, like, name in ((dQ, Q, "dQ"), (dK, K, "dK"), (dV, V, "dV"))]
        g.O, g.ldo, g.hdo = _rows_of_heads(O, "O", S, Q.dtype)
        g.dO, g.lddo, g.hddo = _rows_of_heads(dO, "dO", S, Q.dtype)
        g.lse = lse.data_ptr()
        g.dQ, g.lddq, g.hddq = _rows_of_heads(out[0], "dQ", S, Q.dtype)
        g.dK, g.lddk, g.hddk = _rows_of_heads(out[1], "dK", S, Q.dtype)
        g.dV, g.lddv, g.hddv = _rows_of_heads(out[2], "dV", S, Q.dtype)
        dbias = None
        if bias is not None:
            dbias = torch.empty(bias.shape, dtype=bias.dtype, device=S.device)
            g.dTable, g.lddt = dbias.data_ptr(), int(bias.shape[1])
        work, size = _attention_workspace(L, S, p, 1)
        _check(L.sp_attention_grad(S._h, ctypes.byref(p), ctypes.byref(g), work.data_ptr() if size else None, size, _stream_ptr()), "in sp_attention_grad")
        return out[0], out[1], out[2], dbias
    return _attention_call(S, call)


# The same bytes as SpRotaryProblem, SpCacheStep and SpCacheProblem, made in a third of the time; a step of a serving loop makes one for each call.
# The structures name the fields: tests hold them to the header, and these formats to them.
_ROTARY, _STEP, _PROBLEM = struct.Struct("@iiiidqPPii" + "Pqq" * 4), struct.Struct("@qqqi" + "PPPqPPqqPPPPP"), struct.Struct("@iiidqqPqqPqqPP")


def _heads_of(t, name, dtype, index):
    """_rows_of_heads for a tensor on GPU number `index`, with little work where all is well."""
    st = t.stride()
    if len(st) != 3 or t.dtype is not dtype or t.get_device() != index or (st[2] != 1 and t.shape[2] > 1):
        raise ValueError("%s: a (tokens, heads, d) tensor of %s on GPU %d with a contiguous last dimension, not %s %s strides %s on %s" % (
            name, dtype, index, t.dtype, tuple(t.shape), tuple(st), t.device))
    return t.data_ptr(), st[0], st[1]


def _output_like(t, like, name):
    """An output of `like`'s shape: a new one, or the caller's (its rows must not overlap)."""
    if t is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    if t.shape != like.shape:
        raise ValueError("%s: shape %s, not %s" % (name, tuple(like.shape), tuple(t.shape)))
    return t


def _whole_numbers(t, name, size, index):
    """The address of `size` contiguous int32 numbers on GPU number `index`."""
    if t.dtype is not torch.int32 or t.get_device() != index or t.dim() != 1 or t.numel() != size or not t.is_contiguous():
        raise ValueError("%s: %d contiguous int32 numbers on GPU %d, not %s %s on %s" % (name, size, index, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _gpu_of(t):
    """The number of a tensor's GPU."""
    index = t.get_device()
    if index < 0:
        raise ValueError("a tensor on a GPU, not on %s" % t.device)
    return index


def _on_gpu(index, f, *args):
    """f(*args) with that GPU current: the stream, the workspace and the launches are that device's."""
    if index == torch.cuda.current_device():
        return f(*args)
    with torch.cuda.device(index):
        return f(*args)


def _rotary(grad, index, position, frequencies, Q, K, interleaved, scale, Q_out, K_out):
    L, dt = load_library(), Q.dtype
    code = _ATTENTION_DT.get(dt)
    if code is None:
        raise SpError(9, "in sp_rotary: %s" % dt)
    q = _heads_of(Q, "Q", dt, index)
    (tokens, heads, d), half = Q.shape, frequencies.numel()
    if frequencies.dtype is not torch.float64 or frequencies.get_device() != index or frequencies.dim() != 1 or not frequencies.is_contiguous():
        raise ValueError("frequencies: contiguous float64 numbers on GPU %d" % index)
    at = _whole_numbers(position, "position", tokens, index)
    q_out = _output_like(Q_out, Q, "Q_out")
    qo, k, ko, k_out, kv = _heads_of(q_out, "Q_out", dt, index), (0, 0, 0), (0, 0, 0), None, 0
    if K is not None:
        k = _heads_of(K, "K", dt, index)
        n, kv, dk = K.shape
        if n != tokens or dk != d:
            raise ValueError("K %s beside Q %s" % (tuple(K.shape), tuple(Q.shape)))
        k_out = _output_like(K_out, K, "K_out")
        ko = _heads_of(k_out, "K_out", dt, index)
    f = L.sp_rotary_grad if grad else L.sp_rotary
    _check(f(_ROTARY.pack(code, d, 2 * half, 1 if interleaved else 0, scale, tokens, at, frequencies.data_ptr(), heads, kv, *q, *k, *qo, *ko),
             _stream_ptr()), "in sp_rotary_grad" if grad else "in sp_rotary")
    return q_out if K is None else (q_out, k_out)


def sp_rotary(position, frequencies, Q, K=None, interleaved=False, scale=1.0, Q_out=None, K_out=None):
    """Q (tokens, heads, d) and, if given, K (tokens, kv heads, d) with their pairs turned by position * frequencies (int32 positions, f64 angles a
    position; the first 2 * len(frequencies) numbers of a head turn).  Returns the turned Q, or (Q, K): new tensors, or Q_out and K_out, which may
    be Q and K."""
    return _on_gpu(_gpu_of(Q), _rotary, False, Q.get_device(), position, frequencies, Q, K, interleaved, scale, Q_out, K_out)


def sp_rotary_grad(position, frequencies, dQ, dK=None, interleaved=False, scale=1.0, dQ_out=None, dK_out=None):
    """The gradients with respect to sp_rotary's Q and K, given those with respect to its results (the same arguments otherwise)."""
    return _on_gpu(_gpu_of(dQ), _rotary, True, dQ.get_device(), position, frequencies, dQ, dK, interleaved, scale, dQ_out, dK_out)


def sp_rotary_frequencies(rot_dim, base=10000.0, factor=1.0, trained=0, low=1.0, high=32.0, device=None):
    """base^(-2k / rot_dim) for k < rot_dim / 2 as f64 on `device` (the current GPU unless given), made smaller by `factor` for long contexts:
    all of them, or with trained > 0 those that make fewer than `high` turns in so many positions (wholly below `low`, partly between)."""
    rot_dim = int(rot_dim)
    f = (ctypes.c_double * max(1, rot_dim // 2))()
    _check(load_library().sp_rotary_frequencies(rot_dim, float(base), float(factor), int(trained), float(low), float(high), f), "in sp_rotary_frequencies")
    return torch.tensor(f[:rot_dim // 2], dtype=torch.float64, device="cuda" if device is None else device)


class Cache:
    """Keys and values in 4 bits: the pages' memory (`data`) and their description."""

    def __init__(self, data, spec):
        self._ref, self._index = ctypes.byref(spec), _gpu_of(data)       # tensors of the calls have to be on that GPU
        self.data, self._spec, self.device = data, spec, data.device
        self.pages, self.page_tokens, self.kv_heads, self.head_dim = spec.pages, spec.pageTokens, spec.kvHeads, spec.headDim
        self._workspaces = {}            # bytes of workspace of the attention problems met so far


def sp_cache(pages, page_tokens, kv_heads, head_dim, device=None):
    """A cache of `pages` pages of page_tokens tokens (a multiple of 16), filled with zeros, on `device`, a GPU (the current one unless given)."""
    device = torch.device("cuda" if device is None else device)
    if device.type != "cuda":
        raise ValueError("a cache on a GPU, not on %s" % device)
    spec, size = SpCache(None, int(pages), int(page_tokens), int(kv_heads), int(head_dim)), ctypes.c_size_t()
    _check(load_library().sp_cache_bytes(ctypes.byref(spec), ctypes.byref(size)), "in sp_cache")
    data = torch.zeros(max(1, size.value), dtype=torch.uint8, device=device)
    spec.data = data.data_ptr()
    return Cache(data, spec)


def _block_table(t, requests, index):
    """The address, row stride and width of a block table."""
    st = t.stride()
    if t.dtype is not torch.int32 or t.get_device() != index or len(st) != 2 or t.shape[0] != requests or (st[1] != 1 and t.shape[1] > 1):
        raise ValueError("table: int32 pages (%d, width) on GPU %d with contiguous rows, not %s %s strides %s on %s" % (
            requests, index, t.dtype, tuple(t.shape), st, t.device))
    width = t.shape[1]
    return t.data_ptr(), st[0] if requests > 1 else max(st[0], width), width


def sp_cache_map(lengths, added, free, taken, table, page_tokens, pages, tokens):
    """The pages and slots of a step.  lengths, added: (requests) int32, what each request has in the cache and gets; free: int32 pages to hand
    out, from number taken[0] on; table: (requests, width) int32, updated in place; tokens: rows of the step (sum of added, or more).
    Returns (lengths + added, start (requests + 1), position (tokens), slot (tokens), taken)."""
    return _on_gpu(_gpu_of(lengths), _cache_map, lengths, added, free, taken, table, page_tokens, pages, tokens)


def _cache_map(lengths, added, free, taken, table, page_tokens, pages, tokens):
    n, nfree, index, new = lengths.shape[0], free.shape[0], lengths.get_device(), lengths.new_empty
    at = (_whole_numbers(lengths, "lengths", n, index), _whole_numbers(added, "added", n, index), _whole_numbers(free, "free", nfree, index), nfree,
          _whole_numbers(taken, "taken", 1, index), *_block_table(table, n, index))
    if tokens < 0:
        raise SpError(8, "in sp_cache_map: %d tokens" % tokens)
    out = new(n), new(n + 1), new(tokens), new(tokens), new(1)
    _check(load_library().sp_cache_map(_STEP.pack(n, tokens, pages, page_tokens, *at, *[t.data_ptr() for t in out]), _stream_ptr()), "in sp_cache_map")
    return out


def _cache_rows(cache, t, name, tokens, dtype):
    row = _heads_of(t, name, dtype, cache._index)
    if t.shape[0] != tokens or t.shape[1] != cache.kv_heads or t.shape[2] != cache.head_dim:
        raise ValueError("%s: shape %s, not %s" % (name, (tokens, cache.kv_heads, cache.head_dim), tuple(t.shape)))
    return row


def sp_cache_store(cache, K, V, slots):
    """K and V (tokens, kv heads, d), f32, f16 or bf16, into the cache's slots (int32; -1: not stored), in 4 bits."""
    _on_gpu(cache._index, _cache_store, cache, K, V, slots)


def _cache_store(cache, K, V, slots):
    n, dt = K.shape[0], K.dtype
    code = _ATTENTION_DT.get(dt)
    if code is None:
        raise SpError(9, "in sp_cache_store: %s" % dt)
    k, v = _cache_rows(cache, K, "K", n, dt), _cache_rows(cache, V, "V", n, dt)
    _check(load_library().sp_cache_store(cache._ref, code, n, _whole_numbers(slots, "slots", n, cache._index), *k, *v, _stream_ptr()), "in sp_cache_store")


def sp_cache_load(cache, slots, dtype=torch.bfloat16, K=None, V=None):
    """What the cache's slots hold (int32; -1: zeros): K and V (tokens, kv heads, d) of `dtype`, new tensors or the given ones."""
    return _on_gpu(cache._index, _cache_load, cache, slots, dtype, K, V)


def _cache_load(cache, slots, dtype, K, V):
    code = _ATTENTION_DT.get(dtype)
    if code is None:
        raise SpError(9, "in sp_cache_load: %s" % dtype)
    n = slots.shape[0]
    at = _whole_numbers(slots, "slots", n, cache._index)
    if K is None:
        K = torch.empty((n, cache.kv_heads, cache.head_dim), dtype=dtype, device=cache.device)
    if V is None:
        V = torch.empty((n, cache.kv_heads, cache.head_dim), dtype=dtype, device=cache.device)
    k, v = _cache_rows(cache, K, "K", n, dtype), _cache_rows(cache, V, "V", n, dtype)
    _check(load_library().sp_cache_load(cache._ref, code, n, at, *k, *v, _stream_ptr()), "in sp_cache_load")
    return K, V


def sp_cache_attention(cache, Q, table, lengths, start, scale=None, causal=True, O=None, lse=None):
    """Attention over the cache.  Q: (tokens, heads, d), f32, f16 or bf16; request r's queries are rows start[r] .. start[r + 1] - 1, the last of its
    lengths[r] tokens in the pages of table[r] (all int32); scale: 1 / sqrt(d) unless given.  Returns O (tokens, heads, d) and lse (heads, tokens)
    f32; rows of no request are left as they were."""
    return _on_gpu(cache._index, _cache_attention, cache, Q, table, lengths, start, scale, causal, O, lse)


def _cache_attention(cache, Q, table, lengths, start, scale, causal, O, lse):
    L, dt, index = load_library(), Q.dtype, cache._index
    code = _ATTENTION_DT.get(dt)
    if code is None:
        raise SpError(9, "in sp_cache_attention: %s" % dt)
    q = _heads_of(Q, "Q", dt, index)
    tokens, heads, d = Q.shape
    if d != cache.head_dim:
        raise ValueError("Q %s for a cache of heads of %d" % (tuple(Q.shape), cache.head_dim))
    n = lengths.shape[0]
    at = _block_table(table, n, index)
    p = _PROBLEM.pack(code, heads, 1 if causal else 0, float(d) ** -0.5 if scale is None else scale, n, tokens, *q, *at,
                      _whole_numbers(lengths, "lengths", n, index), _whole_numbers(start, "start", n + 1, index))
    O = _output_like(O, Q, "O")
    if lse is None:
        lse = torch.empty((heads, tokens), dtype=torch.float32, device=cache.device)
    elif tuple(lse.shape) != (heads, tokens) or lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.get_device() != index:
        raise ValueError("lse: a contiguous f32 tensor of (heads, tokens)")
    o = _heads_of(O, "O", dt, index)
    key = (code, heads, n, tokens, at[2])
    size = cache._workspaces.get(key)
    if size is None:
        need = ctypes.c_size_t()
        _check(L.sp_cache_attention_workspace(cache._ref, p, ctypes.byref(need)), "in sp_cache_attention")
        if len(cache._workspaces) >= 1000:               # steps of ever other sizes
            cache._workspaces.clear()
        size = cache._workspaces[key] = need.value
    work = torch.empty(size, dtype=torch.uint8, device=cache.device) if size else None
    _check(L.sp_cache_attention(cache._ref, p, *o, lse.data_ptr(), work.data_ptr() if size else None, size, _stream_ptr()), "in sp_cache_attention")
    return O, lse


def sp_mttkrp(B, C, D, A=None, accumulate=False):
    """A[i,j] = sum_{k,l} B[i,k,l] * D[l,j] * C[k,j] for a packed rank-3 tensor B.  C: (K, J), D: (L, J); returns A (I, J)."""
    L = load_library()
    assert C.is_cuda and D.is_cuda and C.dtype == B.dtype and D.dtype == B.dtype and C.dim() == 2 and D.dim() == 2
    assert C.shape[1] == D.shape[1] and C.stride(1) == 1 and D.stride(1) == 1
    J = int(C.shape[1])
    info = sp_tensor_info(B)
    if A is None:
        assert not accumulate
        A = torch.empty((info.shape[0], J), dtype=B.dtype, device=B.device)
    assert A.is_cuda and A.dtype == B.dtype and A.shape == (info.shape[0], J) and (J == 0 or A.stride(1) == 1)
    _check(L.sp_mttkrp(B._h, C.data_ptr(), int(C.stride(0)), D.data_ptr(), int(D.stride(0)), J,
                       A.data_ptr(), int(A.stride(0)), int(bool(accumulate)), _stream_ptr()), "in sp_mttkrp")
    return A


def sp_convert(A, enc):
    """A new tensor with A's stored entries under another encoding."""
    h = ctypes.c_void_p()
    _check(load_library().sp_convert(A._h, enc._h, _stream_ptr(), ctypes.byref(h)), "in sp_convert")
    return Tensor(h, A._allocator, A.dtype, A.device)


def sp_spgemm(A, B, enc):
    """C = A.B for two packed sparse matrices, as a new tensor under `enc` (it lives in A's allocator)."""
    h = ctypes.c_void_p()
    _check(load_library().sp_spgemm(A._h, B._h, enc._h, _stream_ptr(), ctypes.byref(h)), "in sp_spgemm")
    return Tensor(h, A._allocator, A.dtype, A.device)


def sp_add(A, B, enc):
    """C = A + B element by element, as a new tensor under `enc` (it lives in A's allocator)."""
    h = ctypes.c_void_p()
    _check(load_library().sp_add(A._h, B._h, enc._h, _stream_ptr(), ctypes.byref(h)), "in sp_add")
    return Tensor(h, A._allocator, A.dtype, A.device)


def sp_tensor_tune(A, key, value):
    _check(load_library().sp_tensor_tune(A._h, key, value), "in sp_tensor_tune")


def sp_profile_read(A):
    """(total milliseconds, launches) of the main kernels recorded since the last read."""
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(load_library().sp_profile_read(A._h, ctypes.byref(ms), ctypes.byref(n)), "in sp_profile_read")
    return ms.value, n.value


def sp_stream_copy(dst, src):
    nbytes = src.numel() * src.element_size()
    _check(load_library().sp_stream_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream_ptr()), "in sp_stream_copy")


def sp_stream_read(src, sink):
    nbytes = src.numel() * src.element_size()
    _check(load_library().sp_stream_read(src.data_ptr(), nbytes, sink.data_ptr(), _stream_ptr()), "in sp_stream_read")


def sp_pack_sort_mode(mode):
    """0 = the storage builder chooses its sort, 1 = least significant digit first, 2 = most significant digit first."""
    _check(load_library().sp_pack_sort_mode(int(mode)), "in sp_pack_sort_mode")
