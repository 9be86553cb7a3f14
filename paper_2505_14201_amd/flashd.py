"""Thin binding over libflashd.so: argument marshalling only (ctypes, and for the calls of the
serving path a native module in front of it).

Function names mirror the C ABI in include/flashd.h.  Tensors are torch CUDA
(ROCm) tensors used purely as owners of device memory; every step of the
computation runs inside the library's HIP kernels.  There is no fallback for them: if the
shared library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
import sys
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflashd.so")

F32, F16, BF16 = 0, 1, 2
VARIANT_AUTO, VARIANT_TILE, VARIANT_PER_KEY, VARIANT_ONLINE_SOFTMAX, VARIANT_TILE_BLEND = 0, 1, 2, 3, 4
VARIANT_TILE_256 = 5
MAX_SPLITS = 64
STATIC_SCRATCH_BYTES = 32 << 20

CACHE_FP8 = 3
CACHE_MAX_SEQS = 4096

_DTYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_CACHE_DTYPE = {**_DTYPE, torch.float8_e4m3fn: CACHE_FP8}

EXPORTS = ("flashd_attn_fwd", "flashd_attn_fwd_ex", "flashd_workspace_bytes",
           "flashd_auto_splits", "flashd_auto_variant", "flashd_status_string", "flashd_version", "flashd_skip_stats", "flashd_attn_fwd_state",
           "flashd_attn_fwd_kv8", "flashd_attn_fwd_static", "flashd_attn_fwd_skipv",
           "flashd_release_workspace", "flashd_cache_fork", "flashd_cache_reserve", "flashd_cache_append",
           "flashd_attn_fwd_tree", "flashd_tree_workspace_bytes", "flashd_cache_commit")


class Cache(ctypes.Structure):
    """struct flashd_cache of include/flashd.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("page_stride", ctypes.c_longlong),
                ("layer_stride", ctypes.c_longlong), ("layers", ctypes.c_int), ("P", ctypes.c_int),
                ("page", ctypes.c_int), ("max_pages", ctypes.c_int), ("B", ctypes.c_int),
                ("Hkv", ctypes.c_int), ("d", ctypes.c_int), ("dtype", ctypes.c_int),
                ("kscale", ctypes.c_float), ("vscale", ctypes.c_float)]


class FlashdError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"libflashd status {status}: {status_string(status)}")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2505_14201_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i, f, p, z = ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    base = [p, p, p, p, i, i, i, i, i, i, i, f, i, p]
    lib.flashd_attn_fwd.restype = i
    lib.flashd_attn_fwd.argtypes = base
    lib.flashd_attn_fwd_static.restype = i
    lib.flashd_attn_fwd_static.argtypes = base
    lib.flashd_attn_fwd_ex.restype = i
    lib.flashd_attn_fwd_skipv.restype = i
    lib.flashd_attn_fwd_skipv.argtypes = base + [i, p, z, p]
    lib.flashd_attn_fwd_ex.argtypes = base + [i, i, p, z]
    lib.flashd_workspace_bytes.restype = z
    lib.flashd_workspace_bytes.argtypes = [i] * 9
    lib.flashd_auto_splits.restype = i
    lib.flashd_auto_splits.argtypes = [i] * 8
    lib.flashd_auto_variant.restype = i
    lib.flashd_auto_variant.argtypes = [i] * 8
    lib.flashd_attn_fwd_state.restype = i
    lib.flashd_attn_fwd_state.argtypes = [p, p, p, p, p, p, i, i, i, i, i, i, i, i, f, i, p]
    lib.flashd_attn_fwd_kv8.restype = i
    lib.flashd_attn_fwd_kv8.argtypes = [p, p, p, p, i, i, i, i, i, i, i, f, f, f, i, p]
    lib.flashd_skip_stats.restype = i
    lib.flashd_skip_stats.argtypes = [p, p, i, i, i, i, i, i, i, f, i, f, f, p, p]
    n, c = ctypes.c_longlong, ctypes.POINTER(Cache)
    for name, args in (("fork", [c, p, p, i, p, p, p]), ("reserve", [c, p, p, p, p]),
                       ("append", [c, i, p, n, p, n, p, n, p, n, i, i, p, p, p, i, i, p, p, f, i, p]),
                       ("commit", [c, p, p, i, p, p, p])):
        fn = getattr(lib, "flashd_cache_" + name)
        fn.restype, fn.argtypes = i, args
    lib.flashd_attn_fwd_tree.restype = i
    lib.flashd_attn_fwd_tree.argtypes = [c, i, p, n, p, n, i, i, i, p, p, i, f, i, p, p, z]
    lib.flashd_tree_workspace_bytes.restype = z
    lib.flashd_tree_workspace_bytes.argtypes = [i] * 5
    lib.flashd_release_workspace.restype = i
    lib.flashd_release_workspace.argtypes = []
    lib.flashd_status_string.restype = ctypes.c_char_p
    lib.flashd_status_string.argtypes = [i]
    lib.flashd_version.restype = i
    lib.flashd_version.argtypes = []
    return lib


_lib = _load()
try:
    from . import _flashd_binding as _native
    _built, _here = _native.built_for, "torch {} and Python {}.{}".format(torch.__version__, *sys.version_info[:2])
    if _built != _here:
        raise ImportError(f"built for {_built}, this is {_here}")
except ImportError as e:
    # Missing, or built for another Python or torch than this one.  The C library is tied to neither,
    # and every call has its ctypes form.
    warnings.warn(f"the native part of the binding does not load ({e}): calls go through ctypes and cost some "
                  "3 us of host time more; build it with `python -m paper_2505_14201_amd.build`", RuntimeWarning)

    class _native:
        """Stands in for the native part: leaves every call to the Python form."""
        bind = attn_fwd = attn_fwd_kv8 = attn_fwd_state = staticmethod(lambda *args: None)
        bind_paged = cache_fork = cache_reserve = cache_append = attn_fwd_tree = cache_commit = bind


def raw() -> ctypes.CDLL:
    """The loaded C library (for tests that call the ABI with hand-made arguments)."""
    return _lib


def status_string(status: int) -> str:
    return _lib.flashd_status_string(int(status)).decode()


def version() -> int:
    return int(_lib.flashd_version())


def release_workspace() -> None:
    """flashd_release_workspace: free the scratch memory cached for the current device."""
    rc = int(_lib.flashd_release_workspace())
    if rc != 0:
        raise FlashdError(rc)


def workspace_bytes(B, Hq, Hkv, Lq, Lk, d, dtype, variant=VARIANT_AUTO, splits=0) -> int:
    return int(_lib.flashd_workspace_bytes(B, Hq, Hkv, Lq, Lk, d, dtype, variant, splits))


def auto_splits(B, Hq, Hkv, Lq, Lk, d, dtype, variant=VARIANT_AUTO) -> int:
    return int(_lib.flashd_auto_splits(B, Hq, Hkv, Lq, Lk, d, dtype, variant))


def auto_variant(B, Hq, Hkv, Lq, Lk, d, dtype, causal) -> int:
    return int(_lib.flashd_auto_variant(B, Hq, Hkv, Lq, Lk, d, dtype, int(bool(causal))))


def _marshal(q, k, v, o):
    # (written out: this runs on every call, and a loop over the tensors doubles its time)
    if not (q.is_cuda and k.is_cuda and v.is_cuda and o.is_cuda and q.is_contiguous() and
            k.is_contiguous() and v.is_contiguous() and o.is_contiguous()):
        for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
            if not t.is_cuda:
                raise ValueError(f"{name} must live on the GPU")
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
    dtype, qs, ks = q.dtype, q.shape, k.shape
    if dtype not in _DTYPE or not (k.dtype == v.dtype == o.dtype == dtype):
        raise ValueError("q, k, v, o must share one of float32/float16/bfloat16")
    if len(qs) != 4 or len(ks) != 4 or v.shape != ks or o.shape != qs:
        raise ValueError("expected q,o: [B,Hq,Lq,d] and k,v: [B,Hkv,Lk,d]")
    B, Hq, Lq, d = qs
    Bk, Hkv, Lk, dk = ks
    if Bk != B or dk != d:
        raise ValueError("batch or head dimension mismatch between q and k")
    return B, Hq, Hkv, Lq, Lk, d, _DTYPE[dtype]


# The current device and the raw handle of its current stream.  torch.cuda.current_stream() builds
# a Stream object around the handle and torch.cuda.device() saves and restores the device: 4.5 us
# together, of a call that takes 5.
_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream

# The native forms of attn_fwd, attn_fwd_kv8 and attn_fwd_state: they return the status of the call, or
# None where an argument is out of the ordinary and nothing has been enqueued.
_native.bind(*(ctypes.cast(f, ctypes.c_void_p).value
               for f in (_lib.flashd_attn_fwd, _lib.flashd_attn_fwd_kv8, _lib.flashd_attn_fwd_state)),
             _current_device, _raw_stream)


def _enqueue(fn, device, stream, head, tail=()) -> None:
    """fn(*head, stream handle, *tail) with `device` (an index) current; raises on a status other
    than 0."""
    if device != _current_device():
        with torch.cuda.device(device):
            return _enqueue(fn, device, stream, head, tail)
    rc = fn(*head, _raw_stream(device) if stream is None else stream.cuda_stream, *tail)
    if rc != 0:
        raise FlashdError(rc)


def attn_fwd(q, k, v, o, causal: bool, scale: float, stream=None) -> None:
    """flashd_attn_fwd: o <- attention(q, k, v), enqueued on `stream` (default: current)."""
    if stream is None:
        rc = _native.attn_fwd(q, k, v, o, causal, scale)
        if rc is not None:
            if rc != 0:
                raise FlashdError(rc)
            return
    B, Hq, Hkv, Lq, Lk, d, dt = _marshal(q, k, v, o)
    _enqueue(_lib.flashd_attn_fwd, q.get_device(), stream, (q.data_ptr(), k.data_ptr(),
             v.data_ptr(), o.data_ptr(), B, Hq, Hkv, Lq, Lk, d, int(bool(causal)), float(scale),
             dt))


def attn_fwd_static(q, k, v, o, causal: bool, scale: float, stream=None) -> None:
    """flashd_attn_fwd_static: as attn_fwd, split-K scratch in the library's fixed array
    (no allocation; raises FlashdError(E_WORKSPACE) when the problem needs more)."""
    B, Hq, Hkv, Lq, Lk, d, dt = _marshal(q, k, v, o)
    _enqueue(_lib.flashd_attn_fwd_static, q.get_device(), stream, (q.data_ptr(), k.data_ptr(),
             v.data_ptr(), o.data_ptr(), B, Hq, Hkv, Lq, Lk, d, int(bool(causal)), float(scale),
             dt))


def attn_fwd_ex(q, k, v, o, causal: bool, scale: float, variant: int = VARIANT_AUTO,
                splits: int = 0, workspace=None, stream=None) -> None:
    """flashd_attn_fwd_ex: explicit variant/splits and a caller-owned workspace tensor
    (any dtype, contiguous, on the same device) of at least workspace_bytes(...) bytes."""
    B, Hq, Hkv, Lq, Lk, d, dt = _marshal(q, k, v, o)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _enqueue(_lib.flashd_attn_fwd_ex, q.get_device(), stream, (q.data_ptr(), k.data_ptr(),
             v.data_ptr(), o.data_ptr(), B, Hq, Hkv, Lq, Lk, d, int(bool(causal)), float(scale),
             dt), (int(variant), int(splits), ws_ptr, ws_bytes))


def attn_fwd_skipv(q, k, v, o, causal: bool, scale: float, splits: int = 0, workspace=None,
                   counts=None, stream=None) -> None:
    """flashd_attn_fwd_skipv: decode with the saturation skip on the V fetch.  `counts`:
    optional GPU int64 tensor of 2 elements that the launch adds (blocks visited, blocks whose
    V was not fetched) to."""
    B, Hq, Hkv, Lq, Lk, d, dt = _marshal(q, k, v, o)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if counts is not None and not (counts.is_cuda and counts.dtype == torch.int64
                                   and counts.numel() >= 2 and counts.is_contiguous()):
        raise ValueError("counts must be a contiguous GPU int64 tensor of 2 elements")
    _enqueue(_lib.flashd_attn_fwd_skipv, q.get_device(), stream, (q.data_ptr(), k.data_ptr(),
             v.data_ptr(), o.data_ptr(), B, Hq, Hkv, Lq, Lk, d, int(bool(causal)), float(scale),
             dt), (int(splits), ws_ptr, ws_bytes, None if counts is None else counts.data_ptr()))


def skip_stats(q, k, causal: bool, scale: float, lo: float = -6.0, hi: float = 11.0,
               counts=None, stream=None):
    """flashd_skip_stats: (steps, low, high) of the static skip rule.  `counts`: optional
    GPU int64 tensor of 3 elements to receive the result (then nothing is read back and the
    call only enqueues work); otherwise a tensor is created and the counts are returned."""
    if not (q.is_cuda and k.is_cuda and q.is_contiguous() and k.is_contiguous()):
        raise ValueError("q and k must be contiguous GPU tensors")
    if q.dtype not in _DTYPE or k.dtype != q.dtype or q.dim() != 4 or k.dim() != 4:
        raise ValueError("expected q: [B,Hq,Lq,d] and k: [B,Hkv,Lk,d] of one storage type")
    B, Hq, Lq, d = q.shape
    Bk, Hkv, Lk, dk = k.shape
    if Bk != B or dk != d:
        raise ValueError("batch or head dimension mismatch between q and k")
    own = counts is None
    if own:
        counts = torch.empty(3, dtype=torch.int64, device=q.device)
    elif not (counts.is_cuda and counts.dtype == torch.int64 and counts.numel() >= 3
              and counts.is_contiguous()):
        raise ValueError("counts must be a contiguous GPU int64 tensor of 3 elements")
    _enqueue(_lib.flashd_skip_stats, q.get_device(), stream, (q.data_ptr(), k.data_ptr(), B, Hq,
             Hkv, Lq, Lk, d, int(bool(causal)), float(scale), _DTYPE[q.dtype], float(lo),
             float(hi), counts.data_ptr()))
    if not own:
        return None
    c = counts.cpu()
    return int(c[0]), int(c[1]), int(c[2])


def attn_fwd_state(q, k, v, causal: bool, scale: float, o=None, state_in=None, state_out=None,
                   causal_shift=None, stream=None) -> None:
    """flashd_attn_fwd_state: one chunk of keys with the Alg. 3 state handed in and out.
    States are float32 GPU tensors [B, Hq, Lq, d + 2]; causal_shift defaults to Lk - Lq."""
    if stream is None:
        rc = _native.attn_fwd_state(q, k, v, causal, scale, o, state_in, state_out, causal_shift)
        if rc is not None:
            if rc != 0:
                raise FlashdError(rc)
            return
    for name, t in (("q", q), ("k", k), ("v", v)):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous GPU tensor")
    if q.dtype not in _DTYPE or not (k.dtype == v.dtype == q.dtype):
        raise ValueError("q, k, v must share one of float32/float16/bfloat16")
    B, Hq, Lq, d = q.shape
    Bk, Hkv, Lk, dk = k.shape
    if Bk != B or dk != d or v.shape != k.shape:
        raise ValueError("shape mismatch between q, k and v")
    if o is not None and (o.shape != q.shape or o.dtype != q.dtype or not o.is_cuda
                          or not o.is_contiguous()):
        raise ValueError("o must match q")
    for name, t in (("state_in", state_in), ("state_out", state_out)):
        if t is not None and (tuple(t.shape) != (B, Hq, Lq, d + 2) or t.dtype != torch.float32
                              or not t.is_cuda or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous float32 GPU tensor [B, Hq, Lq, d + 2]")
    shift = Lk - Lq if causal_shift is None else int(causal_shift)
    ptr = lambda t: None if t is None else t.data_ptr()
    _enqueue(_lib.flashd_attn_fwd_state, q.get_device(), stream, (q.data_ptr(), k.data_ptr(),
             v.data_ptr(), ptr(o), ptr(state_in), ptr(state_out), B, Hq, Hkv, Lq, Lk, d,
             int(bool(causal)), shift, float(scale), _DTYPE[q.dtype]))


def attn_fwd_kv8(q, k8, v8, o, causal: bool, scale: float, kscale: float, vscale: float,
                 stream=None) -> None:
    """flashd_attn_fwd_kv8: K and V as torch.float8_e4m3fn tensors [B, Hkv, Lk, d] (the real
    values are kscale * k8 and vscale * v8); q and o float16 or bfloat16."""
    if stream is None:
        rc = _native.attn_fwd_kv8(q, k8, v8, o, causal, scale, kscale, vscale)
        if rc is not None:
            if rc != 0:
                raise FlashdError(rc)
            return
    for name, t in (("q", q), ("k8", k8), ("v8", v8), ("o", o)):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous GPU tensor")
    if q.dtype not in (torch.float16, torch.bfloat16) or o.dtype != q.dtype or o.shape != q.shape:
        raise ValueError("q and o must be float16 or bfloat16 tensors of one shape")
    if k8.dtype != torch.float8_e4m3fn or v8.dtype != k8.dtype or v8.shape != k8.shape:
        raise ValueError("k8 and v8 must be float8_e4m3fn tensors of one shape")
    B, Hq, Lq, d = q.shape
    Bk, Hkv, Lk, dk = k8.shape
    if Bk != B or dk != d:
        raise ValueError("batch or head dimension mismatch between q and k8")
    _enqueue(_lib.flashd_attn_fwd_kv8, q.get_device(), stream, (q.data_ptr(), k8.data_ptr(),
             v8.data_ptr(), o.data_ptr(), B, Hq, Hkv, Lq, Lk, d, int(bool(causal)), float(scale),
             float(kscale), float(vscale), _DTYPE[q.dtype]))


# ---- keys and values in pages ----------------------------------------------------------------------
#
# kcache and vcache are [P, Hkv, page, d] (or [layers, P, Hkv, page, d] for the calls that work on all
# layers), pages and layers at any stride; table is int32 [B, max_pages], lens int32 [B], q_start int32
# [B + 1], refs int32 [P].  What they mean is described in include/flashd.h.

def _ints(name, t, shape, device):
    if t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != device or t.dim() != len(shape) or \
            any(want is not None and have != want for have, want in zip(t.shape, shape)):
        want = ", ".join("any" if x is None else str(x) for x in shape)
        raise ValueError(f"{name} must be a contiguous int32 tensor [{want}] on the cache's GPU")


def _fit(*sizes):
    """FLASHD_E_SHAPE for sizes that the C call's ints do not hold (they would be cut off)."""
    if max(sizes) > 0x7fffffff or min(sizes) < -0x80000000:
        raise FlashdError(-2)


def _cache(kcache, vcache, table, lens, kscale=1.0, vscale=1.0, layers=False):
    """The struct for tensors of a cache; `layers`: five dimensions are allowed."""
    if not kcache.is_cuda or not vcache.is_cuda:
        raise ValueError("kcache and vcache must live on the GPU")
    shape, stride, dtype = kcache.shape, kcache.stride(), kcache.dtype
    if vcache.shape != shape or vcache.stride() != stride or vcache.dtype != dtype or dtype not in _CACHE_DTYPE \
            or vcache.get_device() != kcache.get_device():
        raise ValueError("kcache and vcache must have one shape, stride, device and type "
                         "(float32, float16, bfloat16 or float8_e4m3fn)")
    if len(shape) != 4 and not (layers and len(shape) == 5):
        raise ValueError("expected kcache, vcache: " + ("[(layers,) P, Hkv, page, d]" if layers else "[P, Hkv, page, d]"))
    P, Hkv, page, d = shape[-4:]
    if stride[-3:] != (page * d, d, 1):
        raise ValueError("a page of kcache and vcache must be contiguous")
    device = kcache.get_device()
    _ints("table", table, (None, None), device)
    B, max_pages = table.shape
    _ints("lens", lens, (B,), device)
    if min(P, Hkv, page, d, B, max_pages, shape[0]) < 1:
        raise ValueError("the cache has a dimension of size 0")
    _fit(P, Hkv, page, d, B, max_pages, shape[0])
    return Cache(kcache.data_ptr(), vcache.data_ptr(), table.data_ptr(), lens.data_ptr(),
                 stride[-4] if P > 1 else Hkv * page * d, stride[0] if len(shape) == 5 else 0,
                 shape[0] if len(shape) == 5 else 1, P, page, max_pages, B, Hkv, d, _CACHE_DTYPE[dtype],
                 kscale, vscale)


def _packed(name, t, T, heads, d, dtype, device):
    """The stride of a token of a packed tensor [T, heads, d], whose rows must be contiguous."""
    if t.get_device() != device or t.dtype != dtype or t.dim() != 3 or tuple(t.shape) != (T, heads, d):
        raise ValueError(f"{name} must be [{T}, {heads}, {d}] of type {dtype} on the cache's GPU")
    _fit(T, heads)
    s = t.stride()
    if s[2] != 1 or (heads > 1 and s[1] != d):
        raise ValueError(f"the heads of a token of {name} must be contiguous")
    return s[0] if T > 1 else heads * d


def _ptr(t):
    return None if t is None else t.data_ptr()


# The native forms of the five functions below, as of the three above.
_native.bind_paged(*(ctypes.cast(f, ctypes.c_void_p).value
                     for f in (_lib.flashd_cache_fork, _lib.flashd_cache_reserve, _lib.flashd_cache_append,
                               _lib.flashd_attn_fwd_tree, _lib.flashd_cache_commit)))


def _taken(rc) -> bool:
    """Whether a native form has made the call; raises on a status other than 0."""
    if rc is None:
        return False
    if rc != 0:
        raise FlashdError(rc)
    return True


def cache_fork(parent, refs, table, lens, table_out, lens_out, stream=None) -> None:
    """flashd_cache_fork: sequence i of table_out [B_out, max_pages] and lens_out goes on where
    sequence parent[i] of table and lens ended (empty if that is none); refs follows."""
    if stream is None and _taken(_native.cache_fork(parent, refs, table, lens, table_out, lens_out)):
        return
    if not table.is_cuda:
        raise ValueError("table must live on the GPU")
    device = table.get_device()
    _ints("table", table, (None, None), device)
    B, max_pages = table.shape
    _ints("lens", lens, (B,), device)
    _ints("parent", parent, (None,), device)
    n = parent.shape[0]
    _ints("table_out", table_out, (n, max_pages), device)
    _ints("lens_out", lens_out, (n,), device)
    _ints("refs", refs, (None,), device)
    _fit(n, max_pages, B, refs.shape[0])
    # (the pools themselves are not touched: any valid address and page size stand for them)
    c = Cache(16, 16, table.data_ptr(), lens.data_ptr(), 16 * 64, 0, 1, refs.shape[0], 16, max_pages, B, 1, 64, F16, 1.0, 1.0)
    _enqueue(_lib.flashd_cache_fork, device, stream, (c, refs.data_ptr(), parent.data_ptr(), n,
             table_out.data_ptr(), lens_out.data_ptr()))


def cache_reserve(kcache, vcache, refs, table, lens, q_start, report, stream=None) -> None:
    """flashd_cache_reserve: every sequence gets exactly the pages of its keys and new tokens; those it is to write to are its own.
    `report`: int32 [1 + B], receives the number of pages missing (0: all went well) and for each
    sequence the page that its shared last page was copied from, or -1.  Where pages are missing, shared last
    pages are held back (entries of -2 - page) until the next call: the step's results and new lengths are void then."""
    if stream is None and _taken(_native.cache_reserve(kcache, vcache, refs, table, lens, q_start, report)):
        return
    c = _cache(kcache, vcache, table, lens, layers=True)
    device = kcache.get_device()
    _ints("refs", refs, (c.P,), device)
    _ints("q_start", q_start, (c.B + 1,), device)
    _ints("report", report, (c.B + 1,), device)
    _enqueue(_lib.flashd_cache_reserve, device, stream, (c, refs.data_ptr(), q_start.data_ptr(),
             report.data_ptr()))


def cache_append(q, k, v, q_out, kcache, vcache, table, lens, q_start, positions=None, inv_freq=None,
                 q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                 kscale: float = 1.0, vscale: float = 1.0, stream=None) -> None:
    """flashd_cache_append: q_out [T, Hq, d] <- norm and rotation of q; k (the same) and v [T, Hkv, d] into
    the pages of one layer's cache.  q, k and v may be slices of one projection's output.  Without
    weights nothing is normed, without inv_freq (float32 [rot / 2]) nothing is rotated; positions
    (int32 [T]) default to the tokens' key numbers."""
    if stream is None and _taken(_native.cache_append(q, k, v, q_out, kcache, vcache, table, lens, q_start, positions, inv_freq, q_weight, k_weight,
                                                      eps, interleaved, kscale, vscale)):
        return
    c = _cache(kcache, vcache, table, lens, kscale, vscale)
    device = kcache.get_device()
    if q.dim() != 3 or q.dtype not in _DTYPE:
        raise ValueError("expected q: [T, Hq, d] of type float32, float16 or bfloat16")
    T, Hq, d = q.shape
    if d != c.d:
        raise ValueError("head dimension mismatch between q and kcache")
    dtype = q.dtype
    qs = _packed("q", q, T, Hq, d, dtype, device)
    ks = _packed("k", k, T, c.Hkv, d, dtype, device)
    vs = _packed("v", v, T, c.Hkv, d, dtype, device)
    os_ = _packed("q_out", q_out, T, Hq, d, dtype, device)
    _ints("q_start", q_start, (c.B + 1,), device)
    if positions is not None:
        _ints("positions", positions, (T,), device)
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (tuple(w.shape) != (d,) or w.dtype != dtype or w.get_device() != device or not w.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous tensor [d] of q's type")
    rot = 0
    if inv_freq is not None:
        if inv_freq.dim() != 1 or inv_freq.dtype != torch.float32 or inv_freq.get_device() != device \
                or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be a contiguous float32 tensor [rot / 2] on the cache's GPU")
        rot = 2 * inv_freq.shape[0]
        _fit(rot)
    if T == 0:
        return
    _enqueue(_lib.flashd_cache_append, device, stream, (c, 0, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
             q_out.data_ptr(), os_, T, Hq, q_start.data_ptr(), _ptr(positions), _ptr(inv_freq), rot,
             int(bool(interleaved)), _ptr(q_weight), _ptr(k_weight), float(eps), _DTYPE[dtype]))


def tree_workspace_bytes(Hq, Hkv, max_q, d, dtype) -> int:
    return int(_lib.flashd_tree_workspace_bytes(Hq, Hkv, max_q, d, dtype))


def attn_fwd_tree(q, kcache, vcache, o, table, lens, q_start, max_q: int, scale: float, tree=None,
                  kscale: float = 1.0, vscale: float = 1.0, workspace=None, stream=None) -> None:
    """flashd_attn_fwd_tree: o [T, Hq, d] <- attention of the new tokens' queries q over one layer's
    cache.  `tree`: int64 [T, words], the new tokens of its sequence that each token sees, one bit
    each; without it token i sees tokens 0 .. i.  max_q: the most new tokens of a sequence (a hint).
    `workspace`: a contiguous tensor of at least tree_workspace_bytes(...) bytes; without it scratch
    memory is kept per stream."""
    if stream is None and _taken(_native.attn_fwd_tree(q, kcache, vcache, o, table, lens, q_start, max_q, scale, tree, kscale, vscale,
                                                       workspace)):
        return
    c = _cache(kcache, vcache, table, lens, kscale, vscale)
    device = kcache.get_device()
    if q.dim() != 3 or q.dtype not in _DTYPE:
        raise ValueError("expected q: [T, Hq, d] of type float32, float16 or bfloat16")
    T, Hq, d = q.shape
    if d != c.d:
        raise ValueError("head dimension mismatch between q and kcache")
    qs = _packed("q", q, T, Hq, d, q.dtype, device)
    os_ = _packed("o", o, T, Hq, d, q.dtype, device)
    _ints("q_start", q_start, (c.B + 1,), device)
    words = 0
    if tree is not None:
        if tree.dtype != torch.int64 or tree.dim() != 2 or tree.shape[0] != T or not tree.is_contiguous() \
                or tree.get_device() != device:
            raise ValueError("tree must be a contiguous int64 tensor [T, words] on the cache's GPU")
        words = tree.shape[1]
    _fit(words, max_q)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if workspace.get_device() != device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the cache's GPU")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if T == 0:
        return
    _enqueue(_lib.flashd_attn_fwd_tree, device, stream, (c, 0, q.data_ptr(), qs, o.data_ptr(), os_, T, int(max_q), Hq,
             q_start.data_ptr(), _ptr(tree), words, float(scale), _DTYPE[q.dtype]), (ws_ptr, ws_bytes))


def cache_commit(kcache, vcache, table, lens, q_start, lens_out, keep=None, n_keep=None, stream=None) -> None:
    """flashd_cache_commit: the tokens that keep (int32 [B, max_keep], ascending) names move together
    behind their sequence's keys, in every layer; lens_out [B] <- lens + n_keep.  Without `keep` the
    first n_keep new tokens stay, without n_keep all.  Comes before a cache_fork of the same tokens, not after it."""
    if stream is None and _taken(_native.cache_commit(kcache, vcache, table, lens, q_start, lens_out, keep, n_keep)):
        return
    c = _cache(kcache, vcache, table, lens, layers=True)
    device = kcache.get_device()
    _ints("q_start", q_start, (c.B + 1,), device)
    _ints("lens_out", lens_out, (c.B,), device)
    if keep is not None:
        _ints("keep", keep, (c.B, None), device)
        _fit(keep.shape[1])
    if n_keep is not None:
        _ints("n_keep", n_keep, (c.B,), device)
    _enqueue(_lib.flashd_cache_commit, device, stream, (c, q_start.data_ptr(), _ptr(keep),
             0 if keep is None else keep.shape[1], _ptr(n_keep), lens_out.data_ptr()))
