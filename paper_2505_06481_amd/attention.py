"""Python binding of the attention half of libmmoe (see include/mmoe.h): projections with the variants' low-rank
adapters, rotary positions, the paged cache, attention of drafted tokens over it.

As in :mod:`mmoe`: argument marshalling only, on the current device's current stream, no fallback.  Tensors that are
part of a wider row (queries, keys and values in the output of one projection) may be passed as views.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import mmoe
from .mmoe import MmoeError, _ptr, _stream, lib

HALVES, NEIGHBOURS = 0, 1
PLAIN, INT8, FP8 = 0, 1, 2
PAGE_TOKENS = 64
_LAYOUTS = {"halves": HALVES, "neighbours": NEIGHBOURS}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}
_FORMATS = {"plain": PLAIN, "int8": INT8, "fp8": FP8}
_I32, _F32 = torch.int32, torch.float32


def _check(rc, where):
    if rc:
        raise MmoeError(rc, where)


def _code(value, names):
    return names[value] if isinstance(value, str) else int(value)


def _fields(names, c_type):
    return [(n, c_type) for n in names]


class ProjectShape(ctypes.Structure):
    _fields_ = _fields(("T", "d_in", "d_out", "n_adapters", "rank", "dtype"), ctypes.c_int32) + _fields(("ldx", "ldy"), ctypes.c_int64)


class RotaryShape(ctypes.Structure):
    _fields_ = (_fields(("T", "heads", "head_dim", "rot", "layout", "dtype", "transpose"), ctypes.c_int32)
                + [("magnitude", ctypes.c_float)] + _fields(("x_token", "x_head", "y_token", "y_head"), ctypes.c_int64))


class CacheShape(ctypes.Structure):
    _fields_ = _fields(("n_pages", "kv_heads", "head_dim", "dtype", "format"), ctypes.c_int32)


class _CachePointers(ctypes.Structure):
    _fields_ = _fields(("k", "v", "k_scale", "v_scale"), ctypes.c_void_p)


class _CacheRows(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32)] + _fields(("k_token", "k_head", "v_token", "v_head"), ctypes.c_int64)


class AttendShape(ctypes.Structure):
    _fields_ = ([("cache", CacheShape)]
                + _fields(("T", "n_requests", "heads", "max_pages", "max_drafts", "mask_words", "max_keys"), ctypes.c_int32)
                + [("sum_keys", ctypes.c_int64), ("scale", ctypes.c_float)]
                + _fields(("q_token", "q_head", "o_token", "o_head"), ctypes.c_int64))


class Cache:
    """Pages of keys and values (bytes in the layout of include/mmoe.h) and their scales (None for plain pages), on the GPU.
    Iterates over (k, v, k_scale, v_scale).  The tensors are looked at once: they stay what and where they are."""
    __slots__ = ("_tensors", "_pointers", "_bytes")

    def __init__(self, k, v, k_scale=None, v_scale=None):
        self._tensors = (k, v, k_scale, v_scale)
        if (k_scale is None) != (v_scale is None):
            raise ValueError("k_scale and v_scale go together")
        self._pointers = _CachePointers(_ptr(k, torch.uint8, None, "k"), _ptr(v, torch.uint8, None, "v"), _ptr(k_scale, _F32, None, "k_scale"),
                                        _ptr(v_scale, _F32, None, "v_scale"))
        self._bytes = (min(k.numel(), v.numel()), 0 if k_scale is None else 4 * min(k_scale.numel(), v_scale.numel()))

    k, v, k_scale, v_scale = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    def __iter__(self):
        return iter(self._tensors)

    def address(self, shape):
        """Address of the pointers, for a shape whose pages they have room for."""
        rows = shape.n_pages * shape.kv_heads * PAGE_TOKENS
        kept = rows * shape.head_dim * (1 if shape.format else 4 if shape.dtype == mmoe.F32 else 2)
        if self._bytes[0] < kept or (shape.format and self._bytes[1] < 4 * rows):
            raise ValueError(f"the cache holds {self._bytes} bytes, the shape needs {kept} and {4 * rows if shape.format else 0}")
        return ctypes.addressof(self._pointers)


@functools.lru_cache(maxsize=None)
def _entry(name):
    L = lib()
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    f = getattr(L, name)
    f.argtypes, f.restype = {
        "mmoe_project_workspace_bytes": ([vp], sz),
        "mmoe_project_packed_rank": ([vp], sz),
        "mmoe_pack_projection": ([vp] * 4, ctypes.c_int),
        "mmoe_pack_adapters": ([vp] * 6, ctypes.c_int),
        "mmoe_project": ([vp] * 9 + [sz, vp], ctypes.c_int),
        "mmoe_rotary_steps": ([i32, ctypes.c_double, i32, ctypes.c_double, i32, vp, vp], ctypes.c_int),
        "mmoe_rotary": ([vp] * 6, ctypes.c_int),
        "mmoe_cache_bytes": ([vp] * 2, sz),
        "mmoe_cache_append": ([vp] * 10, ctypes.c_int),
        "mmoe_cache_read": ([vp, vp, i32, vp, vp, vp, vp], ctypes.c_int),
        "mmoe_attend_workspace_bytes": ([vp], sz),
        "mmoe_attend": ([vp] * 10 + [sz, vp], ctypes.c_int),
    }[name]
    return f


def _dtype(dtype):
    return _code(dtype, mmoe._DTYPES)


def _heads_view(t, dtype, T, heads, head_dim, name):
    """Pointer and (token, head) strides of a [T, heads, head_dim] tensor or view whose heads are contiguous."""
    if t.is_cuda and t.dtype is dtype and t.shape == (T, heads, head_dim):
        a, b, c = t.stride()
        if c == 1 and b >= head_dim and a >= b * heads:
            return t.data_ptr(), a, b
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != (T, heads, head_dim):
        raise ValueError(f"{name}: expected shape {(T, heads, head_dim)}, got {tuple(t.shape)}")
    a, b, c = t.stride()
    if c != 1 and head_dim > 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    if T == 1 and a < b * heads:  # (a stride over one token steps over nothing)
        a = max(b, head_dim) * heads
    if heads == 1 and b < head_dim:
        b = head_dim
    if a <= 0 or b <= 0:
        raise ValueError(f"{name}: strides must be positive")
    return t.data_ptr(), a, b


# ---------------------------------------------------------------- projection with adapters
def make_project_shape(T, d_in, d_out, n_adapters, rank, dtype, ldx=0, ldy=0) -> ProjectShape:
    """``n_adapters`` 0: the plain projection.  ``ldx``, ``ldy``: elements from row to row of X and Y, 0 = dense."""
    return ProjectShape(T, d_in, d_out, n_adapters, rank, _dtype(dtype), ldx, ldy)


def project_workspace_bytes(shape: ProjectShape) -> int:
    return int(_entry("mmoe_project_workspace_bytes")(ctypes.addressof(shape)))


def project_workspace(shape: ProjectShape, device="cuda") -> torch.Tensor:
    return torch.empty(max(256, project_workspace_bytes(shape)), dtype=torch.uint8, device=device)


def pack_projection(shape: ProjectShape, W):
    """W [d_in, d_out] -> its packed form (a new tensor of as many elements)."""
    dt = mmoe._TORCH_DT[shape.dtype]
    Wp = torch.empty(shape.d_in * shape.d_out, dtype=dt, device=W.device)
    _check(_entry("mmoe_pack_projection")(ctypes.addressof(shape), _ptr(W, dt, Wp.numel(), "W"), Wp.data_ptr(), _stream()),
           "mmoe_pack_projection")
    return Wp


def pack_adapters(shape: ProjectShape, A, B):
    """A [n, d_in, rank], B [n, rank, d_out] -> their packed forms."""
    dt, n = mmoe._TORCH_DT[shape.dtype], shape.n_adapters
    rank = int(_entry("mmoe_project_packed_rank")(ctypes.addressof(shape)))
    Ap = torch.empty(n * rank * shape.d_in, dtype=dt, device=A.device)
    Bp = torch.empty(n * rank * shape.d_out, dtype=dt, device=A.device)
    _check(_entry("mmoe_pack_adapters")(ctypes.addressof(shape), _ptr(A, dt, n * shape.rank * shape.d_in, "A"),
                                        _ptr(B, dt, n * shape.rank * shape.d_out, "B"), Ap.data_ptr(), Bp.data_ptr(), _stream()),
           "mmoe_pack_adapters")
    return Ap, Bp


def _rows_ptr(t, dtype, rows, cols, ld, name):
    """Pointer of [rows, cols] with rows ``ld`` apart (0: dense)."""
    if t.is_cuda and t.dtype is dtype and t.shape == (rows, cols) and t.stride() == (ld or cols, 1):
        return t.data_ptr()
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: expected shape {(rows, cols)}, got {tuple(t.shape)}")
    if t.stride(1) != 1 or (rows > 1 and t.stride(0) != (ld or cols)):
        raise ValueError(f"{name}: expected rows of contiguous elements, {ld or cols} apart, got strides {t.stride()}")
    return t.data_ptr()


def project(shape: ProjectShape, X, aid, Wp, Ap, Bp, scale, ws, Y=None):
    """Y[t] = X[t] W + scale[a] (X[t] A[a]) B[a], a = aid[t] (none where aid[t] is not an adapter's number)."""
    dt, n = mmoe._TORCH_DT[shape.dtype], shape.n_adapters
    T, K, N = shape.T, shape.d_in, shape.d_out
    if Y is None:
        Y = X.new_empty((T, N)) if not shape.ldy else \
            torch.empty((T, shape.ldy), dtype=dt, device=X.device)[:, :N]
    rank = (shape.rank + 31) // 32 * 32 if dt == torch.bfloat16 else (shape.rank + 15) // 16 * 16
    rc = _entry("mmoe_project")(
        ctypes.addressof(shape), _rows_ptr(X, dt, T, K, shape.ldx, "X"), _ptr(aid, _I32, T, "aid") if n else None,
        _ptr(Wp, dt, K * N, "Wp"), _ptr(Ap, dt, n * rank * K, "Ap") if n else None, _ptr(Bp, dt, n * rank * N, "Bp") if n else None,
        _ptr(scale, _F32, n, "scale") if n else None, _rows_ptr(Y, dt, T, N, shape.ldy, "Y"), _ptr(ws, torch.uint8, None, "ws"),
        ws.numel(), _stream())
    _check(rc, "mmoe_project")
    return Y


# ---------------------------------------------------------------- rotary positions
def rotary_steps(rot, base=10000.0, scaling="none", factor=1.0, original=0, device="cuda"):
    """(turns per position of every pair in units of 2^-64, int64 on the device; magnitude)."""
    steps = torch.empty(rot // 2, dtype=torch.int64)
    magnitude = ctypes.c_float()
    _check(_entry("mmoe_rotary_steps")(int(rot), float(base), _code(scaling, _SCALINGS), float(factor), int(original),
                                       steps.data_ptr(), ctypes.addressof(magnitude)), "mmoe_rotary_steps")
    return steps.to(device), magnitude.value


def make_rotary_shape(T, heads, head_dim, rot, layout, dtype, magnitude=1.0, transpose=False) -> RotaryShape:
    return RotaryShape(T, heads, head_dim, rot, _code(layout, _LAYOUTS), _dtype(dtype), int(transpose), magnitude, 0, 0, 0, 0)


def rotary(shape: RotaryShape, X, pos, steps, Y=None):
    """X [T, heads, head_dim] (a view is fine) with its heads turned by pos [T]; Y = X works in place."""
    dt = mmoe._TORCH_DT[shape.dtype]
    T, H, D = shape.T, shape.heads, shape.head_dim
    if Y is None:
        Y = X.new_empty((T, H, D))
    x, xt, xh = _heads_view(X, dt, T, H, D, "X")
    y, yt, yh = _heads_view(Y, dt, T, H, D, "Y")
    call = RotaryShape(T, H, D, shape.rot, shape.layout, shape.dtype, shape.transpose, shape.magnitude, xt, xh, yt, yh)
    rc = _entry("mmoe_rotary")(ctypes.addressof(call), x, _ptr(pos, _I32, T, "pos"), _ptr(steps, torch.int64, shape.rot // 2, "steps"), y,
                               _stream())
    _check(rc, "mmoe_rotary")
    return Y


# ---------------------------------------------------------------- paged cache
def make_cache_shape(n_pages, kv_heads, head_dim, dtype, format="plain") -> CacheShape:
    return CacheShape(n_pages, kv_heads, head_dim, _dtype(dtype), _code(format, _FORMATS))


def cache_bytes(shape: CacheShape):
    """(bytes of the keys' pages, bytes of their scales); the values take as much again."""
    scales = ctypes.c_size_t()
    n = int(_entry("mmoe_cache_bytes")(ctypes.addressof(shape), ctypes.addressof(scales)))
    return n, scales.value


def alloc_cache(shape: CacheShape, device="cuda") -> Cache:
    n, scales = cache_bytes(shape)
    if n == 0:
        raise ValueError("mmoe_cache_bytes: the cache's shape is not valid")
    k, v = (torch.empty(n, dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.empty(scales // 4, dtype=_F32, device=device) if scales else None for _ in range(2))
    return Cache(k, v, ks, vs)


def cache_append(shape: CacheShape, K, V, places, cache: Cache, rotary=None):
    """Writes K, V [T, kv_heads, head_dim] (views are fine) to the places of their tokens.  ``rotary``: (RotaryShape, steps,
    pos) turns the keys first."""
    dt = mmoe._TORCH_DT[shape.dtype]
    T, H, D = places.numel(), shape.kv_heads, shape.head_dim
    if T == 0:
        return
    k, kt, kh = _heads_view(K, dt, T, H, D, "K")
    v, vt, vh = _heads_view(V, dt, T, H, D, "V")
    rows = _CacheRows(T, kt, kh, vt, vh)
    turn = steps = pos = None
    if rotary is not None:
        spec, steps, pos = rotary
        turn, steps, pos = ctypes.addressof(spec), _ptr(steps, torch.int64, spec.rot // 2, "steps"), _ptr(pos, _I32, T, "pos")
    rc = _entry("mmoe_cache_append")(ctypes.addressof(shape), ctypes.addressof(rows), k, v, _ptr(places, _I32, T, "places"), turn, pos, steps,
                                     cache.address(shape), _stream())
    _check(rc, "mmoe_cache_append")


def cache_read(shape: CacheShape, cache: Cache, places, K=None, V=None):
    """(K, V) [R, kv_heads, head_dim] of the places, in the cache's dtype."""
    dt = mmoe._TORCH_DT[shape.dtype]
    R, H, D = places.numel(), shape.kv_heads, shape.head_dim
    if K is None:
        K = torch.empty((R, H, D), dtype=dt, device=places.device)
    if V is None:
        V = torch.empty((R, H, D), dtype=dt, device=places.device)
    if R == 0:
        return K, V
    rc = _entry("mmoe_cache_read")(ctypes.addressof(shape), cache.address(shape), R, _ptr(places, _I32, R, "places"),
                                   _ptr(K, dt, R * H * D, "K"), _ptr(V, dt, R * H * D, "V"), _stream())
    _check(rc, "mmoe_cache_read")
    return K, V


# ---------------------------------------------------------------- attention of drafted tokens
def make_attend_shape(cache: CacheShape, T, n_requests, heads, max_pages, max_drafts, scale, mask_words=None, max_keys=0,
                      sum_keys=0) -> AttendShape:
    """``mask_words``: 64-bit words of a row of the tree mask (default: as many as max_drafts needs).  ``max_keys``,
    ``sum_keys``: the longest ctx + drafts and their sum, where the caller knows them (they set how the work is shared out)."""
    words = (max_drafts + 63) // 64 if mask_words is None else mask_words
    return AttendShape(cache, T, n_requests, heads, max_pages, max_drafts, words, max_keys, sum_keys, scale, 0, 0, 0, 0)


def attend_workspace_bytes(shape: AttendShape) -> int:
    return int(_entry("mmoe_attend_workspace_bytes")(ctypes.addressof(shape)))


def attend_workspace(shape: AttendShape, device="cuda") -> torch.Tensor:
    """For calls of this shape and of fewer requests, tokens, drafts or pages (with ``sum_keys`` set: of up to as many keys)."""
    n = attend_workspace_bytes(shape)
    if n == 0:
        raise ValueError("mmoe_attend_workspace_bytes: the shape is not valid")
    return torch.empty(n, dtype=torch.uint8, device=device)


def attend(shape: AttendShape, Q, starts, ctx, tree, pages, cache: Cache, ws, out=None, lse=None):
    """(out [T, heads, head_dim], lse [T, heads]) of the drafted tokens of every request over its pages.  ``tree``: int64
    [T, mask_words] bit masks, or None for causal chunks and single tokens."""
    c = shape.cache
    dt = mmoe._TORCH_DT[c.dtype]
    T, H, D, B = shape.T, shape.heads, c.head_dim, shape.n_requests
    if out is None:
        out = Q.new_empty((T, H, D))
    if lse is None:
        lse = torch.empty((T, H), dtype=_F32, device=Q.device)
    q, qt, qh = _heads_view(Q, dt, T, H, D, "Q")
    o, ot, oh = _heads_view(out, dt, T, H, D, "out")
    call = AttendShape.from_buffer_copy(shape)
    call.q_token, call.q_head, call.o_token, call.o_head = qt, qh, ot, oh
    rc = _entry("mmoe_attend")(ctypes.addressof(call), q, _ptr(starts, _I32, B + 1, "starts"), _ptr(ctx, _I32, B, "ctx"),
                               _ptr(tree, torch.int64, T * shape.mask_words, "tree"), _ptr(pages, _I32, B * shape.max_pages, "pages"),
                               cache.address(c), o, _ptr(lse, _F32, T * H, "lse"), _ptr(ws, torch.uint8, None, "ws"),
                               ws.numel(), _stream())
    _check(rc, "mmoe_attend")
    return out, lse
