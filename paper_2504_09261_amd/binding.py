"""Thin binding over the C ABI of include/hack.h: ctypes, and for hack_step, which an image calls layers x scales
times, and the operators around the cache, which a token calls for every layer, CPython entries (csrc/py_step.cpp, csrc/py_ops.cpp).

Argument marshalling only: every step of the path runs in the HIP kernels of
libhack_mi355x.so.  PyTorch is used for device memory and the current stream.
There is no CPU fallback: if the library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhack_mi355x.so")

HACK_BF16, HACK_F32 = 0, 1
CONTEXTUAL, STRUCTURAL = 0, 1

EXPORTS = [
    "hack_create", "hack_destroy", "hack_strerror", "hack_last_error", "hack_check",
    "hack_score", "hack_select", "hack_compact", "hack_attn", "hack_attn_variant",
    "hack_kvcache_rows_required", "hack_kvcache_create", "hack_kvcache_destroy",
    "hack_kvcache_reset", "hack_kvcache_view", "hack_kvcache_step_form", "hack_step", "hack_head_variance",
    "hack_set_score_mode", "hack_get_score_mode", "hack_score_static", "hack_score_item_keys", "hack_merge", "hack_step_final",
    "hack_rope_freqs", "hack_rotate", "hack_norm_rotate", "hack_packed_bytes", "hack_pack", "hack_unpack", "hack_attn_packed", "hack_append_pages",
    "hack_attn_pages",
]


class HackError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"hack status {status}: {msg}")
        self.status = status


class hack_config(C.Structure):
    _fields_ = [("device", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("max_units", C.c_int32), ("max_cache_len", C.c_int32), ("max_queries", C.c_int32),
                ("n_obs", C.c_int32)]


class hack_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("rows", C.c_int64),
                ("off", C.POINTER(C.c_int64)), ("len", C.POINTER(C.c_int32))]


class _raw_cache(C.Structure):
    """The same memory with the host arrays as plain addresses (making a pointer object takes longer than a call)."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("rows", C.c_int64),
                ("off", C.c_void_p), ("len", C.c_void_p)]


class hack_rope(C.Structure):
    _fields_ = [("layout", C.c_int32), ("rot_dim", C.c_int32), ("axes", C.c_int32), ("gain", C.c_float), ("freq", C.POINTER(C.c_double))]


class hack_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pages", C.c_int64), ("page_rows", C.c_int32), ("stride_page", C.c_int64), ("stride_row", C.c_int64),
                ("stride_head", C.c_int64), ("table", C.c_void_p), ("table_pages", C.c_int32), ("table_stride", C.c_int64), ("len", C.c_void_p),
                ("by_head", C.c_int32), ("max_len", C.c_int32)]


_lib = None
_step_call = _step_addr = None    # CPython entry; addresses of hack_step and hack_step_final
_ops_call = _ops_addr = None      # CPython entries; addresses of the functions they call


def load_library() -> C.CDLL:
    """dlopen the in-tree library; torch is imported first so that both use the
    same HIP runtime."""
    global _lib, _step_call, _step_addr, _ops_call, _ops_addr
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (loads libamdhip64 with the soname the library needs)
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2504_09261_amd.build` "
            "(there is no fallback path)")
    try:
        from paper_2504_09261_amd._step_call import step as _step_call
        from paper_2504_09261_amd import _ops_call
    except ImportError as e:
        raise FileNotFoundError(f"an entry beside {LIB_PATH} is missing: build it with "
                                "`python -m paper_2504_09261_amd.build` (there is no fallback path)") from e
    lib = C.CDLL(LIB_PATH)
    _step_addr = tuple(C.cast(f, C.c_void_p).value for f in (lib.hack_step, lib.hack_step_final))
    _ops_addr = {n: C.cast(getattr(lib, "hack_" + n), C.c_void_p).value for n in ("rotate", "norm_rotate", "pack", "unpack", "attn_packed", "append_pages", "attn_pages")}
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    pi32, pi64, pu8 = C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_uint8)
    pcache = C.POINTER(hack_cache)
    lib.hack_create.argtypes = [C.POINTER(vp), C.POINTER(hack_config)]
    lib.hack_destroy.argtypes = [vp]
    lib.hack_destroy.restype = None
    lib.hack_strerror.argtypes = [C.c_int]
    lib.hack_strerror.restype = C.c_char_p
    lib.hack_last_error.argtypes = [vp]
    lib.hack_last_error.restype = C.c_char_p
    lib.hack_check.argtypes = [vp]
    lib.hack_set_score_mode.argtypes = [vp, i32]
    lib.hack_get_score_mode.argtypes = [vp]
    lib.hack_get_score_mode.restype = i32
    lib.hack_score.argtypes = [vp, i32, i32, vp, pi32, i32, f32, pcache, vp, pu8, vp, i64, vp]
    lib.hack_score_static.argtypes = [vp, i32, i32, vp, pi32, i32, f32, pcache, vp, pu8, vp, i64, vp]
    lib.hack_score_item_keys.argtypes = [vp, i32, pi32]
    lib.hack_score_item_keys.restype = i32
    lib.hack_select.argtypes = [vp, i32, vp, i64, pi32, pu8, pi32, i32, i32, vp, i64, pi32, vp]
    lib.hack_compact.argtypes = [vp, i32, i32, pcache, vp, vp, i32, vp, i64, pcache, vp]
    lib.hack_merge.argtypes = [vp, i32, i32, pcache, vp, vp, vp, i64, pu8, pcache, vp]
    lib.hack_step_final.argtypes = [vp, vp, i32, i32, vp, vp, vp, pu8, pi32, i32, f32, vp, vp, i64, vp]
    lib.hack_attn.argtypes = [vp, i32, i32, vp, pcache, f32, vp, vp]
    lib.hack_attn_variant.argtypes = [vp, i32, i32]
    lib.hack_attn_variant.restype = i32
    lib.hack_head_variance.argtypes = [vp, i32, i32, vp, pcache, f32, vp, vp]
    lib.hack_kvcache_rows_required.argtypes = [i32, pi32, pi64]
    lib.hack_kvcache_create.argtypes = [vp, i32, pi32, vp, vp, vp, i64, C.POINTER(vp)]
    lib.hack_kvcache_destroy.argtypes = [vp]
    lib.hack_kvcache_destroy.restype = None
    lib.hack_kvcache_reset.argtypes = [vp]
    lib.hack_kvcache_view.argtypes = [vp, pcache]
    lib.hack_kvcache_step_form.argtypes = [vp]
    lib.hack_kvcache_step_form.restype = i32
    lib.hack_step.argtypes = [vp, vp, i32, i32, vp, vp, vp, pu8, pi32, i32, f32, vp, vp, i64, vp]
    lib.hack_rope_freqs.argtypes = [i32, i32, i32, C.c_double, C.c_double, C.c_double, C.POINTER(C.c_double), C.POINTER(f32)]
    lib.hack_packed_bytes.argtypes = [i32, i64, pi64]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is C.c_int and name not in ("hack_strerror", "hack_last_error"):
            fn.restype = C.c_int
    _lib = lib
    return lib


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _i64(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int64)


def _exact(a, dtype) -> np.ndarray:
    """A host array of an integer type; numbers that it does not hold are refused, not cut."""
    x = np.asarray(a)
    if x.dtype == dtype:
        return np.ascontiguousarray(x)
    with np.errstate(invalid="ignore"):
        y = x.astype(dtype)
    if not np.array_equal(x, y):
        raise OverflowError(f"not all of the numbers are {np.dtype(dtype).name}")
    return np.ascontiguousarray(y)


def _u8(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.uint8)


def _p(a: Optional[np.ndarray], ctype):
    """A host array as a typed pointer argument.  (ndarray.ctypes.data_as, for read-only or empty arrays, costs 3 us an
    array, as much as a kernel launch; the other way 0.4.)  The object keeps the array alive."""
    if a is None:
        return None
    try:
        return C.byref(ctype.from_buffer(a))
    except (TypeError, ValueError):
        return a.ctypes.data_as(C.POINTER(ctype))


def _addr(a: np.ndarray) -> int:
    """Address of a host array for a structure member (the caller keeps the array alive)."""
    try:
        return C.addressof(C.c_char.from_buffer(a))
    except (TypeError, ValueError):
        return a.__array_interface__["data"][0]


def _dev(t) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA/HIP tensors"
    return t.data_ptr()


_raw_stream = _device = None


def _stream() -> int:
    """hipStream_t of the current device's current stream."""
    global _raw_stream, _device
    if _raw_stream is None:
        import torch   # once: looking the module up in every call takes as long as the two typed pointers of a step
        _device = torch.cuda.current_device
        # the raw handle without building a torch.cuda.Stream object for every call
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda _: torch.cuda.current_stream().cuda_stream)
    return _raw_stream(_device())


class Cache:
    """A hack_cache view: device K/V(/pos) tensors plus host offsets and lengths."""

    def __init__(self, k, v, off, length, pos=None):
        self.k, self.v, self.pos = k, v, pos
        self.off, self.len = _i64(off), _i32(length)
        assert k.shape == v.shape and k.dim() == 2
        self.rows = int(k.shape[0])

    def struct(self) -> hack_cache:
        return hack_cache.from_buffer(_raw_cache(_dev(self.k), _dev(self.v), _dev(self.pos), self.rows,
                                                 _addr(self.off), _addr(self.len)))


PACK_ROWS = 64   # rows of a block of a packed cache


def packed_bytes(head_dim: int, rows: int) -> int:
    """Bytes of the K (and of the V) of `rows` rows of a packed cache."""
    n = C.c_int64()
    st = load_library().hack_packed_bytes(head_dim, rows, C.byref(n))
    if st != 0:
        raise HackError(st, load_library().hack_strerror(st).decode())
    return n.value


class PackedCache:
    """A hack_packed_cache view: device byte tensors of K and V (hack_packed_bytes each), host offsets (multiples of 64 rows) and lengths."""

    def __init__(self, k, v, off, length, pos=None):
        import torch
        self.k, self.v, self.pos = k, v, pos
        self.off, self.len = _exact(off, np.int64), _exact(length, np.int32)
        assert k.dtype == v.dtype == torch.uint8 and k.shape == v.shape and k.dim() == 2, "K and V: byte tensors [rows / 64, bytes of 64 rows]"
        assert k.shape[1] in (34 * 64, 34 * 128), "a block of 64 rows has 34 bytes an element of the head"
        assert pos is None or pos.dtype == torch.int32 and pos.numel() >= PACK_ROWS * k.shape[0], "pos: an int32 for every row"
        self.head_dim, self.rows = int(k.shape[1]) // 34, PACK_ROWS * int(k.shape[0])

    @classmethod
    def empty(cls, head_dim: int, cap, device="cuda", with_pos: bool = False) -> "PackedCache":
        """Room for units of up to cap[u] rows, all of them empty."""
        import torch
        blocks = -(-_exact(cap, np.int64) // PACK_ROWS)
        n = int(blocks.sum())
        k, v = (torch.empty((n, packed_bytes(head_dim, PACK_ROWS)), dtype=torch.uint8, device=device) for _ in range(2))
        pos = torch.empty((n * PACK_ROWS,), dtype=torch.int32, device=device) if with_pos else None
        return cls(k, v, PACK_ROWS * (np.cumsum(blocks) - blocks), np.zeros(len(blocks), np.int32), pos)


class PagedCache:
    """A hack_pages view.  k, v: [pages, rows of a page, heads, head_dim] in the same strides, any with head_dim side by side (so a pool that keeps a head's rows
    together is given transposed).  table: int32 [B, pages of a sequence], length: int32 [B], with the rows that a call brings; where pages hold one head and the context has
    more, both go by head, [B heads, ...]; max_len: the most that a length will be (default: what a row of the table holds), which launches are laid out for.  Its
    tensors are not replaced, since the library reads the structure that they were put into; what they hold may change at any time, in captured graphs too."""

    def __init__(self, k, v, table, length, max_len: int = 0):
        import torch
        assert k.is_cuda and all(t.device == k.device for t in (v, table, length)), "device tensors, on one device"
        assert k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.stride() == v.stride() and k.stride(3) == 1, \
            "K and V: [pages, rows, heads, head_dim] in the same strides"
        assert table.dtype == length.dtype == torch.int32 and table.dim() == 2 and length.shape == table.shape[:1], "table: int32 rows of pages; length: an int32 for each"
        assert length.is_contiguous() and (table.stride(1) == 1 or table.shape[1] <= 1), "lengths, and the entries of a table's row, side by side"
        assert 0 <= max_len < 1 << 31, "max_len: an int32"
        pages, rows, heads, head_dim = k.shape
        across = table.stride(0) if table.shape[0] > 1 else table.shape[1]
        struct = hack_pages(k.data_ptr(), v.data_ptr(), pages, rows, k.stride(0) if pages > 1 else 0, k.stride(1), k.stride(2) if heads > 1 else 0, table.data_ptr(),
                            table.shape[1], across, length.data_ptr(), 0, max_len)
        self.__dict__.update(k=k, v=v, table=table, len=length, max_len=max_len, _struct=struct,
                             _info=(C.addressof(struct), k.get_device(), k.dtype, head_dim, heads, int(table.shape[0])))

    def __setattr__(self, name, value):
        raise AttributeError(f"a PagedCache's {name} is not replaced: make another one")

    def __reduce__(self):   # a copy has a structure of its own
        return PagedCache, (self.k, self.v, self.table, self.len, self.max_len)


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}
NORMS = {"rms": 0, "l2": 1}


class Rope:
    """A hack_rope: frequencies (radians per position, axis after axis), which elements rotate and how they pair.  Its parts are not replaced, since the library
    reads the structure that they were put into; frequencies may be changed in place."""

    def __init__(self, freq, rot_dim: int, axes: int = 1, layout: str = "half", gain: float = 1.0):
        freq = np.ascontiguousarray(freq, np.float64)
        assert freq.shape == (rot_dim // 2,), "one frequency for every pair"
        struct = hack_rope(ROPE_LAYOUTS[layout], rot_dim, axes, gain, freq.ctypes.data_as(C.POINTER(C.c_double)))
        self.__dict__.update(freq=freq, rot_dim=rot_dim, axes=axes, layout=layout, gain=gain, _struct=struct, address=C.addressof(struct))

    def __setattr__(self, name, value):
        raise AttributeError(f"a Rope's {name} is not replaced: make another one")

    def __reduce__(self):   # a copy has a structure of its own, which points to its own frequencies
        return Rope, (self.freq.copy(), self.rot_dim, self.axes, self.layout, self.gain)

    @classmethod
    def scaled(cls, rot_dim: int, axes: int = 1, layout: str = "half", scaling: str = "plain", base: float = 10000.0, factor: float = 1.0,
               trained_len: float = 0.0) -> "Rope":
        """The frequencies and the gain of hack_rope_freqs."""
        lib = load_library()
        freq, gain = np.zeros(max(rot_dim // 2, 0)), C.c_float()
        st = lib.hack_rope_freqs(rot_dim, axes, ROPE_SCALINGS[scaling], base, factor, trained_len, freq.ctypes.data_as(C.POINTER(C.c_double)), C.byref(gain))
        if st != 0:
            raise HackError(st, lib.hack_strerror(st).decode())
        return cls(freq, rot_dim, axes, layout, gain.value)


class ManagedCache:
    """hack_kvcache: two slabs of cap[u] rows per unit inside caller-provided tensors."""

    def __init__(self, hack: "Hack", cap: Sequence[int], with_pos: bool = True):
        import torch
        self.hack = hack
        self.cap = _i32(cap)
        lib = hack.lib
        rows = C.c_int64()
        hack._check(lib.hack_kvcache_rows_required(len(self.cap), _p(self.cap, C.c_int32), C.byref(rows)))
        self.rows = rows.value
        dev = torch.device("cuda", hack.device)
        self.k = torch.empty((self.rows, hack.head_dim), dtype=hack.torch_dtype, device=dev)
        self.v = torch.empty((self.rows, hack.head_dim), dtype=hack.torch_dtype, device=dev)
        self.pos = torch.empty((self.rows,), dtype=torch.int32, device=dev) if with_pos else None
        h = C.c_void_p()
        hack._check(lib.hack_kvcache_create(hack.ctx, len(self.cap), _p(self.cap, C.c_int32), _dev(self.k),
                                            _dev(self.v), _dev(self.pos), self.rows, C.byref(h)))
        self.handle = h

    def reset(self):
        self.hack._check(self.hack.lib.hack_kvcache_reset(self.handle))

    def view(self):
        """(off int64[U], len int32[U]) copies of the current state."""
        s = _raw_cache()
        self.hack._check(self.hack.lib.hack_kvcache_view(self.handle, hack_cache.from_buffer(s)))
        n = len(self.cap)
        return (np.frombuffer((C.c_int64 * n).from_address(s.off), np.int64).copy(),
                np.frombuffer((C.c_int32 * n).from_address(s.len), np.int32).copy())

    def step_form(self) -> int:
        """Queries per work-group if one launch served the last step, else 0."""
        return self.hack.lib.hack_kvcache_step_form(self.handle)

    def as_cache(self) -> Cache:
        off, ln = self.view()
        return Cache(self.k, self.v, off, ln, self.pos)

    def close(self):
        if self.handle:
            self.hack.lib.hack_kvcache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Hack:
    """One library context (one element type / head_dim, one stream at a time)."""

    def __init__(self, heads: int, head_dim: int, dtype: str, max_units: int, max_cache_len: int,
                 max_queries: int, n_obs: int = 32, device: int = 0):
        import torch
        self.lib = load_library()
        self.heads, self.head_dim, self.device = heads, head_dim, device
        self.dtype = dtype
        self.torch_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        cfg = hack_config(device, heads, head_dim, HACK_F32 if dtype == "f32" else HACK_BF16, max_units,
                          max_cache_len, max_queries, n_obs)
        ctx = C.c_void_p()
        st = self.lib.hack_create(C.byref(ctx), C.byref(cfg))
        if st != 0:
            raise HackError(st, self.lib.hack_strerror(st).decode())
        self.ctx = ctx
        self._info = (head_dim, heads, device, self.torch_dtype, torch.float32, torch.int32, torch.uint8)

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.hack_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != 0:
            raise HackError(st, f"{self.lib.hack_strerror(st).decode()}: {self.lib.hack_last_error(self.ctx).decode()}")

    def check(self):
        """Raise if a kernel of an earlier call reported a problem (synchronise first)."""
        self._check(self.lib.hack_check(self.ctx))

    def set_score_mode(self, mode: int):
        """0: fused single launch (default); 1: two launches without in-kernel waits."""
        self._check(self.lib.hack_set_score_mode(self.ctx, mode))

    def score_mode(self) -> int:
        return int(self.lib.hack_get_score_mode(self.ctx))

    # ---- a1 ----
    def score(self, q, cache: Cache, scale: float, importance, k_new=None, q_idx=None, n_obs: Optional[int] = None,
              active=None):
        B, H, Nk, d = q.shape
        n_obs = min(32, Nk) if n_obs is None else n_obs
        qi = None if q_idx is None else _i32(q_idx)
        act = None if active is None else _u8(active)
        cs = cache.struct()
        self._check(self.lib.hack_score(self.ctx, B, Nk, _dev(q), _p(qi, C.c_int32), n_obs, scale, C.byref(cs),
                                        _dev(k_new), _p(act, C.c_uint8), _dev(importance),
                                        importance.stride(0), _stream()))

    def score_static(self, q, cache: Cache, scale: float, importance, k_new=None, q_idx=None,
                     n_obs: Optional[int] = None, active=None):
        """hack_score with all kernel scratch in the library's fixed device array (allocates nothing)."""
        B, H, Nk, d = q.shape
        n_obs = min(32, Nk) if n_obs is None else n_obs
        qi = None if q_idx is None else _i32(q_idx)
        act = None if active is None else _u8(active)
        cs = cache.struct()
        self._check(self.lib.hack_score_static(self.ctx, B, Nk, _dev(q), _p(qi, C.c_int32), n_obs, scale, C.byref(cs),
                                               _dev(k_new), _p(act, C.c_uint8), _dev(importance),
                                               importance.stride(0), _stream()))

    def score_item_keys(self, t_in) -> int:
        """Keys per wave of the launches that score units of t_in keys (bf16; 0 for fp32 contexts)."""
        t = _i32(t_in)
        v = int(self.lib.hack_score_item_keys(self.ctx, len(t), _p(t, C.c_int32)))
        if v < 0:
            self._check(v)
        return v

    # ---- a2 ----
    def select(self, B: int, importance, t_in, head_type, budget, n_init: int, n_recent: int, kept_idx) -> np.ndarray:
        t_in, budget, ht = _i32(t_in), _i32(budget), _u8(head_type)
        len_out = np.zeros(len(t_in), np.int32)
        self._check(self.lib.hack_select(self.ctx, B, _dev(importance), importance.stride(0), _p(t_in, C.c_int32),
                                         _p(ht, C.c_uint8), _p(budget, C.c_int32), n_init, n_recent,
                                         _dev(kept_idx), kept_idx.stride(0), _p(len_out, C.c_int32), _stream()))
        return len_out

    # ---- a3 ----
    def compact(self, B: int, Nk: int, cache_in: Cache, kept_idx, cache_out: Cache, k_new=None, v_new=None,
                pos_new: int = 0):
        ci, co = cache_in.struct(), cache_out.struct()
        self._check(self.lib.hack_compact(self.ctx, B, Nk, C.byref(ci), _dev(k_new), _dev(v_new), pos_new,
                                          _dev(kept_idx), kept_idx.stride(0), C.byref(co), _stream()))

    def merge(self, B: int, Nk: int, cache_in: Cache, kept_idx, cache_out: Cache, k_new=None, v_new=None, active=None):
        """Final-step merge: evicted rows folded into their nearest kept rows of cache_out (in place)."""
        ci, co = cache_in.struct(), cache_out.struct()
        act = None if active is None else _u8(active)
        self._check(self.lib.hack_merge(self.ctx, B, Nk, C.byref(ci), _dev(k_new), _dev(v_new), _dev(kept_idx),
                                        kept_idx.stride(0), _p(act, C.c_uint8), C.byref(co), _stream()))

    # ---- a4 ----
    def attn(self, q, cache: Cache, scale: float, out):
        B, H, Nk, d = q.shape
        cs = cache.struct()
        self._check(self.lib.hack_attn(self.ctx, B, Nk, _dev(q), C.byref(cs), scale, _dev(out), _stream()))

    def attn_variant(self, B: int, N_k: int) -> int:
        """0: 128-query work items; 1: 32-query work items with the keys split over the waves."""
        v = int(self.lib.hack_attn_variant(self.ctx, B, N_k))
        if v < 0:
            self._check(v)
        return v

    # ---- offline head classification ----
    def head_variance(self, q, cache: Cache, scale: float, sigma):
        """sigma (device float64 [B*H]) <- sum of column variances of Softmax(scale q k^T) per unit."""
        B, H, Nk, d = q.shape
        cs = cache.struct()
        self._check(self.lib.hack_head_variance(self.ctx, B, Nk, _dev(q), C.byref(cs), scale, _dev(sigma), _stream()))

    # ---- rotary positions, norms ----
    def rotate(self, x, rope: Rope, out, pos=None, pos0: int = 0):
        """out <- the rows of x rotated.  x: [B, heads, N, head_dim] in any strides with head_dim side by side; out: the same shape, contiguous (x itself if
        that is).  pos: int32 [axes, N] for all batch elements or [B, axes, N], with one axis also [N]; None: pos0, pos0 + 1, ..."""
        st = _ops_call.rotate(_ops_addr["rotate"], self.ctx and self.ctx.value, self._info, x, out, None, None, None, None, -1, 0.0, rope.address, rope.axes,
                              pos, pos0, _stream())
        if st != 0:
            self._check(st)

    def norm_rotate(self, q, k, norm: str, eps: float, q_weight, k_weight, rope: Optional[Rope], q_out, k_out, pos=None, pos0: int = 0):
        """Norms ("rms" or "l2") of the rows of q and k (or None), then their rotation (rope None: norms alone).  Operands as in rotate; weights: float32
        [head_dim] or [heads, head_dim], None: ones."""
        st = _ops_call.rotate(_ops_addr["norm_rotate"], self.ctx and self.ctx.value, self._info, q, q_out, q_weight, k, k_out, k_weight, NORMS[norm], eps,
                              None if rope is None else rope.address, 1 if rope is None else rope.axes, pos, pos0, _stream())
        if st != 0:
            self._check(st)

    # ---- caches in 4 bits ----
    def pack(self, B: int, Nk: int, packed: PackedCache, cache_in: Optional[Cache] = None, kept_idx=None, k_new=None, v_new=None,
             pos_new: int = 0, at=None):
        """Rows of cache_in and new ones ([B, heads, Nk, head_dim]), all in order or those of kept_idx, become rows at[u] .. packed.len[u] of unit u."""
        args = (_ops_addr["pack"], self.ctx and self.ctx.value, self._info, B, Nk, cache_in, k_new, v_new, pos_new, kept_idx)
        st = _ops_call.pack(*args, at, packed, _stream())
        if st is None:
            st = _ops_call.pack(*args, _exact(at, np.int32), packed, _stream())
        if st != 0:
            self._check(st)

    def unpack(self, B: int, packed: PackedCache, cache_out: Cache, first=None):
        """Rows first[u] .. first[u] + cache_out.len[u] of every unit, as rows of the context's element type."""
        args = (_ops_addr["unpack"], self.ctx and self.ctx.value, self._info, B, packed)
        st = _ops_call.unpack(*args, first, cache_out, _stream())
        if st is None:
            st = _ops_call.unpack(*args, _exact(first, np.int32), cache_out, _stream())
        if st != 0:
            self._check(st)

    def attn_packed(self, q, packed: PackedCache, scale: float, out):
        """q: [B, G heads, N, head_dim], G query heads to each cache."""
        st = _ops_call.attn(_ops_addr["attn_packed"], self.ctx and self.ctx.value, self._info, q, packed, scale, out, _stream())
        if st != 0:
            self._check(st)

    # ---- caches in pages ----
    def append_pages(self, k, v, cache: PagedCache, rope: Optional[Rope] = None, pos=None, fresh=None, q=None, q_out=None, norm: Optional[str] = None,
                     eps: float = 1e-6, q_weight=None, k_weight=None):
        """The first fresh[b] (int32 [B]; None: all) rows of k and v ([B, heads, N, head_dim] in any strides) become the last ones of their sequences, k normed and
        rotated (rope None: not); q: normed and rotated into q_out.  pos as in rotate; None: the rows' numbers in the cache."""
        st = _ops_call.append_pages(_ops_addr["append_pages"], self.ctx and self.ctx.value, self._info, q, q_out, q_weight, k, k_weight, v,
                                    -1 if norm is None else NORMS[norm], eps, None if rope is None else rope.address, 1 if rope is None else rope.axes, pos, fresh,
                                    cache._info, _stream())
        if st != 0:
            self._check(st)

    def attn_pages(self, q, cache: PagedCache, scale: float, out, causal: bool = False, fresh=None, shared=None):
        """q: [B, G heads, N, head_dim], G query heads to each cache; the first fresh[b] queries (None: all) see their sequence's rows, causal: those up to their own.
        shared: (first, count, rows) of batch elements that have the same first rows, by the table of each."""
        st = _ops_call.attn_pages(_ops_addr["attn_pages"], self.ctx and self.ctx.value, self._info, q, cache._info, fresh, causal, shared, scale, out, _stream())
        if st != 0:
            self._check(st)

    # ---- a5 ----
    def managed_cache(self, cap, with_pos: bool = True) -> ManagedCache:
        return ManagedCache(self, cap, with_pos)

    def step(self, cache: ManagedCache, q, k_new, v_new, head_type, budget, n_init: int, scale: float, out,
             kept_idx=None, final: bool = False):
        """final=True: hack_step_final (the last scale step; contextual units merge what they discard)."""
        fn, kstride = _step_addr[1 if final else 0], 0 if kept_idx is None else kept_idx.stride(0)
        ctx, handle, stream = self.ctx and self.ctx.value, cache.handle and cache.handle.value, _stream()
        st = _step_call(fn, ctx, handle, q, k_new, v_new, head_type, budget, n_init, scale, out, kept_idx, kstride, stream)
        if st is None:
            st = _step_call(fn, ctx, handle, q, k_new, v_new, _u8(head_type), _i32(budget), n_init, scale, out, kept_idx, kstride, stream)
        if st != 0:
            self._check(st)
