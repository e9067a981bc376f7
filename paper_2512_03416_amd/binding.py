"""ctypes binding with the same names as include/tokenscale.h (argument marshalling only)."""
from __future__ import annotations

import ctypes
import os
import sys
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtokenscale.so")

DTYPES = {"f32": 0, "bf16": 1, "fp8": 2}
TS_OK, TS_ERR_INVALID_ARG, TS_ERR_UNSUPPORTED, TS_ERR_HIP, TS_ERR_NOMEM = 0, -1, -2, -3, -4
TS_VELOCITY_RESET, TS_VELOCITY_SYNC = 1, 2

EXPORTS = ["ts_check_desc", "ts_cache_bytes", "ts_create", "ts_destroy", "ts_reserve", "ts_kv_append",
           "ts_mixed_paged_attention", "ts_mixed_paged_attention_noalloc", "ts_token_velocity", "ts_last_error", "ts_set_option",
           "ts_get_option", "ts_plan_describe", "ts_plan_export", "ts_kernel_times",
           "ts_rope_frequencies", "ts_set_rope", "ts_rope_kv_append", "ts_tree_attention", "ts_reserve_tree", "ts_tree_masks",
           "ts_kv_move", "ts_kv_read"]
CALIB_EXPORTS = ["ts_calib_copy", "ts_calib_read", "ts_calib_mfma"]     # include/tokenscale_calib.h

KERNEL_NAMES = ["append", "decode", "combine", "prefill", "rows", "mixed"]


class TokenScaleError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"tokenscale error {code}: {msg}")
        self.code = code


class Desc(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("q_dtype", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
                ("num_pages", ctypes.c_int64), ("max_pages_per_seq", ctypes.c_int32)]

    @classmethod
    def make(cls, Hq, Hkv, D, q_dtype, kv_dtype, num_pages, max_pages_per_seq, page_size=16):
        qd = DTYPES[q_dtype] if isinstance(q_dtype, str) else int(q_dtype)
        kd = DTYPES[kv_dtype] if isinstance(kv_dtype, str) else int(kv_dtype)
        return cls(Hq, Hkv, D, page_size, qd, kd, num_pages, max_pages_per_seq)


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "wavelength": 4, "table": 5}
TREE_MAX_NODES, MAX_MOVES = 256, 64


class RopeDesc(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("original_length", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("attn_scale", ctypes.c_double),
                ("table", ctypes.c_void_p)]

    @classmethod
    def make(cls, rot_dim, base=10000.0, layout="half", scaling="none", factor=1.0, original_length=0, low=0.0, high=0.0,
             attn_scale=0.0, table=None):
        """table: the rot_dim / 2 angles per position, which select the scaling "table"."""
        for name, known in ((layout, ROPE_LAYOUTS), (scaling, ROPE_SCALINGS)):
            if isinstance(name, str) and name not in known:
                raise ValueError(f"{name!r} is none of {sorted(known)}")
        values = None
        if table is not None:
            scaling = "table"
            values = np.ascontiguousarray(table, dtype=np.float64)
            if values.shape != (int(rot_dim) // 2,):
                raise ValueError(f"table has shape {values.shape}, expected {(int(rot_dim) // 2,)}")
        d = cls(int(rot_dim), ROPE_LAYOUTS.get(layout, layout), ROPE_SCALINGS.get(scaling, scaling), int(original_length), base,
                factor, low, high, attn_scale, values.ctypes.data if values is not None else None)
        d._values = values                                 # (the description points into it)
        return d


class Velocity(ctypes.Structure):
    _fields_ = [("prefill_tok_per_s", ctypes.c_double), ("decode_tok_per_s", ctypes.c_double),
                ("prefill_tokens", ctypes.c_uint64), ("decode_tokens", ctypes.c_uint64),
                ("passes", ctypes.c_uint64), ("window_s", ctypes.c_double)]


class KernelStats(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_uint64 * 6), ("mean_ms", ctypes.c_double * 6)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int64), ("decode_tokens", ctypes.c_int64),
                ("prefill_tokens", ctypes.c_int64), ("n_decode_items", ctypes.c_int32),
                ("n_combine_rows", ctypes.c_int32), ("n_prefill_tiles", ctypes.c_int32),
                ("n_generic_rows", ctypes.c_int32), ("split_pages", ctypes.c_int32),
                ("tile_tokens", ctypes.c_int32), ("partial_slots", ctypes.c_int64),
                ("ctx_pages", ctypes.c_int64), ("mixed_mode", ctypes.c_int32), ("prefill_workgroups", ctypes.c_int32),
                ("widened_pages", ctypes.c_int64), ("prefill_parts", ctypes.c_int64)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads the built library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2512_03416_amd.build` "
                          "or __graft_entry__.build(); there is no CPU fallback")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32p = ctypes.c_void_p, ctypes.c_void_p
    lib.ts_check_desc.argtypes = [ctypes.POINTER(Desc)]
    lib.ts_check_desc.restype = ctypes.c_int
    lib.ts_cache_bytes.argtypes = [ctypes.POINTER(Desc)]
    lib.ts_cache_bytes.restype = ctypes.c_int64
    lib.ts_create.argtypes = [ctypes.POINTER(Desc), ctypes.c_int, ctypes.POINTER(vp)]
    lib.ts_create.restype = ctypes.c_int
    lib.ts_destroy.argtypes = [vp]
    lib.ts_destroy.restype = ctypes.c_int
    lib.ts_reserve.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64]
    lib.ts_reserve.restype = ctypes.c_int
    lib.ts_kv_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int]
    lib.ts_kv_append.restype = ctypes.c_int
    lib.ts_mixed_paged_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32p, i32p,
                                             ctypes.c_int, ctypes.c_float, vp]
    lib.ts_mixed_paged_attention.restype = ctypes.c_int
    lib.ts_mixed_paged_attention_noalloc.argtypes = lib.ts_mixed_paged_attention.argtypes
    lib.ts_mixed_paged_attention_noalloc.restype = ctypes.c_int
    lib.ts_token_velocity.argtypes = [vp, ctypes.POINTER(Velocity), ctypes.c_int]
    lib.ts_token_velocity.restype = ctypes.c_int
    lib.ts_last_error.argtypes = [vp]
    lib.ts_last_error.restype = ctypes.c_char_p
    lib.ts_set_option.argtypes = [vp, ctypes.c_char_p, ctypes.c_int64]
    lib.ts_set_option.restype = ctypes.c_int
    lib.ts_get_option.argtypes = [vp, ctypes.c_char_p, ctypes.POINTER(ctypes.c_int64)]
    lib.ts_get_option.restype = ctypes.c_int
    lib.ts_plan_describe.argtypes = [ctypes.POINTER(Desc), i32p, i32p, ctypes.c_int, ctypes.c_int32,
                                     ctypes.POINTER(PlanInfo)]
    lib.ts_plan_describe.restype = ctypes.c_int
    lib.ts_plan_export.argtypes = [ctypes.POINTER(Desc), i32p, i32p, ctypes.c_int, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_int, i32p, ctypes.c_int64]
    lib.ts_plan_export.restype = ctypes.c_int64
    lib.ts_kernel_times.argtypes = [vp, ctypes.POINTER(KernelStats), ctypes.c_int]
    lib.ts_kernel_times.restype = ctypes.c_int
    lib.ts_rope_frequencies.argtypes = [ctypes.POINTER(RopeDesc), vp, vp]
    lib.ts_rope_frequencies.restype = ctypes.c_int
    lib.ts_set_rope.argtypes = [vp, ctypes.POINTER(RopeDesc)]
    lib.ts_set_rope.restype = ctypes.c_int
    lib.ts_rope_kv_append.argtypes = [vp, vp, vp, ctypes.c_int64, vp, ctypes.c_int64, vp, ctypes.c_int64, vp, vp, vp, vp, vp, vp, vp,
                                      i32p, i32p, ctypes.c_int]
    lib.ts_rope_kv_append.restype = ctypes.c_int
    lib.ts_tree_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, i32p, i32p, ctypes.c_int, ctypes.c_float, vp]
    lib.ts_tree_attention.restype = ctypes.c_int
    lib.ts_reserve_tree.argtypes = [vp]
    lib.ts_reserve_tree.restype = ctypes.c_int
    lib.ts_tree_masks.argtypes = [i32p, i32p, ctypes.c_int, ctypes.c_int, vp, i32p]
    lib.ts_tree_masks.restype = ctypes.c_int
    lib.ts_kv_move.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int]
    lib.ts_kv_move.restype = ctypes.c_int
    lib.ts_kv_read.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int, vp, vp]
    lib.ts_kv_read.restype = ctypes.c_int
    lib.ts_calib_copy.argtypes = [vp, vp, vp, ctypes.c_int64]
    lib.ts_calib_copy.restype = ctypes.c_int
    lib.ts_calib_read.argtypes = [vp, vp, vp, ctypes.c_int64]
    lib.ts_calib_read.restype = ctypes.c_int
    lib.ts_calib_mfma.argtypes = [vp, vp, vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int64)]
    lib.ts_calib_mfma.restype = ctypes.c_int
    _lib = lib
    return lib


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _np_ptr(a: Optional[np.ndarray]):
    return ctypes.c_void_p(a.ctypes.data if a is not None and a.size else 0) if a is not None else ctypes.c_void_p(0)


def _dev_ptr(t) -> int:
    """Device pointer of a torch tensor (or None / int), as the integer that a void* argument takes."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a GPU tensor")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _i32_bytes(a) -> bytes:
    """int32 values as bytes, which a void* argument takes as they are (host arrays are consumed by the call).
    A quarter of the time of going through numpy's ctypes interface, twice per pass."""
    return np.asarray(a, dtype=np.int32).tobytes()


def _host_lens(first, second=None):
    """(first, second: int32 arrays as bytes, second may be None; their common length; the sum of the first)."""
    one = np.asarray(first, dtype=np.int32)
    n = one.size
    other = None
    if second is not None:
        two = np.asarray(second, dtype=np.int32)
        if two.size != n:
            raise ValueError(f"lengths of {[n, two.size]} sequences")
        other = two.tobytes()
    # (adding up a short list takes a tenth of numpy's sum)
    total = sum(one.reshape(-1).tolist()) if n < 64 else int(one.sum(dtype=np.int64))
    return one.tobytes(), other, n, total


def _count(lens) -> int:
    try:
        return len(lens)
    except TypeError:                                      # a single number
        return 1


def check_desc(desc: Desc) -> int:
    return int(load_library().ts_check_desc(ctypes.byref(desc)))


def cache_bytes(desc: Desc) -> int:
    return int(load_library().ts_cache_bytes(ctypes.byref(desc)))


def plan_describe(desc: Desc, q_lens, ctx_lens, split_pages: int = 0) -> PlanInfo:
    ql, cl = _i32(q_lens), _i32(ctx_lens)
    info = PlanInfo()
    rc = load_library().ts_plan_describe(ctypes.byref(desc), _np_ptr(ql), _np_ptr(cl), len(ql),
                                         split_pages, ctypes.byref(info))
    if rc != TS_OK:
        raise TokenScaleError(rc, "ts_plan_describe")
    return info


PLAN_LISTS = {"decode": (0, 8), "combine": (1, 4), "prefill": (2, 12), "pfmap": (3, 2), "rows": (4, 4),
              "queue": (5, 4), "qoff": (6, 1), "append": (7, 8),
              "append_rows": (8, 4), "widen": (9, 2), "pfcombine": (10, 4)}


def plan_export(desc: Desc, q_lens, ctx_lens, which: str, split_pages: int = 0, wg_slots: int = 0,
                mixed_mode: int = -1) -> np.ndarray:
    """One of the planner's work lists as an int32 array [records, words] (see tokenscale.h)."""
    ql, cl = _i32(q_lens), _i32(ctx_lens)
    lib = load_library()
    code, words = PLAN_LISTS[which]
    n = lib.ts_plan_export(ctypes.byref(desc), _np_ptr(ql), _np_ptr(cl), len(ql), split_pages, wg_slots, mixed_mode,
                           code, ctypes.c_void_p(0), 0)
    if n < 0:
        raise TokenScaleError(int(n), "ts_plan_export")
    out = np.zeros((int(n), words), dtype=np.int32)
    if n:
        lib.ts_plan_export(ctypes.byref(desc), _np_ptr(ql), _np_ptr(cl), len(ql), split_pages, wg_slots, mixed_mode,
                           code, _np_ptr(out), int(n) * words)
    return out


def plan_decode_items(desc: Desc, q_lens, ctx_lens, split_pages: int = 0) -> np.ndarray:
    return plan_export(desc, q_lens, ctx_lens, "decode", split_pages)[:, :5]


def rope_frequencies(rot_dim: int, **kw):
    """(angles per position of the rot_dim / 2 pairs, factor of cosine and sine); arguments as for Context.set_rope."""
    desc = RopeDesc.make(rot_dim, **kw)
    freq, scale = np.zeros(max(1, int(rot_dim) // 2)), ctypes.c_double(0.0)
    rc = load_library().ts_rope_frequencies(ctypes.byref(desc), _np_ptr(freq), ctypes.byref(scale))
    if rc != TS_OK:
        raise TokenScaleError(rc, "ts_rope_frequencies")
    return freq, float(scale.value)


def tree_masks(parents, q_lens, mask_words: int = 0):
    """(masks uint64 [T, mask_words], depths int32 [T]) of trees given by their nodes' parents (-1 = a root).  mask_words 0 = as
    many as the largest tree needs.  torch has no use for uint64 here: hand masks over as masks.view(np.int64)."""
    pa, ql = _i32(parents), _i32(q_lens)
    if pa.size != int(ql.sum()):
        raise ValueError(f"{pa.size} parents for {int(ql.sum())} nodes")
    words = mask_words or max(1, -(-int(ql.max(initial=0)) // 64))
    masks, depths = np.zeros((pa.size, words), np.uint64), np.zeros(pa.size, np.int32)
    rc = load_library().ts_tree_masks(_np_ptr(pa), _np_ptr(ql), len(ql), words, _np_ptr(masks), _np_ptr(depths))
    if rc != TS_OK:
        raise TokenScaleError(rc, "ts_tree_masks")
    return masks, depths


_raw_stream = None


def _current_stream(device=None) -> int:
    """Handle of torch's current stream on a GPU (None = the current one).  torch.cuda.current_stream() builds a Stream object for it (2.9 us a call); the
    function under it returns the handle itself (0.1 us)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                        # initialises the GPU if nothing has yet
        get, current = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = (lambda d: get(current() if d is None else d)) if get and current else (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream(device)


class Context:
    """Owns a ts_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, desc: Desc, device: int = 0):
        self._lib = load_library()
        self.desc = desc
        self.device = device
        self._cache_bytes = cache_bytes(desc)
        self._hq, self._hkv, self._dim, self._width = desc.num_q_heads, desc.num_kv_heads, desc.head_dim, desc.max_pages_per_seq
        self._h = ctypes.c_void_p(0)
        rc = self._lib.ts_create(ctypes.byref(desc), device, ctypes.byref(self._h))
        if rc != TS_OK:
            msg = self._lib.ts_last_error(ctypes.c_void_p(0)).decode()
            self._h = ctypes.c_void_p(0)
            raise TokenScaleError(rc, msg)

    def __getattr__(self, name):
        # torch's types, which become attributes once torch is there.  Before, no argument can be a tensor, and none is compared.
        if name not in ("_f32", "_i32", "_i64", "_q_type"):
            raise AttributeError(name)
        torch = sys.modules.get("torch")
        if torch is None:
            return None
        self._f32, self._i32, self._i64 = torch.float32, torch.int32, torch.int64
        self._q_type = torch.float32 if self.desc.q_dtype == DTYPES["f32"] else torch.bfloat16
        return self.__dict__[name]

    def close(self):
        if self._h:
            self._lib.ts_destroy(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        return self._lib.ts_last_error(self._h).decode()

    def _check(self, rc: int):
        if rc != TS_OK:
            raise TokenScaleError(rc, self.last_error())

    @staticmethod
    def _stream(stream, device=None) -> int:
        if stream is None:
            return _current_stream(device)
        if isinstance(stream, int):
            return stream
        return stream.cuda_stream

    def reserve(self, max_tokens: int, max_seqs: int, max_ctx_pages: int):
        self._check(self._lib.ts_reserve(self._h, max_tokens, max_seqs, max_ctx_pages))

    def set_option(self, name: str, value: int):
        self._check(self._lib.ts_set_option(self._h, name.encode(), int(value)))

    def get_option(self, name: str) -> int:
        v = ctypes.c_int64(0)
        rc = self._lib.ts_get_option(self._h, name.encode(), ctypes.byref(v))
        if rc != TS_OK:
            raise TokenScaleError(rc, f"ts_get_option({name})")
        return int(v.value)

    def kv_append(self, k_new, v_new, k_cache, v_cache, k_scale, v_scale, block_table, q_lens,
                  ctx_lens, stream=None):
        self._check(self._lib.ts_kv_append(self._h, self._stream(stream), _dev_ptr(k_new), _dev_ptr(v_new),
                                           _dev_ptr(k_cache), _dev_ptr(v_cache), _dev_ptr(k_scale),
                                           _dev_ptr(v_scale), _dev_ptr(block_table), _i32_bytes(q_lens),
                                           _i32_bytes(ctx_lens), _count(q_lens)))

    def mixed_paged_attention(self, q, k_new, v_new, k_cache, v_cache, k_scale, v_scale, block_table,
                              q_lens, ctx_lens, sm_scale: float, out, stream=None, noalloc: bool = False):
        """noalloc=True calls ts_mixed_paged_attention_noalloc (same arguments)."""
        fn = self._lib.ts_mixed_paged_attention_noalloc if noalloc else self._lib.ts_mixed_paged_attention
        rc = fn(self._h, self._stream(stream), _dev_ptr(q), _dev_ptr(k_new), _dev_ptr(v_new),
                _dev_ptr(k_cache), _dev_ptr(v_cache), _dev_ptr(k_scale), _dev_ptr(v_scale),
                _dev_ptr(block_table), _i32_bytes(q_lens), _i32_bytes(ctx_lens), _count(q_lens), sm_scale, _dev_ptr(out))
        if rc != TS_OK:
            self._check(rc)

    def set_rope(self, rot_dim: int, **kw):
        """Rotation of this layer's heads for rope_kv_append: base, layout ("half" / "interleaved"), scaling ("none", "linear",
        "ntk", "yarn", "wavelength") with factor, original_length, low, high, attn_scale; or table = angles per position."""
        desc = RopeDesc.make(rot_dim, **kw)
        self._check(self._lib.ts_set_rope(self._h, ctypes.byref(desc)))

    # The following calls check their tensors: a wrong size or device would not be noticed before the GPU reads past an end.  (Written
    # for few Python operations: a call of a few short sequences takes the GPU about 5 us.)

    def _ptr(self, t, name: str, dtype, n: int) -> int:
        """Device pointer of a packed tensor of at least n elements of dtype (None = any) on this context's GPU."""
        if t is None:
            return 0
        if t.__class__ is int:
            return t
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on GPU {self.device}")
        if dtype is not None and t.dtype is not dtype:
            raise ValueError(f"{name} is {t.dtype}, expected {dtype}")
        if t.numel() < n:
            raise ValueError(f"{name} has {t.numel()} elements, needs {n}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    def _rows(self, t, name: str, heads: int, total: int):
        """(device pointer, elements from row to row) of token rows [tokens, heads, dim], whose heads and dims are packed."""
        if t is None:
            return 0, 0
        dim = self._dim
        if t.dim() != 3:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [{total}, {heads}, {dim}]")
        tokens, h, d = t.shape
        if tokens < total or h != heads or d != dim:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [{total}, {heads}, {dim}]")
        if total == 0:
            return 0, 0
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on GPU {self.device}")
        if t.dtype is not self._q_type:
            raise ValueError(f"{name} is {t.dtype}, expected {self._q_type}")
        row, head, one = t.stride()
        if one != 1 or (head != dim and heads > 1):
            raise ValueError(f"{name}: a row's heads and dims must be packed")
        if total > 1 and row < heads * dim:                # (an expanded tensor's 0 would be taken for packed rows)
            raise ValueError(f"{name}: rows {row} elements apart overlap")
        return t.data_ptr(), row if total > 1 else 0

    def _cache_ptr(self, t, name: str) -> int:
        if t is None:
            return 0
        if t.__class__ is int:
            return t
        n = t.numel()
        if n < self._cache_bytes and n * t.element_size() < self._cache_bytes:
            raise ValueError(f"{name} has {n * t.element_size()} bytes, needs {self._cache_bytes}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on GPU {self.device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    def _cache_ptrs(self, k_cache, v_cache, k_scale, v_scale):
        """Device pointers of the caches and their scales."""
        ks = 0 if k_scale is None else self._ptr(k_scale, "k_scale", self._f32, self._hkv)
        vs = 0 if v_scale is None else self._ptr(v_scale, "v_scale", self._f32, self._hkv)
        return self._cache_ptr(k_cache, "k_cache"), self._cache_ptr(v_cache, "v_cache"), ks, vs

    def rope_kv_append(self, q, k_new, v_new, q_out, k_cache, v_cache, k_scale, v_scale, block_table, q_lens, ctx_lens,
                       positions=None, stream=None):
        """q, k_new, v_new: [T, heads, dim], rows may be strided (slices of one projection's output); q_out packed, may be q."""
        ptr, rows, hq, hkv = self._ptr, self._rows, self._hq, self._hkv
        ql, cl, n, total = _host_lens(q_lens, ctx_lens)
        q_at, q_row = rows(q, "q", hq, total)
        k_at, k_row = rows(k_new, "k_new", hkv, total)
        v_at, v_row = rows(v_new, "v_new", hkv, total)
        kc, vc, ks, vs = self._cache_ptrs(k_cache, v_cache, k_scale, v_scale)
        rc = self._lib.ts_rope_kv_append(self._h, self._stream(stream, self.device), q_at, q_row, k_at, k_row, v_at, v_row,
                                         ptr(q_out, "q_out", self._q_type, total * hq * self._dim), kc, vc, ks, vs,
                                         ptr(block_table, "block_table", self._i32, n * self._width),
                                         0 if positions is None else ptr(positions, "positions", self._i32, total), ql, cl, n)
        if rc != TS_OK:
            self._check(rc)

    def reserve_tree(self):
        """Allocates tree_attention's scratch now (before a capture, say)."""
        self._check(self._lib.ts_reserve_tree(self._h))

    def tree_attention(self, q, k_cache, v_cache, k_scale, v_scale, block_table, tree_mask, q_lens, ctx_lens, sm_scale: float, out,
                       stream=None):
        """tree_mask: int64 [T, words] on the GPU (see tree_masks), or None for chains."""
        ptr = self._ptr
        ql, cl, n, total = _host_lens(q_lens, ctx_lens)
        words = 0
        if tree_mask is not None:
            if tree_mask.dim() != 2:
                raise ValueError(f"tree_mask has shape {tuple(tree_mask.shape)}, expected [tokens, words]")
            words = tree_mask.shape[1]
        elems = total * self._hq * self._dim
        kc, vc, ks, vs = self._cache_ptrs(k_cache, v_cache, k_scale, v_scale)
        rc = self._lib.ts_tree_attention(self._h, self._stream(stream, self.device), ptr(q, "q", self._q_type, elems), kc, vc, ks, vs,
                                         ptr(block_table, "block_table", self._i32, n * self._width),
                                         ptr(tree_mask, "tree_mask", self._i64, total * words), words, ql, cl, n, sm_scale,
                                         ptr(out, "out", self._q_type, elems))
        if rc != TS_OK:
            self._check(rc)

    def kv_move(self, k_cache, v_cache, block_table, src, dst, move_lens, ctx_lens, stream=None):
        """Entries at positions dst take what positions src held; pairs packed by sequence, -1 = no pair."""
        ptr = self._ptr
        ml, cl, n, total = _host_lens(move_lens, ctx_lens)
        kc, vc, _, _ = self._cache_ptrs(k_cache, v_cache, None, None)
        rc = self._lib.ts_kv_move(self._h, self._stream(stream, self.device), kc, vc,
                                  ptr(block_table, "block_table", self._i32, n * self._width),
                                  ptr(src, "src", self._i32, total), ptr(dst, "dst", self._i32, total), ml, cl, n)
        if rc != TS_OK:
            self._check(rc)

    def kv_read(self, k_cache, v_cache, k_scale, v_scale, block_table, starts, lens, k_out, v_out, stream=None):
        """Tokens starts .. starts + lens - 1 of every sequence as rows [sum of lens, KV heads, dim]; starts None = 0."""
        ptr = self._ptr
        ln, st, n, total = _host_lens(lens, starts)
        elems = total * self._hkv * self._dim
        kc, vc, ks, vs = self._cache_ptrs(k_cache, v_cache, k_scale, v_scale)
        rc = self._lib.ts_kv_read(self._h, self._stream(stream, self.device), kc, vc, ks, vs,
                                  ptr(block_table, "block_table", self._i32, n * self._width), st, ln, n,
                                  ptr(k_out, "k_out", self._q_type, elems), ptr(v_out, "v_out", self._q_type, elems))
        if rc != TS_OK:
            self._check(rc)

    def kernel_times(self, reset: bool = False) -> dict:
        """{kernel name: (launches, mean ms)} of the launches timed since the last reset."""
        st = KernelStats()
        self._check(self._lib.ts_kernel_times(self._h, ctypes.byref(st), 1 if reset else 0))
        return {n: (int(st.launches[i]), float(st.mean_ms[i])) for i, n in enumerate(KERNEL_NAMES)}

    def token_velocity(self, reset: bool = False, sync: bool = False) -> Velocity:
        v = Velocity()
        flags = (TS_VELOCITY_RESET if reset else 0) | (TS_VELOCITY_SYNC if sync else 0)
        self._check(self._lib.ts_token_velocity(self._h, ctypes.byref(v), flags))
        return v


def calib_copy(src, dst, nbytes: int, stream=None):
    rc = load_library().ts_calib_copy(Context._stream(stream), _dev_ptr(src), _dev_ptr(dst), nbytes)
    if rc != TS_OK:
        raise TokenScaleError(rc, "ts_calib_copy")


def calib_read(src, result4, nbytes: int, stream=None):
    rc = load_library().ts_calib_read(Context._stream(stream), _dev_ptr(src), _dev_ptr(result4), nbytes)
    if rc != TS_OK:
        raise TokenScaleError(rc, "ts_calib_read")


def calib_mfma(operands, result4, iters: int, softmax: bool, stream=None) -> int:
    """Launches the MFMA calibration stream; returns the floating-point operations of the launch."""
    flops = ctypes.c_int64(0)
    rc = load_library().ts_calib_mfma(Context._stream(stream), _dev_ptr(operands), _dev_ptr(result4), int(iters),
                                      int(bool(softmax)), ctypes.byref(flops))
    if rc != 0:
        raise TokenScaleError(rc, "ts_calib_mfma")
    return int(flops.value)
