"""ctypes binding of the C ABI declared in ``include/buzz.h``.

Argument marshalling only: every step of the decode path runs in the HIP kernels of ``libbuzz.so``.
PyTorch supplies device memory (tensors' ``data_ptr()``) and the HIP stream; nothing here computes.
There is no fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libbuzz.so")

FLAG_AUTO_EVICT = 1
FLAG_DRY_RUN = 2
FLAG_STREAMING = 4
FLAG_CACHED = 8
FLAG_LOG_N = 16
FLAG_THRESHOLD_TOTAL = 32
FLAG_DETERMINISTIC = 64
FLAG_INTERVAL_NEW = 128
FLAG_DEVICE_MERGE = 256
FLAG_GLOBAL_TOPK = 512
DTYPE_CODES = {"fp32": 0, "fp16": 1, "bf16": 2}
PAGE_DTYPE_CODES = dict(DTYPE_CODES, e4m3=3)

EXPORTS = ["buzz_workspace_bytes", "buzz_cache_create", "buzz_prefill", "buzz_decode_step",
           "buzz_decode_step_static", "buzz_evict",
           "buzz_cache_destroy", "buzz_cache_len", "buzz_cache_export", "buzz_cache_import", "buzz_cache_set_splits",
           "buzz_cache_override_die_map", "buzz_cache_profile",
           "buzz_cache_profile_read", "buzz_bench_copy", "buzz_suggest_threshold", "buzz_strerror",
           "buzz_qk_norm_rotate", "buzz_paged_workspace_bytes", "buzz_paged_create", "buzz_paged_destroy",
           "buzz_paged_append", "buzz_paged_read", "buzz_paged_decode"]


class BuzzError(RuntimeError):
    def __init__(self, code: int, what: str, text: str):
        super().__init__(f"{what}: {text} ({code})")
        self.code = code


class _Cfg(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("kv_dtype", ctypes.c_int32), ("sink", ctypes.c_int32),
        ("window", ctypes.c_int32), ("segment", ctypes.c_int32), ("keep", ctypes.c_int32),
        ("evict_every", ctypes.c_int32), ("old_stride", ctypes.c_int32), ("flags", ctypes.c_uint32),
        ("max_context", ctypes.c_int64), ("capacity", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float), ("reserved", ctypes.c_int32),
    ]


class _Profile(ctypes.Structure):
    _fields_ = [("attn_launches", ctypes.c_int64), ("epilogue_launches", ctypes.c_int64),
                ("evictions", ctypes.c_int64), ("attn_ms", ctypes.c_double), ("epilogue_ms", ctypes.c_double),
                ("evict_ms", ctypes.c_double), ("attn_row_bytes", ctypes.c_double)]


class _Rotary(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class _PagedCfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "page_dtype",
                                              "page_rows", "n_pages", "table_cols", "sink", "window")] + [
        ("flags", ctypes.c_uint32), ("softmax_scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class _Pages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_exp", "v_exp")]


@dataclass
class BuzzConfig:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    kv_dtype: str          # "fp32" | "fp16" | "bf16"
    sink: int
    window: int
    segment: int
    keep: int
    evict_every: int
    max_context: int
    old_stride: int = 0    # 0 => floor((s+1)/2), the paper's default; 1 => survivors persist
    flags: int = FLAG_AUTO_EVICT
    capacity: int = 0
    softmax_scale: float = 0.0

    def to_c(self) -> _Cfg:
        return _Cfg(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, DTYPE_CODES[self.kv_dtype],
                    self.sink, self.window, self.segment, self.keep, self.evict_every, self.old_stride,
                    self.flags, self.max_context, self.capacity, self.softmax_scale, 0)


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load ``libbuzz.so``; build it first if it has never been built.  Raises if that fails."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from .build import build
        build()
    lib = ctypes.CDLL(_LIB_PATH)
    P, I64 = ctypes.c_void_p, ctypes.c_int64
    lib.buzz_workspace_bytes.argtypes = [ctypes.POINTER(_Cfg), ctypes.POINTER(ctypes.c_size_t)]
    lib.buzz_cache_create.argtypes = [ctypes.POINTER(_Cfg), P, ctypes.c_size_t, ctypes.POINTER(P)]
    lib.buzz_prefill.argtypes = [P, P, P, I64, P, I64, P, P]
    lib.buzz_decode_step.argtypes = [P, P, P, P, P, P]
    lib.buzz_decode_step_static.argtypes = [P, P, P, P, P, P]
    lib.buzz_evict.argtypes = [P, P]
    lib.buzz_cache_destroy.argtypes = [P]
    lib.buzz_cache_len.argtypes = [P, ctypes.POINTER(I64), ctypes.POINTER(I64), ctypes.POINTER(I64)]
    lib.buzz_cache_export.argtypes = [P, P, P, P, P, P]
    lib.buzz_cache_import.argtypes = [P, P, P, P, P, I64, I64, I64, P]
    lib.buzz_cache_set_splits.argtypes = [P, ctypes.c_int32]
    lib.buzz_cache_override_die_map.argtypes = [P, I64]
    lib.buzz_cache_profile.argtypes = [P, ctypes.c_int]
    lib.buzz_cache_profile_read.argtypes = [P, ctypes.POINTER(_Profile)]
    lib.buzz_bench_copy.argtypes = [P, P, ctypes.c_size_t, P]
    lib.buzz_suggest_threshold.argtypes = [ctypes.c_int32, ctypes.c_int32]
    lib.buzz_suggest_threshold.restype = ctypes.c_int64
    I32 = ctypes.c_int32
    lib.buzz_qk_norm_rotate.argtypes = [I32, I32, I32, I32, P, P, P, P, P, I32, I64, P, P, P]
    lib.buzz_paged_workspace_bytes.argtypes = [ctypes.POINTER(_PagedCfg), ctypes.POINTER(ctypes.c_size_t)]
    lib.buzz_paged_create.argtypes = [ctypes.POINTER(_PagedCfg), ctypes.POINTER(_Pages), P, ctypes.c_size_t, P, ctypes.POINTER(P)]
    lib.buzz_paged_destroy.argtypes = [P]
    lib.buzz_paged_append.argtypes = [P, P, P, P, P, P, I32, I64, P, P, P, P]
    lib.buzz_paged_read.argtypes = [P, P, P, I32, I64, P, P, P, P]
    lib.buzz_paged_decode.argtypes = [P, P, I32, P, P, P, P, P]
    lib.buzz_strerror.argtypes = [ctypes.c_int]
    lib.buzz_strerror.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(rc: int, what: str):
    if rc != 0:
        raise BuzzError(rc, what, load_library().buzz_strerror(rc).decode())


def workspace_bytes(cfg: BuzzConfig) -> int:
    out = ctypes.c_size_t()
    c = cfg.to_c()
    _check(load_library().buzz_workspace_bytes(ctypes.byref(c), ctypes.byref(out)), "buzz_workspace_bytes")
    return out.value


def suggest_threshold(segment: int, window: int) -> int:
    """Eviction threshold recommended by the Parameter Estimation theorem (Sec. 3.4) for FLAG_THRESHOLD_TOTAL."""
    return load_library().buzz_suggest_threshold(segment, window)


def bench_copy(dst, src, stream=None):
    """Plain device copy of ``src`` into ``dst`` (same byte size) with the library's own copy kernel."""
    nbytes = src.numel() * src.element_size()
    _check(load_library().buzz_bench_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream(stream)), "buzz_bench_copy")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


class BuzzCache:
    """One layer's BUZZ cache on the GPU.  Tensors must be contiguous, on the GPU and of the config's dtype."""

    def __init__(self, cfg: BuzzConfig, device="cuda"):
        self.cfg = cfg
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.nbytes = workspace_bytes(cfg)
        self.dry = bool(cfg.flags & FLAG_DRY_RUN)
        self.workspace = None
        ws_ptr = None
        if not self.dry:
            import torch
            self.workspace = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
            ws_ptr = self.workspace.data_ptr()
        c = cfg.to_c()
        _check(self._lib.buzz_cache_create(ctypes.byref(c), ws_ptr, self.nbytes, ctypes.byref(self._h)),
               "buzz_cache_create")

    def close(self):
        if getattr(self, "_h", None):
            self._lib.buzz_cache_destroy(self._h)
            self._h = None

    __del__ = close

    def _stream(self, stream):
        return None if self.dry else _stream(stream)

    def prefill(self, k, v, q_obs=None, init_score=None, stream=None, n_prompt=None):
        n_prompt = k.shape[2] if n_prompt is None else n_prompt
        n_obs = 0 if q_obs is None else q_obs.shape[2]
        _check(self._lib.buzz_prefill(self._h, _ptr(k), _ptr(v), n_prompt, _ptr(q_obs) if n_obs else None, n_obs,
                                      _ptr(init_score), self._stream(stream)), "buzz_prefill")

    def _step(self, entry, what, q, k_new, v_new, out, stream):
        # A short step takes the GPU 4 us, and the host has to keep up: without the general helpers' calls per argument
        # one step costs it 0.1 to 0.5 us less, by machine (0.70 -> 0.60 us with a stream handle given and nothing launched).
        try:
            q, k_new, v_new, out = q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr()
        except AttributeError:                             # None among them
            q, k_new, v_new, out = _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out)
        rc = entry(self._h, q, k_new, v_new, out, stream if type(stream) is int and not self.dry else self._stream(stream))
        if rc:
            _check(rc, what)

    def decode_step(self, q, k_new, v_new, out, stream=None):
        self._step(self._lib.buzz_decode_step, "buzz_decode_step", q, k_new, v_new, out, stream)

    def decode_step_static(self, q, k_new, v_new, out, stream=None):
        """``decode_step`` with the split-softmax scratch in the library's static device array (allocates nothing)."""
        self._step(self._lib.buzz_decode_step_static, "buzz_decode_step_static", q, k_new, v_new, out, stream)

    def evict(self, stream=None):
        _check(self._lib.buzz_evict(self._h, self._stream(stream)), "buzz_evict")

    def lengths(self):
        n, n_old, nc = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        _check(self._lib.buzz_cache_len(self._h, ctypes.byref(n), ctypes.byref(n_old), ctypes.byref(nc)),
               "buzz_cache_len")
        return n.value, n_old.value, nc.value

    def set_splits(self, n_splits: int):
        _check(self._lib.buzz_cache_set_splits(self._h, n_splits), "buzz_cache_set_splits")

    def override_die_map(self, die_map: int):
        _check(self._lib.buzz_cache_override_die_map(self._h, die_map), "buzz_cache_override_die_map")

    def profile(self, enable: bool):
        _check(self._lib.buzz_cache_profile(self._h, int(enable)), "buzz_cache_profile")

    def profile_read(self) -> dict:
        p = _Profile()
        _check(self._lib.buzz_cache_profile_read(self._h, ctypes.byref(p)), "buzz_cache_profile_read")
        return {k: getattr(p, k) for k, _ in _Profile._fields_}

    def import_rows(self, k, v, score, pos, n_old: int, tokens_seen: int, stream=None, n=None):
        """Load retained rows (as ``export`` returns them) into this cache; ``n`` only for dry-run caches."""
        n = k.shape[2] if n is None else n
        _check(self._lib.buzz_cache_import(self._h, _ptr(k), _ptr(v), _ptr(score), _ptr(pos), n, n_old, tokens_seen,
                                           self._stream(stream)), "buzz_cache_import")

    def export(self, stream=None):
        """Retained rows in cache order: (K, V, score, pos) as new GPU tensors."""
        import torch
        c = self.cfg
        n, _, _ = self.lengths()
        dt = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[c.kv_dtype]
        dev = self.workspace.device
        K = torch.empty(c.batch, c.n_kv_heads, n, c.head_dim, dtype=dt, device=dev)
        V = torch.empty_like(K)
        score = torch.empty(c.batch, c.n_kv_heads, n, dtype=torch.float32, device=dev)
        pos = torch.empty(c.batch, c.n_kv_heads, n, dtype=torch.int32, device=dev)
        _check(self._lib.buzz_cache_export(self._h, _ptr(K), _ptr(V), _ptr(score), _ptr(pos), self._stream(stream)),
               "buzz_cache_export")
        return K, V, score, pos


# ---------------------------------------------------------------------------------------------- paged cache
# A decode step takes the GPU some 5 us, and the host has to keep up: rows go to the C ABI as packed bytes (a ctypes structure
# takes three times as long to make), and tensors are looked at by their cheapest attributes.
_pack_rows = struct.Struct("Pqqq").pack                    # buzz_rows_t
_dtypes = {}


def _dtype(name):
    if not _dtypes:
        import torch
        _dtypes.update(fp32=torch.float32, fp16=torch.float16, bf16=torch.bfloat16, e4m3=torch.float8_e4m3fn, int32=torch.int32)
    return _dtypes[name]


def _wrong(what, t, want):
    raise BuzzError(-1, what, f"got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}; {want}")


def _rows(what, t, dtype, shape, index):
    """Rows ``[batch, heads, n, D]`` or ``[batch, heads, D]`` of GPU ``index`` (-1: the CPU) as the C ABI takes them; None stays None."""
    if t is None:
        return None
    s = t.stride()
    if t.dtype is not dtype or t.shape != shape or s[-1] != 1 or t.get_device() != index:
        _wrong(what, t, f"wanted {tuple(shape)} {dtype} on device {index} with contiguous rows")
    return _pack_rows(t.data_ptr(), s[0], s[1], s[2])


def _dense(what, t, dtype, shape, index):
    """Device pointer of a contiguous tensor; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        _wrong(what, t, f"wanted {tuple(shape)} {dtype} on device {index}, contiguous")
    return t.data_ptr()


def _gpu(what, device):
    """Only tensors on the GPU are handed to kernels."""
    if device.type != "cuda":
        raise BuzzError(-1, what, f"tensors must be on the GPU, not on {device}")


_gpus = 0


def _launch(index, stream, entry, *args):
    """``entry(*args, stream)`` on the given stream or the current one of GPU ``index``, with that GPU current: kernels are
    launched on the current device.  A dry-run cache (-1) launches nothing."""
    global _gpus
    if index < 0:
        return entry(*args, None)
    if type(stream) is not int:
        import torch
        stream = torch.cuda.current_stream(index).cuda_stream if stream is None else stream.cuda_stream
    if _gpus == 1:
        return entry(*args, stream)
    import torch
    _gpus = torch.cuda.device_count()
    with torch.cuda.device(index):
        return entry(*args, stream)


class Rotary:
    """What is done to query and key rows before they are used: a norm per head (weights ``[head_dim]`` in the rows' dtype,
    None: no norm) and the rotation of pairs by position * ``inv_freq`` (``[rot_dim / 2]`` float64, None: no rotation)."""

    def __init__(self, q_weight=None, k_weight=None, inv_freq=None, eps: float = 1e-6, interleaved: bool = False):
        import torch
        for name, t in (("q_weight", q_weight), ("k_weight", k_weight), ("inv_freq", inv_freq)):
            if t is not None and (t.dim() != 1 or not t.is_contiguous() or (t.dtype == torch.float64) != (name == "inv_freq")):
                _wrong("Rotary " + name, t, "wanted a contiguous vector, inv_freq (and only it) in float64")
        self.q_weight, self.k_weight, self.inv_freq = q_weight, k_weight, inv_freq        # kept alive
        self.c = _Rotary(_ptr(q_weight), _ptr(k_weight), _ptr(inv_freq), eps, 0 if inv_freq is None else 2 * inv_freq.numel(),
                         int(interleaved), 0)
        self.ref = ctypes.addressof(self.c)
        weights = [t for t in (q_weight, k_weight) if t is not None]
        if len({(t.dtype, t.shape[0]) for t in weights}) > 1 or len({t.device for t in weights + ([] if inv_freq is None else [inv_freq])}) > 1:
            raise BuzzError(-1, "Rotary", "weights of one length and type, all on one device")
        # what rows must be like: anything where nothing says so
        self.dtype, self.dim = (weights[0].dtype, weights[0].shape[0]) if weights else (None, None)
        self.at = weights[0].get_device() if weights else None if inv_freq is None else inv_freq.get_device()

    def check(self, dtype, head_dim, index):
        if (self.dtype is not dtype and self.dtype is not None) or (self.dim != head_dim and self.dim is not None) or \
                (self.at != index and self.at is not None):
            raise BuzzError(-1, "Rotary", f"made for rows of {self.dim} {self.dtype} on device {self.at}, not {head_dim} {dtype} on {index}")
        return self.ref


def qk_norm_rotate(q, k, q_out, k_out, rotary: Rotary, start=None, count=None, stream=None):
    """Norm and rotation of query rows ``[batch, q heads, n, D]`` to ``q_out`` and key rows likewise to ``k_out`` (either
    pair may be None, outputs may be the inputs).  Row t of sequence b stands at position ``start[b] + t``; ``count[b]`` rows
    are there, the others stay as they were (int32 ``[batch]``; None: 0, all)."""
    some = q if q is not None else k
    if some is None:
        raise BuzzError(-1, "qk_norm_rotate", "neither queries nor keys")
    B, _, n, D = some.shape
    dtype, at, i32 = some.dtype, some.get_device(), _dtype("int32")
    if at < 0:
        _gpu("qk_norm_rotate", some.device)
    code = 2 if dtype is _dtypes["bf16"] else 1 if dtype is _dtypes["fp16"] else 0 if dtype is _dtypes["fp32"] else -1
    if code < 0:
        _wrong("qk_norm_rotate", some, "wanted fp32, fp16 or bf16")
    hq, hk = 0 if q is None else q.shape[1], 0 if k is None else k.shape[1]
    qs, ks = (B, hq, n, D), (B, hk, n, D)
    rc = _launch(at, stream, load_library().buzz_qk_norm_rotate, code, D, hq, hk, rotary.check(dtype, D, at),
                 _rows("qk_norm_rotate q", q, dtype, qs, at), _rows("qk_norm_rotate k", k, dtype, ks, at),
                 _rows("qk_norm_rotate q_out", q_out, dtype, qs, at), _rows("qk_norm_rotate k_out", k_out, dtype, ks, at),
                 B, n, _dense("qk_norm_rotate start", start, i32, (B,), at), _dense("qk_norm_rotate count", count, i32, (B,), at))
    if rc:
        _check(rc, "buzz_qk_norm_rotate")


@dataclass
class PagedConfig:
    batch: int                     # most sequences per call
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    dtype: str                     # "fp32" | "fp16" | "bf16": rows that come and go
    page_rows: int                 # tokens per page: 16, 32, 64, 128 or 256
    n_pages: int
    table_cols: int                # page-table entries per sequence
    page_dtype: str | None = None  # None: dtype; "e4m3": 8 bits (16-bit dtype only)
    sink: int = 0
    window: int = 0                # 0: a new token attends to every token
    softmax_scale: float = 0.0
    flags: int = 0                 # FLAG_DRY_RUN

    def to_c(self) -> _PagedCfg:
        return _PagedCfg(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, DTYPE_CODES[self.dtype],
                         PAGE_DTYPE_CODES[self.page_dtype or self.dtype], self.page_rows, self.n_pages, self.table_cols,
                         self.sink, self.window, self.flags, self.softmax_scale, 0)


def paged_workspace_bytes(cfg: PagedConfig) -> int:
    out = ctypes.c_size_t()
    _check(load_library().buzz_paged_workspace_bytes(cfg.to_c(), ctypes.byref(out)), "buzz_paged_workspace_bytes")
    return out.value


class PagedCache:
    """One layer's paged cache.  ``pages`` = (k, v, k_exp, v_exp) stands over pages that exist already (the layout that
    ``include/buzz.h`` gives); without it they are allocated, uninitialised, and kept as attributes of these names."""

    def __init__(self, cfg: PagedConfig, device="cuda", pages=None, stream=None):
        self.cfg = cfg
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.nbytes = paged_workspace_bytes(cfg)
        self.dry = bool(cfg.flags & FLAG_DRY_RUN)
        self.k_pages = self.v_pages = self.k_exp = self.v_exp = self.workspace = None
        import torch
        self.dtype, self.at = _dtype(cfg.dtype), -1        # the GPU's number; -1: none
        raw, ws = _Pages(), None
        if not self.dry:
            e4m3 = cfg.page_dtype == "e4m3"
            g = 16 // (1 if e4m3 else self.dtype.itemsize)
            k_shape = (cfg.n_pages, cfg.n_kv_heads, cfg.page_rows, cfg.head_dim)
            v_shape = (cfg.n_pages, cfg.n_kv_heads, cfg.page_rows // g, cfg.head_dim, g)
            store = _dtype(cfg.page_dtype or cfg.dtype)
            if pages is None:
                exps = [torch.empty(k_shape[:3], dtype=torch.uint8, device=device) if e4m3 else None for _ in range(2)]
                pages = (torch.empty(k_shape, dtype=store, device=device), torch.empty(v_shape, dtype=store, device=device), *exps)
            _gpu("PagedCache", pages[0].device)
            self.at = pages[0].get_device()
            exps = ("PagedCache exponents", torch.uint8, k_shape[:3])
            wanted = (("PagedCache k", store, k_shape), ("PagedCache v", store, v_shape)) + ((exps, exps) if e4m3 else (None, None))
            if any((t is None) != (want is None) for t, want in zip(pages, wanted)):
                raise BuzzError(-1, "PagedCache", "exponents belong to 8-bit pages and only to them")
            raw = _Pages(*(None if t is None else _dense(want[0], t, want[1], want[2], self.at) for t, want in zip(pages, wanted)))
            self.k_pages, self.v_pages, self.k_exp, self.v_exp = pages
            self.workspace = torch.empty(self.nbytes, dtype=torch.uint8, device=pages[0].device)
            ws = self.workspace.data_ptr()
        c_cfg, entry = cfg.to_c(), self._lib.buzz_paged_create
        _check(_launch(self.at, stream, lambda st: entry(c_cfg, raw, ws, self.nbytes, st, ctypes.byref(self._h))),
               "buzz_paged_create")
        # what every call compares its tensors with
        self._table = cfg.table_cols
        self._heads = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        self._f32, self._i32 = _dtype("fp32"), _dtype("int32")

    def close(self):
        if getattr(self, "_h", None):
            self._lib.buzz_paged_destroy(self._h)
            self._h = None

    __del__ = close

    def append(self, k, v, table, start=None, count=None, q=None, q_out=None, rotary: Rotary | None = None, stream=None):
        """Store rows ``[batch, kv heads, n, D]``: row t of sequence b becomes token ``start[b] + t``, keys after norm and
        rotation.  Queries, if given, go through the same pass to ``q_out``.  ``table``: int32 ``[batch, table_cols]``."""
        hq, h, D = self._heads
        B, _, n, _ = k.shape
        dt, at, i32, kv, qs = self.dtype, self.at, self._i32, (B, h, n, D), (B, hq, n, D)
        rc = _launch(at, stream, self._lib.buzz_paged_append, self._h, None if rotary is None else rotary.check(dt, D, at),
                     _rows("append q", q, dt, qs, at), _rows("append k", k, dt, kv, at), _rows("append v", v, dt, kv, at),
                     _rows("append q_out", q_out, dt, qs, at), B, n, _dense("append table", table, i32, (B, self._table), at),
                     _dense("append start", start, i32, (B,), at), _dense("append count", count, i32, (B,), at))
        if rc:
            _check(rc, "buzz_paged_append")

    def read(self, table, start, count, k, v, stream=None):
        """Tokens ``start[b] ..`` of every sequence back into rows 0 .. ``count[b]`` - 1 of ``k`` and ``v``
        ``[batch, kv heads, n, D]`` (either may be None)."""
        some = k if k is not None else v
        if some is None:
            raise BuzzError(-1, "read", "neither keys nor values")
        _, h, D = self._heads
        B, _, n, _ = some.shape
        dt, at, i32, kv = self.dtype, self.at, self._i32, (B, h, n, D)
        rc = _launch(at, stream, self._lib.buzz_paged_read, self._h, _rows("read k", k, dt, kv, at), _rows("read v", v, dt, kv, at),
                     B, n, _dense("read table", table, i32, (B, self._table), at), _dense("read start", start, i32, (B,), at),
                     _dense("read count", count, i32, (B,), at))
        if rc:
            _check(rc, "buzz_paged_read")

    def decode(self, q, table, length, out, lse=None, stream=None):
        """Attention of one new token per sequence, q ``[batch, q heads, D]``, over tokens 0 .. ``length[b]`` - 1; ``out``
        fp32 like q, ``lse`` fp32 ``[batch, q heads]`` or None."""
        hq, _, D = self._heads
        at, i32, B = self.at, self._i32, q.shape[0]
        shape = (B, hq, D)
        rc = _launch(at, stream, self._lib.buzz_paged_decode, self._h, _rows("decode q", q, self.dtype, shape, at), B,
                     _dense("decode table", table, i32, (B, self._table), at), _dense("decode length", length, i32, (B,), at),
                     _dense("decode out", out, self._f32, shape, at), _dense("decode lse", lse, self._f32, shape[:2], at))
        if rc:
            _check(rc, "buzz_paged_decode")
