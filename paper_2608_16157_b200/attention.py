"""ctypes binding of ``include/ftattn.h`` (argument checks and marshalling only): block tables and slot maps of a serving
step, per-head norm with rotation and cache write, attention over the paged cache.

Every operator runs in the CUDA library on tensors the caller owns; nothing here computes or allocates device memory.
A tensor of the wrong type, shape, layout or device raises :class:`FtMoeError` with ``FT_ERR_INVALID_ARG`` before anything
is launched.  ``stream=None`` is the current torch stream of the handle's device.

    attn = FtAttn(make_config(n_q_heads=32, n_kv_heads=4, head_dim=128, page_tokens=16, n_pages=..., ...))
    attn.slots(new_len, ctx_len, table, free_pages, n_free, max_new, q_start=..., ...)      # once per step
    for layer in layers:
        attn.qk_rope(q, k, v, q_rot, cache[layer], position, slot, cos_sin, w_q=..., w_k=...)
        attn.forward(q_rot, cache[layer], table, out)
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b
from .binding import FT_ERR_CUDA, FT_ERR_INVALID_ARG, FT_ERR_OOM, FtMoeError

FT_ATTN_BF16, FT_ATTN_FP16 = 0, 1
DTYPES = {"bf16": (FT_ATTN_BF16, torch.bfloat16), "fp16": (FT_ATTN_FP16, torch.float16)}

# every symbol include/ftattn.h declares
SYMBOLS = (
    "ft_attn_cache_bytes", "ft_attn_create", "ft_attn_destroy", "ft_attn_slots", "ft_attn_plan", "ft_attn_qk_rope",
    "ft_attn_forward", "ft_attn_sync_status", "ft_attn_debug_inject", "ft_attn_launch_count", "ft_attn_last_cuda_error",
)


class Config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("device", C.c_int32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32), ("n_pages", C.c_int32),
        ("max_requests", C.c_int32), ("max_tokens", C.c_int32), ("max_pages", C.c_int32), ("window", C.c_int32),
    ]


_lib = None


def load():
    """The library of :mod:`binding` with the signatures of ``include/ftattn.h``."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _b.load()
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_size_t, C.c_float
    sig = {
        "ft_attn_cache_bytes": (sz, [C.POINTER(Config)]),
        "ft_attn_create": (i32, [C.POINTER(Config), C.POINTER(vp)]),
        "ft_attn_destroy": (i32, [vp]),
        "ft_attn_slots": (i32, [vp, i32, i32, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "ft_attn_plan": (i32, [vp, i32, i32, i32, vp, vp, vp]),
        "ft_attn_qk_rope": (i32, [vp, i32, vp, i64, vp, i64, vp, i64, vp, vp, f32, vp, i32, i32, i32, vp, vp, vp, i64, vp, vp]),
        "ft_attn_forward": (i32, [vp, vp, i64, vp, vp, i64, vp, i64, vp, f32, vp]),
        "ft_attn_sync_status": (i32, [vp]),
        "ft_attn_debug_inject": (i32, [vp, C.c_uint32, C.c_uint32]),
        "ft_attn_launch_count": (i32, [vp, C.POINTER(C.c_uint64)]),
        "ft_attn_last_cuda_error": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


class FtAttnError(FtMoeError):
    """A call of ``ft_attn_*`` that failed; ``code`` is its status."""

    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        if code in (FT_ERR_CUDA, FT_ERR_OOM):
            detail = load().ft_attn_last_cuda_error().decode()
        RuntimeError.__init__(self, f"{where}: {_b.status_string(code)} ({code})" + (f" [{detail}]" if detail else ""))


def _check(code: int, where: str):
    if code != 0:
        raise FtAttnError(code, where)


def make_config(*, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_requests, max_tokens, max_pages, dtype="bf16",
                window=0, device=0) -> Config:
    return Config(C.sizeof(Config), device, DTYPES[dtype][0], n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages,
                  max_requests, max_tokens, max_pages, window)


def cache_bytes(cfg: Config) -> int:
    """Bytes of one layer's key/value cache; 0 if the configuration is not supported."""
    return int(load().ft_attn_cache_bytes(C.byref(cfg)))


class FtAttn:
    """Handle of the attention operators of one cache geometry.  Methods mirror the C entry points."""

    def __init__(self, cfg: Config):
        self._lib = load()
        self.cfg = cfg
        self._h = C.c_void_p()
        _check(self._lib.ft_attn_create(C.byref(cfg), C.byref(self._h)), "ft_attn_create")
        self._index, self._device = cfg.device, torch.device("cuda", cfg.device)
        self._dtype = torch.bfloat16 if cfg.dtype == FT_ATTN_BF16 else torch.float16
        self._max_pages, self._n_pages, self._hq, self._hkv, self._d = cfg.max_pages, cfg.n_pages, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        self._n_req = self._rows = None
        self._cache_shape = (cfg.n_pages, 2, cfg.n_kv_heads, cfg.page_tokens, cfg.head_dim)

    def destroy(self):
        if self._h is not None and self._h.value:
            h, self._h = self._h, None
            _check(self._lib.ft_attn_destroy(h), "ft_attn_destroy")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # ---- checks ---------------------------------------------------------------------
    def _stream(self, s):
        if s is None:
            return torch._C._cuda_getCurrentRawStream(self._index)     # (torch.cuda.current_stream builds an object: 1 us)
        return s if isinstance(s, int) else s.cuda_stream

    def _vec(self, where, name, t, n, dtype=torch.int32):
        """Address of a contiguous device vector of at least n elements."""
        if t.dtype is not dtype or t.get_device() != self._index or not t.is_contiguous() or t.numel() < n:
            raise FtAttnError(FT_ERR_INVALID_ARG, where, f"{name}: contiguous {dtype} tensor of >= {n} elements on {self._device}")
        return t.data_ptr()

    def _heads(self, where, name, t, rows, heads):
        """(address, row stride) of a [rows, heads, D] tensor whose heads are contiguous."""
        d = self._d
        if t.dtype is not self._dtype or t.get_device() != self._index or t.shape != (rows, heads, d):
            raise FtAttnError(FT_ERR_INVALID_ARG, where, f"{name}: {self._dtype} [{rows}, {heads}, {d}] on {self._device}")
        s = t.stride()
        if s[2] != 1 or (s[1] != d and heads > 1):
            raise FtAttnError(FT_ERR_INVALID_ARG, where, f"{name}: the heads of a token must be contiguous")
        return t.data_ptr(), (s[0] if rows > 1 else heads * d)

    def _cache(self, where, t):
        if t.dtype is not self._dtype or t.get_device() != self._index or t.shape != self._cache_shape or not t.is_contiguous():
            raise FtAttnError(FT_ERR_INVALID_ARG, where, f"kv_cache: contiguous {self._dtype} {list(self._cache_shape)} on {self._device}")
        return t.data_ptr()

    def _table(self, where, t, n_req):
        shape, stride = t.shape, t.stride()
        if (t.dtype is not torch.int32 or t.get_device() != self._index or len(shape) != 2 or shape[0] < n_req or
                shape[1] != self._max_pages or (shape[1] > 1 and stride[1] != 1)):
            raise FtAttnError(FT_ERR_INVALID_ARG, where, f"table: torch.int32 [>= {n_req}, {self._max_pages}] on {self._device}")
        return t.data_ptr(), (stride[0] if shape[0] > 1 else shape[1])

    # ---- the operators --------------------------------------------------------------
    def slots(self, new_len, ctx_len, table, free_pages, n_free, max_new, *, q_start, kv_len, n_free_out, admitted, position, slot,
              stream=None):
        """Block tables and slot maps of a step (``ft_attn_slots``); the step has ``new_len.numel()`` requests and
        ``position.numel()`` packed rows.  Also makes the work partition of :meth:`forward`."""
        w = "ft_attn_slots"
        r, t = new_len.numel(), position.numel()
        tab, stride = self._table(w, table, r)
        v = self._vec
        _check(self._lib.ft_attn_slots(
            self._h, r, t, max_new, v(w, "new_len", new_len, r), v(w, "ctx_len", ctx_len, r), tab, stride,
            v(w, "free_pages", free_pages, self._n_pages), v(w, "n_free", n_free, 1), v(w, "q_start", q_start, r + 1),
            v(w, "kv_len", kv_len, r), v(w, "n_free_out", n_free_out, 1), v(w, "admitted", admitted, r),
            v(w, "position", position, t), v(w, "slot", slot, t), self._stream(stream)), w)
        self._n_req = r
        self._rows = t

    def plan(self, q_start, kv_len, rows, max_new, stream=None):
        """The work partition alone (``ft_attn_plan``), for callers with their own block tables."""
        w = "ft_attn_plan"
        r = kv_len.numel()
        _check(self._lib.ft_attn_plan(self._h, r, rows, max_new, self._vec(w, "q_start", q_start, r + 1),
                                      self._vec(w, "kv_len", kv_len, r), self._stream(stream)), w)
        self._n_req = r
        self._rows = rows

    def qk_rope(self, q, k, v, q_out, kv_cache, position, slot, cos_sin=None, *, w_q=None, w_k=None, eps=1e-6, interleaved=False,
                stream=None):
        """Norm of the query and key heads, rotation, cache write (``ft_attn_qk_rope``).  ``cos_sin`` is float32
        ``[max_pos, rot_dim]`` (cosines, then sines) or None for no rotation; ``w_q`` / ``w_k`` None for no norm."""
        w = "ft_attn_qk_rope"
        t = q.shape[0]
        qp, qs = self._heads(w, "q", q, t, self._hq)
        kp, ks = self._heads(w, "k", k, t, self._hkv)
        vp, vs = self._heads(w, "v", v, t, self._hkv)
        op, os_ = self._heads(w, "q_out", q_out, t, self._hq)
        csp, max_pos, rot = None, 0, 0
        if cos_sin is not None:
            if cos_sin.dim() != 2:
                raise FtAttnError(FT_ERR_INVALID_ARG, w, "cos_sin: [max_pos, rot_dim]")
            max_pos, rot = cos_sin.shape
            csp = self._vec(w, "cos_sin", cos_sin, 1, torch.float32)
        wq = None if w_q is None else self._vec(w, "w_q", w_q, self._d, self._dtype)
        wk = None if w_k is None else self._vec(w, "w_k", w_k, self._d, self._dtype)
        _check(self._lib.ft_attn_qk_rope(self._h, t, qp, qs, kp, ks, vp, vs, wq, wk, eps, csp, max_pos, rot, 1 if interleaved else 0,
                                         self._vec(w, "position", position, t), self._vec(w, "slot", slot, t), op, os_,
                                         self._cache(w, kv_cache), self._stream(stream)), w)

    def forward(self, q, kv_cache, table, out, lse=None, scale=None, stream=None):
        """Causal attention of the planned step's rows over the cache (``ft_attn_forward``); ``scale`` defaults to
        ``head_dim ** -0.5``, ``lse`` is float32 ``[T, n_q_heads]``."""
        w = "ft_attn_forward"
        t = self._rows
        if t is None:
            raise FtAttnError(_b.FT_ERR_STATE, w)
        qp, qs = self._heads(w, "q", q, t, self._hq)
        op, os_ = self._heads(w, "out", out, t, self._hq)
        tab, stride = self._table(w, table, self._n_req)
        lp = None if lse is None else self._vec(w, "lse", lse, t * self._hq, torch.float32)
        _check(self._lib.ft_attn_forward(self._h, qp, qs, self._cache(w, kv_cache), tab, stride, op, os_, lp,
                                         self._d ** -0.5 if scale is None else scale, self._stream(stream)), w)

    def sync_status(self):
        return int(self._lib.ft_attn_sync_status(self._h))

    def debug_inject(self, withhold_mask, wait_polls):
        _check(self._lib.ft_attn_debug_inject(self._h, int(withhold_mask), int(wait_polls)), "ft_attn_debug_inject")

    def launch_count(self):
        n = C.c_uint64()
        _check(self._lib.ft_attn_launch_count(self._h, C.byref(n)), "ft_attn_launch_count")
        return int(n.value)
