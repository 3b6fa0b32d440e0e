"""ctypes binding of ``include/ftdense.h`` (argument checks and marshalling only): residual and norm between two blocks, products with
4-bit weights, log probabilities from logits.

Every operator runs in the CUDA library on tensors the caller owns.  A tensor of the wrong type, shape, layout or device raises
:class:`FtDenseError` with ``FT_ERR_INVALID_ARG`` before anything is launched.  ``stream=None`` is the current torch stream of the
handle's device.

    dense = FtDense()
    w = dense.w4_pack(codes, scales)                                        # once, when the weights are loaded
    dense.add_norm(y, res, res, x, w_pre=norm_weight)                       # res += y; x = norm(res)
    dense.w4(x, w, logits)
    dense.logprobs(logits, tokens=tokens, logprob=logprob, top_ids=ids, top_logprobs=top)
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b
from .binding import FT_ERR_CUDA, FT_ERR_INVALID_ARG, FT_ERR_OOM, FT_ERR_UNSUPPORTED, FtMoeError

FT_DENSE_BF16, FT_DENSE_FP16, FT_DENSE_FP32 = 0, 1, 2
FT_DENSE_NORM_POST = 1
_CODE = {torch.bfloat16: FT_DENSE_BF16, torch.float16: FT_DENSE_FP16, torch.float32: FT_DENSE_FP32}

# every symbol include/ftdense.h declares
SYMBOLS = (
    "ft_dense_create", "ft_dense_destroy", "ft_dense_add_norm", "ft_dense_w4_bytes", "ft_dense_w4_pack", "ft_dense_w4_forward",
    "ft_dense_logprobs", "ft_dense_sync_status", "ft_dense_debug_inject", "ft_dense_launch_count", "ft_dense_last_cuda_error",
)

_lib = None


def load():
    """The library of :mod:`binding` with the signatures of ``include/ftdense.h``."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _b.load()
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_size_t, C.c_float
    sig = {
        "ft_dense_create": (i32, [i32, C.POINTER(vp)]),
        "ft_dense_destroy": (i32, [vp]),
        "ft_dense_add_norm": (i32, [vp, i32, i32, i32, i32, i32, vp, i64, vp, i64, vp, i64, i32, vp, vp, f32, f32, f32, f32, vp, i64, vp, i64, vp]),
        "ft_dense_w4_bytes": (sz, [i64, i64, i32, i32]),
        "ft_dense_w4_pack": (i32, [vp, i64, i64, i32, i32, vp, i64, vp, vp, vp, vp]),
        "ft_dense_w4_forward": (i32, [vp, i32, i64, i64, i32, i32, i32, vp, i64, vp, vp, vp, i64, i32, vp]),
        "ft_dense_logprobs": (i32, [vp, i32, i64, i32, vp, i64, f32, vp, i64, i32, vp, vp, i32, vp, vp, vp]),
        "ft_dense_sync_status": (i32, [vp]),
        "ft_dense_debug_inject": (i32, [vp, C.c_uint32, C.c_uint32]),
        "ft_dense_launch_count": (i32, [vp, C.POINTER(C.c_uint64)]),
        "ft_dense_last_cuda_error": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


class FtDenseError(FtMoeError):
    """A call of ``ft_dense_*`` that failed; ``code`` is its status."""

    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        if code in (FT_ERR_CUDA, FT_ERR_OOM):
            detail = load().ft_dense_last_cuda_error().decode()
        RuntimeError.__init__(self, f"{where}: {_b.status_string(code)} ({code})" + (f" [{detail}]" if detail else ""))


def _check(code: int, where: str):
    if code != 0:
        raise FtDenseError(code, where)


def w4_bytes(n: int, k: int, group: int, zeros: bool = False) -> int:
    """Bytes of the image of an [n, k] matrix; 0 if the shape is not supported."""
    return int(load().ft_dense_w4_bytes(n, k, group, 1 if zeros else 0))


class W4Weight:
    """A matrix in the layout of ``ft_dense_w4_pack``: its image and what the image was made of."""
    __slots__ = ("image", "n", "k", "group", "dtype", "zeros")

    def __init__(self, image, n, k, group, dtype, zeros):
        self.image, self.n, self.k, self.group, self.dtype, self.zeros = image, n, k, group, dtype, zeros


def _device_index(device):
    """Index of a device; None and a CUDA device without an index are the current one."""
    if isinstance(device, int):
        return device
    index = None
    if device is not None:
        device = torch.device(device)
        if device.type != "cuda":
            raise FtDenseError(FT_ERR_INVALID_ARG, "ft_dense_create", f"{device} is no CUDA device")
        index = device.index
    return torch.cuda.current_device() if index is None else index


class FtDense:
    """Handle of the operators on one device (the current one if none, or none by number, is given).  Methods mirror the C entry points."""

    def __init__(self, device=None):
        self._lib = load()
        self._h = C.c_void_p()
        index = _device_index(device)
        _check(self._lib.ft_dense_create(index, C.byref(self._h)), "ft_dense_create")
        self._index, self._device = index, torch.device("cuda", index)

    def destroy(self):
        if self._h is not None and self._h.value:
            h, self._h = self._h, None
            _check(self._lib.ft_dense_destroy(h), "ft_dense_destroy")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # ---- checks ---------------------------------------------------------------------
    def _stream(self, s):
        if s is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        return s if isinstance(s, int) else s.cuda_stream

    def _fail(self, where, text):
        raise FtDenseError(FT_ERR_INVALID_ARG, where, f"{text} on {self._device}")

    def _rows(self, where, name, t, rows, cols, dtype):
        """(address, row stride) of a [rows, cols] tensor with contiguous rows; None is NULL."""
        if t is None:
            return None, 0
        if t.dtype is dtype and t.get_device() == self._index and t.shape == (rows, cols):
            if t.is_contiguous():
                return t.data_ptr(), cols
            stride, step = t.stride()
            if cols == 1 or step == 1:
                return t.data_ptr(), (stride if rows > 1 else cols)
        self._fail(where, f"{name}: {dtype} [{rows}, {cols}], contiguous rows,")

    def _vec(self, where, name, t, n, dtype):
        """Address of a contiguous vector of n elements; None is NULL."""
        if t is None:
            return None
        if t.dtype is not dtype or t.get_device() != self._index or t.numel() != n or not t.is_contiguous():
            self._fail(where, f"{name}: contiguous {dtype} tensor of {n} elements")
        return t.data_ptr()

    # ---- the operators --------------------------------------------------------------
    def add_norm(self, y, res, res_out, out, *, post=False, w_post=None, w_pre=None, gate=None, w_offset=0.0, eps=1e-6, res_scale=1.0,
                 y_scale=1.0, stream=None):
        """``res_out = res_scale * res + y_scale * gate * u`` with ``u = y`` or, with ``post``, its norm; ``out`` = the norm of that
        (``ft_dense_add_norm``).  y, out ``[T, d]`` bf16 or fp16, res, res_out the same or float32; gate ``[T or 1, d or 1]``; any of y, res,
        gate, res_out, out may be None.  res_out may be res, out may be y."""
        w = "ft_dense_add_norm"
        one = y if y is not None else out if out is not None else w_pre
        stream_t = res if res is not None else res_out
        if one is None:
            one = stream_t
        first = y if y is not None else stream_t if stream_t is not None else out
        if first is None or first.dim() != 2:
            self._fail(w, "y, res: [T, d]")
        shape = first.shape
        t, d = shape
        dt = torch.bfloat16 if one is stream_t and one.dtype is torch.float32 else one.dtype       # (no tensor of the 16-bit type: any)
        rt = stream_t.dtype if stream_t is not None else dt
        if dt not in _CODE or rt not in _CODE:
            self._fail(w, "y, out: bfloat16 or float16; res: the same or float32")
        yp, ys = self._rows(w, "y", y, t, d, dt)
        rp, rs = self._rows(w, "res", res, t, d, rt)
        rop, ros = self._rows(w, "res_out", res_out, t, d, rt)
        op, os_ = self._rows(w, "out", out, t, d, dt)
        gp, gs, step = None, 0, 0
        if gate is not None:
            gsh = gate.shape
            if gate.dtype is not dt or gate.get_device() != self._index or len(gsh) != 2 or gsh[0] not in (1, t) or gsh[1] not in (1, d):
                self._fail(w, f"gate: {dt} [{t} or 1, {d} or 1]")
            gst = gate.stride()
            step = 1 if gsh[1] > 1 else 0
            if step and gst[1] not in (0, 1):
                self._fail(w, "gate: contiguous rows")
            step = gst[1] if step else 0
            gp, gs = gate.data_ptr(), (gst[0] if gsh[0] > 1 else 0)
        _check(self._lib.ft_dense_add_norm(self._h, t, d, _CODE[dt], _CODE[rt], FT_DENSE_NORM_POST if post else 0, yp, ys, rp, rs, gp, gs, step,
                                           self._vec(w, "w_post", w_post, d, dt), self._vec(w, "w_pre", w_pre, d, dt), w_offset, eps, res_scale,
                                           y_scale, rop, ros, op, os_, self._stream(stream)), w)

    def w4_pack(self, codes, scales, zeros=None, image=None, stream=None) -> W4Weight:
        """Lays a matrix out once (``ft_dense_w4_pack``): codes uint8 ``[n, k / 2]`` (the even k in the low half of a byte), scales bf16 or fp16
        ``[n, k / group]``, zeros uint8 of the same shape or None (8).  ``image``: uint8 tensor of :func:`w4_bytes` elements to
        write to, or None: one is made on the current stream, whose work so far another ``stream`` then waits for."""
        w = "ft_dense_w4_pack"
        if codes.dim() != 2 or scales.dim() != 2 or scales.shape[0] != codes.shape[0] or scales.shape[1] < 1 or scales.dtype not in (torch.bfloat16, torch.float16):
            self._fail(w, "codes: uint8 [n, k / 2], scales: bfloat16 or float16 [n, k / group]")
        n, k = codes.shape[0], 2 * codes.shape[1]
        group = k // scales.shape[1]
        size = w4_bytes(n, k, group, zeros is not None) if group * scales.shape[1] == k else 0
        if size == 0:
            raise FtDenseError(FT_ERR_UNSUPPORTED, w, f"{n} x {k} in groups of {group}")
        cp, cs = self._rows(w, "codes", codes, n, k // 2, torch.uint8)
        if zeros is not None and zeros.shape != scales.shape:
            self._fail(w, f"zeros: uint8 {list(scales.shape)}")
        if image is None:
            image = torch.empty(size, dtype=torch.uint8, device=self._device)
            if stream is not None:
                # the memory may have been another tensor's, which work queued on the current stream still uses
                at, own = torch.cuda.current_stream(self._device), self._stream(stream)
                if own != at.cuda_stream:
                    own = torch.cuda.ExternalStream(own, device=self._device)
                    own.wait_stream(at)
                    image.record_stream(own)
        elif image.dtype is not torch.uint8 or image.get_device() != self._index or not image.is_contiguous() or image.numel() < size:
            self._fail(w, f"image: contiguous uint8 tensor of >= {size} elements")
        _check(self._lib.ft_dense_w4_pack(self._h, n, k, group, _CODE[scales.dtype], cp, cs, self._vec(w, "scales", scales, scales.numel(), scales.dtype),
                                          self._vec(w, "zeros", zeros, scales.numel(), torch.uint8), image.data_ptr(), self._stream(stream)), w)
        return W4Weight(image, n, k, group, scales.dtype, zeros is not None)

    def w4(self, x, weight: W4Weight, y, bias=None, stream=None):
        """``y = x @ w.T + bias`` with 4-bit weights (``ft_dense_w4_forward``): x ``[T, k]`` of the scales' type, y ``[T, n]`` of it or float32."""
        w = "ft_dense_w4_forward"
        if x.dim() != 2:
            self._fail(w, f"x: {weight.dtype} [T, {weight.k}]")
        t, n, k, dt = x.shape[0], weight.n, weight.k, weight.dtype
        out_dt = y.dtype
        if out_dt is not dt and out_dt is not torch.float32:
            self._fail(w, f"y: {dt} or float32")
        xp, xs = self._rows(w, "x", x, t, k, dt)
        yp, ys = self._rows(w, "y", y, t, n, out_dt)
        if weight.image.get_device() != self._index:
            self._fail(w, "weight: an image")
        _check(self._lib.ft_dense_w4_forward(self._h, t, n, k, weight.group, _CODE[dt], 1 if weight.zeros else 0, xp, xs, weight.image.data_ptr(),
                                             self._vec(w, "bias", bias, n, dt), yp, ys, _CODE[out_dt], self._stream(stream)), w)

    def logprobs(self, logits, *, tokens=None, logprob=None, entropy=None, top_ids=None, top_logprobs=None, scale=1.0, stream=None):
        """Log probabilities of ``scale * logits`` (``ft_dense_logprobs``): logits ``[T, vocab]`` bf16, fp16 or float32; tokens int32 ``[T, n]`` with
        logprob float32 ``[T, n]``; entropy float32 ``[T]``; top_ids int32 with top_logprobs float32 ``[T, k]``, k <= 32."""
        w = "ft_dense_logprobs"
        if logits.dim() != 2 or logits.dtype not in _CODE:
            self._fail(w, "logits: bfloat16, float16 or float32 [T, vocab]")
        t, v = logits.shape
        lp, ls = self._rows(w, "logits", logits, t, v, logits.dtype)
        n = k = ts = 0
        tp = pp = ip = vp = None
        if tokens is not None:
            if tokens.dim() != 2 or logprob is None:
                self._fail(w, "tokens: int32 [T, n], with logprob")
            n = tokens.shape[1]
            tp, ts = self._rows(w, "tokens", tokens, t, n, torch.int32)
            pp = self._vec(w, "logprob", logprob, t * n, torch.float32)
        if top_ids is not None or top_logprobs is not None:
            if top_ids is None or top_logprobs is None or top_ids.dim() != 2 or top_ids.shape[0] != t or top_logprobs.shape != top_ids.shape:
                self._fail(w, "top_ids: int32 [T, k], with top_logprobs")
            k = top_ids.shape[1]
            ip = self._vec(w, "top_ids", top_ids, t * k, torch.int32)
            vp = self._vec(w, "top_logprobs", top_logprobs, t * k, torch.float32)
        ep = self._vec(w, "entropy", entropy, t, torch.float32)
        _check(self._lib.ft_dense_logprobs(self._h, t, v, _CODE[logits.dtype], lp, ls, scale, tp, ts, n, pp, ep, k, ip, vp, self._stream(stream)), w)

    def sync_status(self):
        return int(self._lib.ft_dense_sync_status(self._h))

    def debug_inject(self, withhold_mask, wait_polls):
        _check(self._lib.ft_dense_debug_inject(self._h, int(withhold_mask), int(wait_polls)), "ft_dense_debug_inject")

    def launch_count(self):
        n = C.c_uint64()
        _check(self._lib.ft_dense_launch_count(self._h, C.byref(n)), "ft_dense_launch_count")
        return int(n.value)
