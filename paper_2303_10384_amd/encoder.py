"""The operators of an encoder's layers that have no library product, in training and in
streaming service: the root-mean-square norm, rotary positions, the product in 8-bit integers,
and the attention of a chunk of new tokens over a paged cache (C-ABI in
include/rnnt_encoder_mi355x.h, HIP kernels in librnnt_mi355x.so).

    rows, x = rms_norm8(x, w_norm, attended, lens)                     # 8 bits, and the residual
    q, k, v = linear8(rows, w_qkv, dtype=x.dtype).view(B, L, 3, H, D).unbind(2)
    q, k = (rotary(t, freq, cached, lens) for t in (q, k))
    out = cached_attention(q, k, v, k_cache, v_cache, pages, cached, lens, left=256)
    attended = linear8(out.flatten(2), w_out)

rms_norm and rotary are differentiable; the others serve trained weights and have no gradient.
As for the operators of network.py, every tensor of a call is on one GPU, which need not be
the current one, work is queued on that GPU's current stream, and calls may be captured into a
graph.
"""
import ctypes
import functools
import math
from typing import NamedTuple

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from .binding import RNNT_ERR_UNSUPPORTED, RNNTError, _ptr, _result, _workspace_args, dtype_code, load_library
from .network import _call, _check, _dense, _recorded

# every symbol declared in include/rnnt_encoder_mi355x.h
EXPORTED = ("rnnt_rms_norm", "rnnt_rms_norm_grad_workspace_bytes", "rnnt_rms_norm_grad", "rnnt_quantize_rows",
            "rnnt_rms_norm8", "rnnt_linear8", "rnnt_linear8_dynamic_workspace_bytes", "rnnt_linear8_dynamic",
            "rnnt_rotary", "rnnt_cached_attention_workspace_bytes", "rnnt_cached_attention")

_i32, _i64, _vp, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t


class NormShape(ctypes.Structure):
    _fields_ = [("B", _i32), ("L", _i32), ("D", _i32), ("dtype", ctypes.c_int)]


class Linear8Shape(ctypes.Structure):
    _fields_ = [("M", _i32), ("N", _i32), ("K", _i32), ("dtype", ctypes.c_int), ("x_pitch", _i64), ("w_pitch", _i64)]


class RotaryShape(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("B", "L", "H", "D", "R", "interleaved")] + [("dtype", ctypes.c_int)] + [
        (n, _i64) for n in ("stride_b", "stride_t", "stride_h")]


class AttentionShape(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("B", "L", "Hq", "Hkv", "D", "page", "table", "num_pages", "causal", "left")] + [
        ("dtype", ctypes.c_int)] + [("%s_stride_%s" % (t, d), _i64) for t in "qkv" for d in "bth"]


@functools.lru_cache(maxsize=None)
def _library():
    lib = load_library()
    ints, f32 = ctypes.c_int, ctypes.c_float
    n, m, r, a = NormShape, Linear8Shape, RotaryShape, AttentionShape
    for name, res, args in (
            ("rnnt_rms_norm", ints, [_vp, _vp, n, _vp, _vp, f32, _vp, _vp, _vp]),
            ("rnnt_rms_norm_grad_workspace_bytes", _sz, [n]),
            ("rnnt_rms_norm_grad", ints, [_vp, _vp, n, _vp, _vp, f32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
            ("rnnt_quantize_rows", ints, [_vp, _i64, _i32, ints, _vp, _i64, _vp, _vp]),
            ("rnnt_rms_norm8", ints, [_vp, _vp, n, _vp, _vp, f32, _vp, _i64, _vp, _vp, _vp]),
            ("rnnt_linear8", ints, [_vp, _vp, _vp, _vp, m, _vp, _vp, _vp]),
            ("rnnt_linear8_dynamic_workspace_bytes", _sz, [m]),
            ("rnnt_linear8_dynamic", ints, [_vp, _vp, _vp, m, _vp, _vp, _vp, _sz, _vp]),
            ("rnnt_rotary", ints, [_vp, r, _vp, _vp, _vp, _i32, _vp, _vp]),
            ("rnnt_cached_attention_workspace_bytes", _sz, [a]),
            ("rnnt_cached_attention", ints, [_vp, _vp, _vp, a, _vp, _vp, _vp, _vp, _vp, f32, _vp, _vp, _sz, _vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


# A call's descriptor and the bytes of its workspace; a program makes the same few again and again.
@functools.lru_cache(maxsize=1024)
def _shape(kind, size_of, *fields):
    # ctypes would keep the low half of a size past 32 bits
    if any(c_type is _i32 and v > 0x7fffffff for (_, c_type), v in zip(kind._fields_, fields)):
        raise RNNTError(RNNT_ERR_UNSUPPORTED, kind.__name__)
    shape = kind(*fields)
    return shape, getattr(_library(), size_of)(shape) if size_of else 0


# What a call's checks found, by the sizes, strides, types and GPUs of its tensors: a program makes the same few calls again
# and again, and the checks of eight tensors cost as much as a launch.
_plans = {}


def _plan(key, check, *args):
    """check(*args), or what it gave before for tensors alike.  key: what describes them; None, where they are no tensors, is
    not kept."""
    try:
        plan = _plans.get(key)
    except TypeError:
        key = plan = None
    if plan is None:
        plan = check(*args)
        if key is not None:
            if len(_plans) >= 1024:
                _plans.clear()
            _plans[key] = plan
    return plan


def _key(what, *tensors):
    try:
        return (what,) + tuple([None if t is None else (t.shape, t.stride(), t.dtype, t.device) for t in tensors])
    except AttributeError:
        return None


def _no_gradient(what, *tensors):
    """Calls that only serve are refused where a gradient or a tangent would be lost."""
    if not _recorded(*tensors):
        return
    for t in tensors:
        if t is None:
            continue
        if torch.is_grad_enabled() and t.requires_grad:
            raise RuntimeError("%s has no gradient: call it under torch.no_grad() or on detached tensors" % what)
        if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
            raise NotImplementedError("%s has no forward mode" % what)


def _contiguous_channels(t):
    return t.stride(-1) == 1 or t.shape[-1] == 1 or t.numel() == 0


def _strides(t):
    """Strides of all dimensions but the channels; those of a dimension of one element, or of none at all, say nothing."""
    empty = t.numel() == 0
    return (0 if empty or n == 1 else s for n, s in zip(t.shape[:-1], t.stride()))


def _check_lens(lens, x):
    if lens is not None:
        if x.dim() < 3:
            raise ValueError("lens needs x of (B, L, ...)")
        _check("lens", lens, x.device, torch.int32, x.shape[:1])


# ---------------------------------------------------------------- root-mean-square norm

def _norm_checks(x, weight, residual, lens):
    _check("x", x)
    if x.dim() < 1:
        raise ValueError("x must be (..., D)")
    code = dtype_code(x.dtype, "x")
    _check("weight", weight, x.device, x.dtype, x.shape[-1:])
    if residual is not None:
        _check("residual", residual, x.device, x.dtype, x.shape)
    if lens is not None and x.dim() != 3:
        raise ValueError("lens needs x of (B, L, D)")
    _check_lens(lens, x)
    B, L = x.shape[:2] if lens is not None else (1, math.prod(x.shape[:-1]))
    return _shape(NormShape, "rnnt_rms_norm_grad_workspace_bytes", B, L, x.shape[-1], code)


def _norm_args(x, weight, residual, lens, eps):
    eps = float(eps)
    if not 0.0 <= eps < math.inf:
        raise ValueError("eps must be finite and not below 0, got %r" % eps)
    return _plan(_key("norm", x, weight, residual, lens), _norm_checks, x, weight, residual, lens), eps


def _norm_forward(x, weight, residual, lens, eps, shape):
    y = torch.empty_like(x)
    total = None if residual is None else torch.empty_like(x)
    _call(_library().rnnt_rms_norm, x.device, _ptr(x), _ptr(residual), shape, _ptr(lens), _ptr(weight), eps, _ptr(y),
          _ptr(total))
    return y, total


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, lens, eps, shape):
        ctx.set_materialize_grads(False)
        ctx.shape, ctx.eps = shape, eps
        y, total = _norm_forward(x, weight, residual, lens, eps, shape[0])
        ctx.save_for_backward(x, residual, weight, lens)
        return y if total is None else (y, total)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dsum=None):
        x, residual, weight, lens = _dense(*ctx.saved_tensors)
        shape, nbytes = ctx.shape
        dy = torch.zeros_like(x) if dy is None else dy.contiguous()
        dsum = None if dsum is None else dsum.contiguous()
        dx, ws = _result(x.shape, x.dtype, x.device, nbytes)
        dw = torch.empty_like(weight)
        _call(_library().rnnt_rms_norm_grad, x.device, _ptr(x), _ptr(residual), shape, _ptr(lens), _ptr(weight), ctx.eps,
              _ptr(dy), _ptr(dsum), _ptr(dx), _ptr(dw), *_workspace_args(ws))
        return dx, dw, dx if ctx.needs_input_grad[2] else None, None, None, None


def rms_norm(x, weight, residual=None, lens=None, eps=1e-5):
    """t / sqrt(mean(t^2) + eps) * weight over the rows of t = x + residual; with a residual (y, t).

    x (..., D) contiguous, float32/bfloat16/float16; weight (D,) and residual (x's shape) of its
    type; lens (B,) int32 with x (B, L, D): rows behind a length are exactly 0, in t too, and
    their gradients as well.
    """
    shape, eps = _norm_args(x, weight, residual, lens, eps)
    if _recorded(x, weight, residual):
        return _RmsNorm.apply(x, weight, residual, lens, eps, shape)
    y, total = _norm_forward(x, weight, residual, lens, eps, shape[0])
    return y if total is None else (y, total)


# ---------------------------------------------------------------- rows in 8 bits

class Rows8(NamedTuple):
    """Rows in 8-bit integers with one scale a row: the value is values * scale[..., None].

    values (..., K) int8, whose rows begin at multiples of 16 bytes and lie at one pitch (a view
    of padded rows where K is no multiple of 16); scale (...) float32.
    """
    values: torch.Tensor
    scale: torch.Tensor


def _empty_rows8(lead, K, device):
    pitch = -(-K // 16) * 16
    values = torch.empty((*lead, pitch), dtype=torch.int8, device=device)
    return Rows8(values if pitch == K else values[..., :K], torch.empty(lead, dtype=torch.float32, device=device)), pitch


def _check_rows8(name, rows, device=None):
    """The checks of rows in 8 bits; returns their pitch in bytes."""
    if not isinstance(rows, Rows8):
        raise TypeError("%s must be Rows8, got %s" % (name, type(rows).__name__))
    values, scale = rows
    _check(name + ".values", values, device, torch.int8, contiguous=False)
    if values.dim() < 1 or values.shape[-1] < 1:
        raise ValueError("%s.values must be (..., K)" % name)
    _check(name + ".scale", scale, values.device, torch.float32, values.shape[:-1])
    K, pitch, at = values.shape[-1], None, None
    uniform = K == 1 or values.stride(-1) == 1
    for n, stride in zip(reversed(values.shape[:-1]), reversed(values.stride()[:-1])):
        if n == 1:
            continue
        pitch = stride if pitch is None else pitch
        uniform = uniform and (at is None or stride == at)
        at = stride * n
    pitch = -(-K // 16) * 16 if pitch is None else pitch
    if not uniform or pitch < K or pitch % 16 or (values.numel() and values.data_ptr() % 16):
        raise ValueError("%s.values must have rows at one pitch, a multiple of 16 bytes (quantize_rows lays them out)" % name)
    # the last row's last 16 bytes are read whole
    if values.numel() and K % 16:
        last = values.storage_offset() + (scale.numel() - 1) * pitch + -(-K // 16) * 16
        if last > values.untyped_storage().nbytes():
            raise ValueError("%s.values must have whole pieces of 16 bytes behind its last row" % name)
    return pitch


def quantize_rows(x):
    """x (..., K), contiguous, float32/bfloat16/float16, as Rows8: scale = max |row| / 127, values to the nearest
    integer, ties to even.  A row of zeros has scale 0, one with an infinity or NaN scale NaN."""
    _check("x", x)
    if x.dim() < 1:
        raise ValueError("x must be (..., K)")
    code = dtype_code(x.dtype, "x")
    _no_gradient("quantize_rows", x)
    rows, pitch = _empty_rows8(x.shape[:-1], x.shape[-1], x.device)
    if x.shape[-1] > 0x7fffffff:
        raise RNNTError(RNNT_ERR_UNSUPPORTED, "quantize_rows")
    _call(_library().rnnt_quantize_rows, x.device, _ptr(x), rows.scale.numel(), x.shape[-1], code, _ptr(rows.values), pitch,
          _ptr(rows.scale))
    return rows


def rms_norm8(x, weight, residual=None, lens=None, eps=1e-5):
    """rms_norm with its result as Rows8, quantized before it is rounded; with a residual (rows, t).  No gradient."""
    (shape, _), eps = _norm_args(x, weight, residual, lens, eps)
    _no_gradient("rms_norm8", x, weight, residual)
    rows, pitch = _empty_rows8(x.shape[:-1], x.shape[-1], x.device)
    total = None if residual is None else torch.empty_like(x)
    _call(_library().rnnt_rms_norm8, x.device, _ptr(x), _ptr(residual), shape, _ptr(lens), _ptr(weight), eps,
          _ptr(rows.values), pitch, _ptr(rows.scale), _ptr(total))
    return rows if total is None else (rows, total)


def linear8(x, weight, bias=None, dtype=None):
    """x @ weight.T + bias in 8-bit integers, the sums exact: (..., N).

    x (..., K): Rows8, or a contiguous float32/bfloat16/float16 tensor that is taken to 8 bits row
    by row within the call; weight: Rows8 of (N, K), laid out once (quantize_rows of the trained
    weight, a scale for each channel); bias (N,) of the result's type.  dtype: the result's type;
    by default x's, or for Rows8 the bias's, or float32.  No gradient.
    """
    rows = isinstance(x, Rows8)
    key = None
    if isinstance(weight, Rows8):
        values, scale = x if rows else (x, None)
        key = _key((Rows8, rows, dtype), values, scale, *weight, bias)
        # a row's last 16 bytes may lie behind the tensor, which its memory says
        if key is not None and weight.values.dim() and weight.values.shape[-1] % 16:
            key += tuple([(t.storage_offset(), t.untyped_storage().nbytes()) for t in ((values, weight.values) if rows else (weight.values,))])
    (shape, nbytes), dev, out_shape, dtype = _plan(key, _linear8_checks, x, weight, bias, dtype)
    if rows:
        _no_gradient("linear8", x.scale, weight.scale, bias)
    else:
        _no_gradient("linear8", x, weight.scale, bias)
    y, ws = _result(out_shape, dtype, dev, nbytes)
    w, w_scale = weight
    if rows:
        _call(_library().rnnt_linear8, dev, _ptr(x.values), _ptr(x.scale), _ptr(w), _ptr(w_scale), shape, _ptr(bias), _ptr(y))
    else:
        _call(_library().rnnt_linear8_dynamic, dev, _ptr(x), _ptr(w), _ptr(w_scale), shape, _ptr(bias), _ptr(y),
              *_workspace_args(ws))
    return y


def _linear8_checks(x, weight, bias, dtype):
    w_pitch = _check_rows8("weight", weight)
    w = weight.values
    dev = w.device
    if w.dim() != 2:
        raise ValueError("weight must be (N, K)")
    N, K = w.shape
    rows = isinstance(x, Rows8)
    if rows:
        x_pitch, lead, values = _check_rows8("x", x, dev), x.scale.shape, x.values
        if dtype is None:
            dtype = torch.float32 if bias is None else bias.dtype
    else:
        _check("x", x, dev)
        if x.dim() < 1:
            raise ValueError("x must be (..., K)")
        x_pitch, lead, values = 0, x.shape[:-1], x
        if dtype is None:
            dtype = x.dtype
        elif dtype != x.dtype:
            raise TypeError("dtype must be x's, %s, got %s" % (x.dtype, dtype))
    code = dtype_code(dtype, "x")
    if values.shape[-1] != K:
        raise ValueError("x must be (..., %d), got %s" % (K, tuple(values.shape)))
    if bias is not None:
        _check("bias", bias, dev, dtype, w.shape[:1])
    shape = _shape(Linear8Shape, None if rows else "rnnt_linear8_dynamic_workspace_bytes", math.prod(lead), N, K, code,
                   x_pitch, w_pitch)
    return shape, dev, (*lead, N), dtype


# ---------------------------------------------------------------- rotary positions

def rotary_frequencies(dim, base=10000.0, stretch=1.0, trained=None, slow=1.0, fast=32.0, device="cuda"):
    """The angles a position of rotary's dim / 2 pairs, base ** (-2 i / dim): float64 (dim / 2,).

    For contexts `stretch` times the ones trained on, all of them are divided by stretch, or, with
    `trained` (tokens), those that turn at most `slow` times within the trained context; pairs that
    turn `fast` times or more keep their frequency, and between the two it goes over linearly: the
    interpolation by parts of YaRN (Peng et al., ICLR 2024), without its factor on the scores.
    """
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even and at least 2, got %r" % (dim,))
    if not (base > 0 and stretch > 0 and fast > slow):
        raise ValueError("base and stretch must be above 0 and fast above slow")
    freq = float(base) ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    if trained is None:
        freq = freq / stretch
    else:
        keep = ((freq * (trained / (2 * math.pi)) - slow) / (fast - slow)).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / stretch)
    return freq.to(device)


def _rotary_call(x, freq, start, lens, interleaved, inverse):
    B, L, H, D = x.shape
    shape, _ = _shape(RotaryShape, None, B, L, H, D, 2 * freq.numel(), int(interleaved), dtype_code(x.dtype, "x"),
                      *_strides(x))
    y = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _call(_library().rnnt_rotary, x.device, _ptr(x), shape, _ptr(freq), _ptr(start), _ptr(lens), inverse, _ptr(y))
    return y


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, freq, start, lens, interleaved):
        ctx.interleaved = interleaved
        ctx.save_for_backward(freq, start, lens)
        return _rotary_call(x, freq, start, lens, interleaved, 0)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        if not _contiguous_channels(dy):
            dy = dy.contiguous()
        return _rotary_call(dy, *_dense(*ctx.saved_tensors), ctx.interleaved, 1), None, None, None, None


def rotary(x, freq, start=None, lens=None, interleaved=False):
    """x (B, L, H, D) with the first 2 len(freq) channels of every head turned in pairs by the angles
    (start[b] + t) * freq: channels (2i, 2i + 1) interleaved, else (i, len(freq) + i).

    x float32/bfloat16/float16 with contiguous channels (views such as a part of one projection are
    taken as they are); freq float64, of rotary_frequencies; start (B,) int32 positions of the
    first tokens, or None (0); lens (B,) int32: rows behind a length are exactly 0.  Angles are
    formed in float64.
    """
    _plan(_key("rotary", x, freq, start, lens), _rotary_checks, x, freq, start, lens)
    if freq.requires_grad:
        raise ValueError("freq has no gradient")
    if _recorded(x):
        return _Rotary.apply(x, freq, start, lens, bool(interleaved))
    return _rotary_call(x, freq, start, lens, interleaved, 0)


def _rotary_checks(x, freq, start, lens):
    _check("x", x, contiguous=False)
    if x.dim() != 4:
        raise ValueError("x must be (B, L, H, D)")
    dtype_code(x.dtype, "x")
    if not _contiguous_channels(x):
        raise ValueError("x must have contiguous channels")
    _check("freq", freq, x.device, torch.float64)
    if freq.dim() != 1 or not 1 <= freq.numel() <= x.shape[3] // 2:
        raise ValueError("freq must hold at most half as many values as a head has channels, and one at least")
    if start is not None:
        _check("start", start, x.device, torch.int32, x.shape[:1])
    _check_lens(lens, x)
    return True


# ---------------------------------------------------------------- attention over a paged cache

def cached_attention(q, k, v, k_cache, v_cache, pages, cached, lens=None, scale=None, causal=True, left=None):
    """Writes a chunk's keys and values into the cache and attends from its queries: (B, L, Hq, D).

    q (B, L, Hq, D), k and v (B, L, Hkv, D), float32/bfloat16/float16, views with contiguous
    channels, Hq a multiple of Hkv; k_cache, v_cache (pages, Hkv, page, D) of the same type,
    contiguous, page a power of two; pages (B, table) int32: position j of utterance b lies on page
    pages[b, j // page]; cached (B,) int32 tokens that are in the cache before the call, and lens
    (B,) int32 the new ones, or None (all L).  The caller then adds lens to cached.

    A query sees the tokens up to its own (causal), or all of them, the chunk's too (else), and
    with left none that lies more than left before it; entries of pages that nothing sees are not
    used.  scale: of the scores, D ** -0.5 by default.  Rows behind lens are exactly 0.  A page that
    a call writes to belongs to one utterance.  No gradient.
    """
    if left is not None and left < 0:
        raise ValueError("left must be None or at least 0, got %r" % (left,))
    causal, left = bool(causal), -1 if left is None else int(left)
    key = _key((causal, left), q, k, v, k_cache, v_cache, pages, cached, lens)
    shape, nbytes = _plan(key, _attention_checks, q, k, v, k_cache, v_cache, pages, cached, lens, causal, left)
    _no_gradient("cached_attention", q, k, v, k_cache, v_cache)
    scale = max(shape.D, 1) ** -0.5 if scale is None else float(scale)
    if nbytes or not q.is_contiguous():
        out, ws = _result(q.shape, q.dtype, q.device, nbytes)
    else:
        out, ws = torch.empty_like(q), None
    _call(_library().rnnt_cached_attention, q.device, _ptr(q), _ptr(k), _ptr(v), shape, _ptr(lens), _ptr(cached), _ptr(pages),
          _ptr(k_cache), _ptr(v_cache), scale, _ptr(out), *_workspace_args(ws))
    # autograd then refuses what it saved of the caches before the call, as after any write in place
    increment_version((k_cache, v_cache))
    return out


def _attention_checks(q, k, v, k_cache, v_cache, pages, cached, lens, causal, left):
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(name, t, q.device if isinstance(q, torch.Tensor) else None, q.dtype if isinstance(q, torch.Tensor) else None,
               contiguous=False)
        if t.dim() != 4:
            raise ValueError("%s must be (B, L, heads, D)" % name)
        if not _contiguous_channels(t):
            raise ValueError("%s must have contiguous channels" % name)
    dev, code = q.device, dtype_code(q.dtype, "q")
    B, L, Hq, D = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, L, Hkv, D) or v.shape != k.shape or not Hkv or Hq % Hkv:
        raise ValueError("k and v must be (B, L, Hkv, D) with q's B, L and D, and Hkv a divisor of its heads")
    _check("k_cache", k_cache, dev, q.dtype)
    if k_cache.dim() != 4 or k_cache.shape[1] != Hkv or k_cache.shape[3] != D:
        raise ValueError("k_cache must be (pages, Hkv, page, D) with k's Hkv and D")
    _check("v_cache", v_cache, dev, q.dtype, k_cache.shape)
    _check("pages", pages, dev, torch.int32)
    if pages.dim() != 2 or pages.shape[0] != B:
        raise ValueError("pages must be (B, table)")
    _check("cached", cached, dev, torch.int32, (B,))
    if lens is not None:
        _check("lens", lens, dev, torch.int32, (B,))
    return _shape(AttentionShape, "rnnt_cached_attention_workspace_bytes", B, L, Hq, Hkv, D, k_cache.shape[2],
                  pages.shape[1], k_cache.shape[0], int(causal), min(left, 0x7fffffff), code, *_strides(q), *_strides(k),
                  *_strides(v))
