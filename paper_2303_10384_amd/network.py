"""The operators between an encoder and the transducer loss, differentiable: the label
embedding and the gated recurrence of a prediction network, dropout, and the joint's hidden
layer (C-ABI in include/rnnt_network_mi355x.h, HIP kernels in librnnt_mi355x.so).

    emb = label_embedding(labels, weight, label_lens, scale=..., start=blank)    # (B, U+1, D)
    pred, state = gated_recurrence(emb @ w_x, emb @ w_z, lens=label_lens + 1)    # (B, U+1, H)
    hidden = joint_hidden(enc, pred, logit_lens, label_lens, "tanh", p, rng)     # (B, T, U+1, H)
    loss = rnnt_loss_autograd(hidden @ w_out, labels, logit_lens, label_lens)

A streaming decoder takes the same calls one step at a time: labels (B, 1), x and z (B, 1, H)
with h0 the state before, enc (B, 1, H) against pred (B, 1, H).

Every tensor of a call is on one GPU, which need not be the current one; work is queued on
that GPU's current stream.  A gradient of a gradient and forward mode are not offered.  Calls
may be captured into a graph, backward passes too (as with any operation, while no eager graph
of the same leaves is alive).
"""
import ctypes
import functools

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from .binding import (RNNT_ERR_UNSUPPORTED, RNNT_OK, RNNTError, _ptr, _result, _stream_handle, _workspace_args, dtype_code,
                      load_library)

ACTIVATIONS = {"relu": 0, "tanh": 1}
STATE_STEPS = 8  # RNNT_RECURRENCE_STATE_STEPS

# every symbol declared in include/rnnt_network_mi355x.h
EXPORTED = ("rnnt_label_embedding", "rnnt_label_embedding_grad_workspace_bytes", "rnnt_label_embedding_grad",
            "rnnt_recurrence_states_bytes", "rnnt_recurrence_workspace_bytes", "rnnt_recurrence", "rnnt_recurrence_grad",
            "rnnt_dropout", "rnnt_joint_hidden", "rnnt_joint_hidden_grad_workspace_bytes", "rnnt_joint_hidden_grad")

_i32, _i64, _vp, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t


class EmbeddingShape(ctypes.Structure):
    _fields_ = [("B", _i32), ("N", _i32), ("V", _i32), ("D", _i32), ("start", _i32), ("dtype", ctypes.c_int)]


class RecurrenceShape(ctypes.Structure):
    _fields_ = [("B", _i32), ("L", _i32), ("D", _i32), ("dtype", ctypes.c_int), ("x_stride_b", _i64),
                ("x_stride_t", _i64), ("z_stride_b", _i64), ("z_stride_t", _i64)]


class JointShape(ctypes.Structure):
    _fields_ = [("B", _i32), ("T_max", _i32), ("U_max", _i32), ("H", _i32), ("dtype", ctypes.c_int)]


@functools.lru_cache(maxsize=None)
def _library():
    lib = load_library()
    e, r, j = EmbeddingShape, RecurrenceShape, JointShape
    ints, f32, f64 = ctypes.c_int, ctypes.c_float, ctypes.c_double
    for name, res, args in (
            ("rnnt_label_embedding", ints, [_vp, _vp, e, _vp, f32, _vp, _vp]),
            ("rnnt_label_embedding_grad_workspace_bytes", _sz, [e]),
            ("rnnt_label_embedding_grad", ints, [_vp, _vp, e, _vp, f32, _vp, _vp, _sz, _vp]),
            ("rnnt_recurrence_states_bytes", _sz, [r]),
            ("rnnt_recurrence_workspace_bytes", _sz, [r]),
            ("rnnt_recurrence", ints, [_vp, _vp, r, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
            ("rnnt_recurrence_grad", ints, [_vp, _vp, r, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
            ("rnnt_dropout", ints, [_vp, _i64, ints, f64, _vp, _vp, _vp, _vp]),
            ("rnnt_joint_hidden", ints, [_vp, _vp, j, _vp, _vp, ints, f64, _vp, _vp, _vp, _vp]),
            ("rnnt_joint_hidden_grad_workspace_bytes", _sz, [j]),
            ("rnnt_joint_hidden_grad", ints, [_vp, _vp, j, _vp, _vp, ints, f64, _vp, _vp, _vp, _vp, _vp, _sz, _vp])):
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
    return shape, getattr(_library(), size_of)(shape)


def _call(fn, device, *args):
    """fn(*args, stream) with the tensors' GPU current; its status as an RNNTError."""
    if device.index == torch._C._cuda_getDevice():
        st = fn(*args, _stream_handle(device))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream_handle(device))
    if st != RNNT_OK:
        raise RNNTError(st, fn.__name__)


def _check(name, t, device=None, dtype=None, shape=None, contiguous=True):
    """The checks every call makes on a tensor."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor, got %s" % (name, type(t).__name__))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor (no CPU path exists)" % name)
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s, got %s" % (name, device, t.device))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if contiguous and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _check_p(p):
    p = float(p)
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be in [0, 1), got %r" % p)
    return p


def _recorded(*tensors):
    """Whether a call goes through autograd: for a gradient, and wherever a tensor could carry a tangent, which
    autograd refuses (the operators have no forward mode)."""
    if forward_ad._current_level >= 0:
        return True
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _dense(*saved):
    """Saved tensors as the kernels take them: hooks on saved tensors may give any layout back."""
    return (None if t is None else t.contiguous() for t in saved)


def _check_gradient(shape_and_bytes, *sizes):
    """A step whose gradient would be refused, for which its workspace's size is 0, is refused before it starts (an
    empty tensor is left to the forward call's own error)."""
    shape, nbytes = shape_and_bytes
    if not nbytes and 0 not in sizes:
        raise RNNTError(RNNT_ERR_UNSUPPORTED, "gradient of %s" % type(shape).__name__)


# ---------------------------------------------------------------- label embedding

def _embedding_forward(labels, weight, lens, scale, start, for_gradient=False):
    B, N = labels.shape
    V, D = weight.shape
    shape = _shape(EmbeddingShape, "rnnt_label_embedding_grad_workspace_bytes", B, N, V, D, start, dtype_code(weight.dtype))
    if for_gradient:
        _check_gradient(shape, B, V, D)
    out = torch.empty((B, N + (start >= 0), D), dtype=weight.dtype, device=weight.device)
    _call(_library().rnnt_label_embedding, weight.device, _ptr(labels), _ptr(lens), shape[0], _ptr(weight), scale,
          _ptr(out))
    return out, shape


class _LabelEmbedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, labels, weight, lens, scale, start):
        out, ctx.shape = _embedding_forward(labels, weight, lens, scale, start, ctx.needs_input_grad[1])
        ctx.scale = scale
        ctx.save_for_backward(labels, lens)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        labels, lens = _dense(*ctx.saved_tensors)
        (shape, nbytes), dout = ctx.shape, dout.contiguous()
        dw, ws = _result((shape.V, shape.D), dout.dtype, dout.device, nbytes)
        _call(_library().rnnt_label_embedding_grad, dout.device, _ptr(labels), _ptr(lens), shape, _ptr(dout), ctx.scale,
              _ptr(dw), *_workspace_args(ws))
        return None, dw, None, None, None


def label_embedding(labels, weight, lens=None, scale=1.0, start=None):
    """scale * weight[labels], rows behind lens exactly 0: (B, N, D), or (B, N + 1, D) with start.

    labels (B, N) int32; weight (V, D) float32/bfloat16/float16; lens (B,) int32 labels of each
    utterance, or None (all N); start: None, or the weight row put before every utterance (the
    prediction network's input before the first unit), whose gradient it also takes.  A label
    outside [0, V) gives a row of NaN and no gradient.
    """
    _check("weight", weight)
    _check("labels", labels, weight.device, torch.int32)
    if labels.dim() != 2 or weight.dim() != 2:
        raise ValueError("labels must be (B, N) and weight (V, D)")
    if lens is not None:
        _check("lens", lens, weight.device, torch.int32, labels.shape[:1])
    dtype_code(weight.dtype, "weight")
    if start is not None and not 0 <= start < weight.shape[0]:
        raise ValueError("start must be None or a row of weight, got %r" % (start,))
    args = (labels, weight, lens, float(scale), -1 if start is None else int(start))
    if _recorded(weight):
        return _LabelEmbedding.apply(*args)
    return _embedding_forward(*args)[0]


# ---------------------------------------------------------------- gated recurrence

def _contiguous_channels(t):
    return t.stride(2) == 1 or t.shape[2] == 1 or t.numel() == 0


def _recurrence_shape(x, z):
    return _shape(RecurrenceShape, "rnnt_recurrence_workspace_bytes", *x.shape, dtype_code(x.dtype), *x.stride()[:2],
                  *z.stride()[:2])


def _recurrence_forward(x, z, h0, lens, with_states):
    B, L, D = x.shape
    dev = x.device
    shape, nbytes = _recurrence_shape(x, z)
    h, ws = _result((B, L, D), x.dtype, dev, nbytes)
    last = torch.empty((B, D), dtype=torch.float32, device=dev)
    states = torch.empty((B, -(-L // STATE_STEPS), D), dtype=torch.float32, device=dev) if with_states else None
    _call(_library().rnnt_recurrence, dev, _ptr(x), _ptr(z), shape, _ptr(lens), _ptr(h0), _ptr(h), _ptr(last), _ptr(states),
          *_workspace_args(ws))
    return h, last, states


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, z, h0, lens):
        ctx.set_materialize_grads(False)
        h, last, states = _recurrence_forward(x, z, h0, lens, True)
        ctx.save_for_backward(x, z, lens, states)
        return h, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dlast):
        x, z, lens, states = ctx.saved_tensors
        # hooks on saved tensors may have laid x and z out anew: their strides are taken from what came back
        x, z = (t if _contiguous_channels(t) else t.contiguous() for t in (x, z))
        (shape, nbytes), dev = _recurrence_shape(x, z), x.device
        lens, states = _dense(lens, states)
        dh = None if dh is None else dh.contiguous()
        dlast = None if dlast is None else dlast.contiguous()
        dx, ws = _result(x.shape, x.dtype, dev, nbytes)
        dz = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dh0 = torch.empty((shape.B, shape.D), dtype=torch.float32, device=dev) if ctx.needs_input_grad[2] else None
        _call(_library().rnnt_recurrence_grad, dev, _ptr(x), _ptr(z), shape, _ptr(lens), _ptr(states), _ptr(dh), _ptr(dlast),
              _ptr(dx), _ptr(dz), _ptr(dh0), *_workspace_args(ws))
        return dx, dz, dh0, None


def gated_recurrence(x, z, h0=None, lens=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(z_t), channel by channel.

    x, z (B, L, D) float32/bfloat16/float16 with contiguous channels (views such as the halves
    of one projection are taken as they are); h0 (B, D) float32 the state before, or None
    (zero); lens (B,) int32 steps of each sequence, or None (all L).  Returns h (B, L, D) in
    x's dtype, exactly 0 behind lens, and the last state (B, D) float32, which the next call
    over the same sequences takes as h0.
    """
    _check("x", x, contiguous=False)
    if x.dim() != 3:
        raise ValueError("x must be (B, L, D)")
    dtype_code(x.dtype, "x")
    _check("z", z, x.device, x.dtype, x.shape, contiguous=False)
    for name, t in (("x", x), ("z", z)):
        if not _contiguous_channels(t):
            raise ValueError("%s must have contiguous channels" % name)
    if h0 is not None:
        _check("h0", h0, x.device, torch.float32, (x.shape[0], x.shape[2]))
    if lens is not None:
        _check("lens", lens, x.device, torch.int32, x.shape[:1])
    if _recorded(x, z, h0):
        return _GatedRecurrence.apply(x, z, h0, lens)
    return _recurrence_forward(x, z, h0, lens, False)[:2]


# ---------------------------------------------------------------- dropout

def _dropout_call(x, p, rng, rng_out=None):
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _call(_library().rnnt_dropout, x.device, _ptr(x), x.numel(), dtype_code(x.dtype), p, _ptr(rng), _ptr(rng_out), _ptr(y))
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, rng):
        ctx.p = p
        used = torch.empty_like(rng)  # the caller may move rng on before the backward pass
        y = _dropout_call(x, p, rng, used)
        ctx.save_for_backward(used)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return _dropout_call(dy.contiguous(), ctx.p, *_dense(*ctx.saved_tensors)), None, None


def dropout(x, p, rng):
    """x with every element 0 with probability p, the others divided by 1 - p (p to 16 bits).

    x contiguous, float32/bfloat16/float16; rng: int64 GPU tensor {seed, offset}, read on the
    device and not changed.  Equal seeds and offsets give equal masks, so a program takes a new
    offset for every call (`rng[1] += 1`, also inside a captured graph).  The mask is never
    stored: the backward pass counts the same numbers again.
    """
    _check("x", x)
    dtype_code(x.dtype, "x")
    p = _check_p(p)
    _check("rng", rng, x.device, torch.int64, (2,))
    if _recorded(x):
        return _Dropout.apply(x, p, rng)
    return _dropout_call(x, p, rng)


# ---------------------------------------------------------------- the joint's hidden layer

def _joint_forward(enc, pred, logit_lens, label_lens, act, p, rng, rng_out=None, for_gradient=False):
    B, T, H = enc.shape
    U1 = pred.shape[1]
    shape = _shape(JointShape, "rnnt_joint_hidden_grad_workspace_bytes", B, T, U1 - 1, H, dtype_code(enc.dtype))
    if for_gradient:
        _check_gradient(shape, B, T, U1, H)
    h = torch.empty((B, T, U1, H), dtype=enc.dtype, device=enc.device)
    _call(_library().rnnt_joint_hidden, enc.device, _ptr(enc), _ptr(pred), shape[0], _ptr(logit_lens), _ptr(label_lens),
          act, p, _ptr(rng), _ptr(rng_out), _ptr(h))
    return h, shape


class _JointHidden(torch.autograd.Function):
    @staticmethod
    def forward(ctx, enc, pred, logit_lens, label_lens, act, p, rng):
        ctx.act, ctx.p = act, p
        used = None if rng is None else torch.empty_like(rng)
        h, ctx.shape = _joint_forward(enc, pred, logit_lens, label_lens, act, p, rng, used,
                                      any(ctx.needs_input_grad[:2]))
        ctx.save_for_backward(enc, pred, logit_lens, label_lens, used)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        enc, pred, logit_lens, label_lens, used = _dense(*ctx.saved_tensors)
        (shape, nbytes), dh = ctx.shape, dh.contiguous()
        denc, ws = _result(enc.shape, enc.dtype, enc.device, nbytes)
        dpred = torch.empty_like(pred)
        _call(_library().rnnt_joint_hidden_grad, enc.device, _ptr(enc), _ptr(pred), shape, _ptr(logit_lens),
              _ptr(label_lens), ctx.act, ctx.p, _ptr(used), _ptr(dh), _ptr(denc), _ptr(dpred), *_workspace_args(ws))
        return denc, dpred, None, None, None, None, None


def joint_hidden(enc, pred, logit_lens, label_lens, activation="relu", p=0.0, rng=None):
    """dropout(activation(enc[:, :, None] + pred[:, None])): (B, T, U+1, H), the input of the
    projection whose output rnnt_loss takes.

    enc (B, T, H) and pred (B, U+1, H) contiguous, of one dtype; logit_lens, label_lens (B,)
    int32; activation "relu" or "tanh"; p and rng as in dropout (p = 0 needs no rng).  Rows
    t >= logit_lens[b] or u > label_lens[b] are exactly 0.
    """
    _check("enc", enc)
    if enc.dim() != 3:
        raise ValueError("enc must be (B, T, H)")
    dtype_code(enc.dtype, "enc")
    _check("pred", pred, enc.device, enc.dtype)
    if pred.dim() != 3 or pred.shape[0] != enc.shape[0] or pred.shape[2] != enc.shape[2]:
        raise ValueError("pred must be (B, U+1, H) with enc's B and H")
    for name, lens in (("logit_lens", logit_lens), ("label_lens", label_lens)):
        _check(name, lens, enc.device, torch.int32, (enc.shape[0],))
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be one of %s" % sorted(ACTIVATIONS))
    p = _check_p(p)
    if p > 0.0 and rng is None:
        raise ValueError("dropout needs rng")
    if rng is not None:
        _check("rng", rng, enc.device, torch.int64, (2,))
    args = (enc, pred, logit_lens, label_lens, ACTIVATIONS[activation], p, rng)
    if _recorded(enc, pred):
        return _JointHidden.apply(*args)
    return _joint_forward(*args)[0]
