"""Operators around the frozen int8 convolutions: what is tuned and served beside them.

Functions of torch tensors on the GPU over the library's C entry points (``include/sfc.h``); every
numeric step runs in its HIP kernels.  They work on the tensors' device and its current stream, return
new tensors and never synchronize.  Descriptions are checked by the library (:class:`binding.SfcError`),
shapes, types and devices here (``ValueError``).

* ``group_norm``: group norm with an activation, channels last or planes; ``group_norm_i8`` hands on the
  next convolution's int8 activations.
* ``adapters``: low-rank adapters of many requests, added to a projection that all of them share.
* ``distill``: the loss of a student's logits against a teacher's top ones; ``distill_loss_and_grad`` gives
  the gradient in the same pass over the logits.
"""
from __future__ import annotations

import ctypes as C
from functools import lru_cache

import torch

from . import binding

_TYPE = {torch.float32: binding.TYPE_F32, torch.float16: binding.TYPE_F16, torch.bfloat16: binding.TYPE_BF16,
         torch.int8: binding.TYPE_I8}


def _require(ok, message):
    if not ok:
        raise ValueError(message)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(device, name, *args):
    """Calls a C entry point with the current stream of `device`, which is made the current one."""
    lib = binding._lib or binding.load()
    if device.index == torch.cuda.current_device():
        status = getattr(lib, name)(*args, binding._stream_ptr(None))
    else:
        with torch.cuda.device(device):
            status = getattr(lib, name)(*args, binding._stream_ptr(None))
    if status != binding.SFC_OK:
        raise binding.SfcError(status, name)


def _bytes(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


# ---- group norm ----

def _layout(shape, stride, what):
    """(layout, image stride, row stride) of a 4-axis tensor, a stride that is not used as 0 (dense)."""
    n, c, h, w = shape
    sn, sc, sh, sw = stride
    image = sn if n > 1 else 0
    pixels = h * w
    if pixels != 1 and (w == 1 or sw == 1) and (h == 1 or sh == w):
        return binding.LAYOUT_NCHW, image, sc if c > 1 else 0
    if c == 1 or sc == 1:
        if pixels <= 1:
            return binding.LAYOUT_NHWC, image, 0
        row = sw if w > 1 else sh
        if h == 1 or w == 1 or sh == w * sw:
            return binding.LAYOUT_NHWC, image, row
    if pixels == 1:
        return binding.LAYOUT_NCHW, image, sc
    raise ValueError(f"{what}: neither planes (NCHW) nor channels last (NHWC): shape {shape}, strides {stride}")


class _Norm:
    """A checked description with its workspace sizes."""

    def __init__(self, shape, x, y, groups, eps, activation, y_scale):
        _require(activation in binding.ACTIVATION, f"activation {activation!r}: one of {sorted(binding.ACTIVATION)}")
        self.desc = binding.GroupNormDesc(*shape, groups, x[0], y[0], x[1], y[1], binding.ACTIVATION[activation],
                                          eps, y_scale, x[2], x[3], y[2], y[3])
        self.at = C.addressof(self.desc)
        forward, backward = C.c_size_t(), C.c_size_t()
        binding._check(binding.load().sfc_group_norm_sizes(self.at, C.byref(forward), C.byref(backward)),
                       "sfc_group_norm_sizes")
        self.forward_bytes, self.backward_bytes = forward.value, backward.value


@lru_cache(maxsize=1024)
def _norm(shape, x_stride, x_dtype, y_stride, y_dtype, groups, eps, activation, y_scale):
    x, y = _layout(shape, x_stride, "x"), _layout(shape, y_stride, "y")
    if shape[2] * shape[3] == 1 or shape[1] == 1:
        # (one pixel, or one channel: both layouts at once; the other tensor's is taken)
        if y_dtype == torch.int8:
            y = (binding.LAYOUT_NCHW, y[1], y[2] if y[0] == binding.LAYOUT_NCHW else 0)
    return _Norm(shape, (_TYPE[x_dtype], *x), (_TYPE[y_dtype], *y), groups, eps, activation, y_scale)


def _check_norm(x, weight, bias):
    _require(x.is_cuda and x.dim() == 4, f"x: a 4-axis tensor on the GPU, not {tuple(x.shape)} on {x.device}")
    _require(x.dtype in _TYPE and x.dtype != torch.int8, f"x: float32, float16 or bfloat16, not {x.dtype}")
    for name, p in (("weight", weight), ("bias", bias)):
        if p is not None:
            _require(p.dtype == torch.float32 and p.shape == x.shape[1:2] and p.device == x.device
                     and (p.is_contiguous()), f"{name}: float32 [{x.shape[1]}] on {x.device}, contiguous")


def _norm_forward(x, groups, weight, bias, eps, activation, dtype, y_scale, channels_last):
    _check_norm(x, weight, bias)
    shape = tuple(x.shape)
    if channels_last is None:
        planes = (dtype == torch.int8 or x.is_contiguous()
                  or _layout(shape, x.stride(), "x")[0] == binding.LAYOUT_NCHW)
    else:
        planes = not channels_last
    y = torch.empty(shape, dtype=dtype, device=x.device,
                    memory_format=torch.contiguous_format if planes else torch.channels_last)
    norm = _norm(shape, x.stride(), x.dtype, y.stride(), dtype, groups, eps, activation, y_scale)
    stats = torch.empty((shape[0], groups, 2), dtype=torch.float32, device=x.device)
    space = _bytes(norm.forward_bytes, x.device)
    _call(x.device, "sfc_group_norm", norm.at, x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(),
          stats.data_ptr(), _ptr(space), norm.forward_bytes)
    return y, stats


def group_norm_forward(x, groups, weight=None, bias=None, eps=1e-5, activation="none", dtype=None,
                       channels_last=None):
    """(y, stats): y = activation(h weight + bias), h the values of x [N, C, H, W] less the mean of their
    group (C / groups channels, all pixels of an image), over its standard deviation.

    x is planes (NCHW) or channels last, with any image and row strides, in float32, float16 or bfloat16;
    weight and bias float32 [C] or None.  y has x's type and layout, or `dtype` (a 16-bit type from
    float32) and `channels_last`.  stats, float32 [N, groups, 2], are mean and 1 / sqrt(var + eps).
    activation: "none", "relu", "silu" or "gelu" (the exact one, with erf)."""
    return _norm_forward(x, groups, weight, bias, eps, activation, dtype or x.dtype, 0.0, channels_last)


def group_norm_i8(x, groups, weight=None, bias=None, eps=1e-5, activation="relu", *, y_scale):
    """The next convolution's activations: y of group_norm_forward as int8 planes,
    clamp(round-half-even(y / y_scale), -127, 127)."""
    return _norm_forward(x, groups, weight, bias, eps, activation, torch.int8, float(y_scale), False)[0]


def group_norm_backward(dy, x, stats, groups, weight=None, bias=None, eps=1e-5, activation="none"):
    """(dx, dweight, dbias) from y's gradient dy (x's type and layout), x and the forward call's stats.
    dweight and dbias, float32 [C], are sums over images in a fixed order."""
    _check_norm(x, weight, bias)
    _require(dy.shape == x.shape and dy.dtype == x.dtype and dy.device == x.device,
             f"dy: as x, {tuple(x.shape)} {x.dtype}, not {tuple(dy.shape)} {dy.dtype}")
    _require(stats.shape == (x.shape[0], groups, 2) and stats.dtype == torch.float32 and stats.is_contiguous()
             and stats.device == x.device, f"stats: float32 {(x.shape[0], groups, 2)}, as the forward call gave them")
    shape = tuple(x.shape)
    norm = _norm(shape, x.stride(), x.dtype, dy.stride(), x.dtype, groups, eps, activation, 0.0)
    if x.is_contiguous() or x.is_contiguous(memory_format=torch.channels_last):
        dx = torch.empty_like(x)
    else:  # (x's strides, gaps included)
        dx = torch.empty_strided(shape, x.stride(), dtype=x.dtype, device=x.device)
    grads = torch.empty((2, shape[1]), dtype=torch.float32, device=x.device)
    dweight, dbias = grads.unbind(0)
    space = _bytes(norm.backward_bytes, x.device)
    _call(x.device, "sfc_group_norm_backward", norm.at, x.data_ptr(), dy.data_ptr(), _ptr(weight), _ptr(bias),
          stats.data_ptr(), dx.data_ptr(), dweight.data_ptr(), dbias.data_ptr(), _ptr(space), norm.backward_bytes)
    return dx, dweight, dbias


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, activation):
        y, stats = group_norm_forward(x, groups, weight, bias, eps, activation)
        ctx.save_for_backward(x, weight, bias, stats)
        ctx.how = groups, eps, activation
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, stats = ctx.saved_tensors
        groups, eps, activation = ctx.how
        last = _layout(tuple(x.shape), x.stride(), "x")[0] == binding.LAYOUT_NHWC
        dy = dy.contiguous(memory_format=torch.channels_last if last else torch.contiguous_format)
        dx, dweight, dbias = group_norm_backward(dy, x, stats, groups, weight, bias, eps, activation)
        return dx, None if weight is None else dweight, None if bias is None else dbias, None, None, None


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, activation="none"):
    """y of group_norm_forward, in x's type and layout; differentiable in x, weight and bias."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias)):
        return _GroupNorm.apply(x, weight, bias, groups, eps, activation)
    return group_norm_forward(x, groups, weight, bias, eps, activation)[0]


# ---- low-rank adapters ----

class _Lowrank:
    """A description with its workspace sizes."""

    def __init__(self, *fields):
        self.desc = binding.LowrankDesc(*fields)
        self.at = C.addressof(self.desc)
        forward, backward = C.c_size_t(), C.c_size_t()
        binding._check(binding.load().sfc_lowrank_sizes(self.at, C.byref(forward), C.byref(backward)),
                       "sfc_lowrank_sizes")
        self.forward_bytes, self.backward_bytes = forward.value, backward.value


_lowrank = lru_cache(maxsize=1024)(_Lowrank)


def _row_stride(t, what):
    _require(t.shape[1] <= 1 or t.stride(1) == 1, f"{what}: a row's values lie side by side, not strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else 0


def _check_adapters(x, ids, down, up, scale, outputs, wide):
    """`outputs`, `wide`: (name, tensor or None) with as many columns as `up` has outputs, `down` inputs."""
    _require(x.is_cuda and x.dim() == 2, f"x: [tokens, inputs] on the GPU, not {tuple(x.shape)} on {x.device}")
    _require(x.dtype in _TYPE and x.dtype != torch.int8, f"x: float32, float16 or bfloat16, not {x.dtype}")
    tokens, inputs = x.shape
    _require(down.dim() == 3 and down.shape[2] == inputs and down.dtype == x.dtype and down.is_contiguous()
             and down.device == x.device, f"down: {x.dtype} [adapters, rank, {inputs}] on {x.device}, contiguous")
    adapters, rank, _ = down.shape
    _require(up.dim() == 3 and up.shape[0] == adapters and up.shape[2] == rank and up.dtype == x.dtype
             and up.is_contiguous() and up.device == x.device,
             f"up: {x.dtype} [{adapters}, outputs, {rank}] on {x.device}, contiguous")
    _require(ids.shape == (tokens,) and ids.dtype == torch.int32 and ids.is_contiguous() and ids.device == x.device,
             f"ids: int32 [{tokens}] on {x.device}, contiguous")
    if scale is not None:
        _require(scale.shape == (adapters,) and scale.dtype == torch.float32 and scale.is_contiguous()
                 and scale.device == x.device, f"scale: float32 [{adapters}] on {x.device}, contiguous")
    for columns, tensors in ((up.shape[1], outputs), (inputs, wide)):
        for name, t in tensors:
            _require(t is None or (t.shape == (tokens, columns) and t.dtype == x.dtype and t.device == x.device),
                     f"{name}: {x.dtype} [{tokens}, {columns}] on {x.device}")
    return tokens, inputs, up.shape[1], rank, adapters, _TYPE[x.dtype]


def add_adapters(base, x, ids, down, up, scale=None, out=None):
    """y[t] = base[t] + scale[l] up[l] (down[l] x[t]), l = ids[t]: the low-rank adapters of many requests, beside a
    projection that all of them share.

    x [tokens, inputs]; base [tokens, outputs], the shared projection's output, or None; down [adapters, rank, inputs] and
    up [adapters, outputs, rank]; one type, float32, float16 or bfloat16.  ids, int32 [tokens]: any order; an id
    outside the adapters is none, y = base.  scale, float32 [adapters], or None.  `out` may be base."""
    fields = _check_adapters(x, ids, down, up, scale, (("base", base), ("out", out)), ())
    y = torch.empty((fields[0], fields[2]), dtype=x.dtype, device=x.device) if out is None else out
    plan = _lowrank(*fields, _row_stride(x, "x"), 0 if base is None else _row_stride(base, "base"), _row_stride(y, "out"), 0)
    space = _bytes(plan.forward_bytes, x.device)
    _call(x.device, "sfc_lowrank_add", plan.at, x.data_ptr(), ids.data_ptr(), down.data_ptr(), up.data_ptr(), _ptr(scale),
          _ptr(base), y.data_ptr(), _ptr(space), plan.forward_bytes)
    return y


def add_adapters_backward(dy, x, ids, down, up, scale=None, dx_base=None):
    """(dx, d_down, d_up) from y's gradient dy: dx = dx_base + scale[l] (up[l] down[l])^T dy, where dx_base is the shared
    projection's part or None; the factors' gradients, in their type, are sums over each adapter's tokens."""
    fields = _check_adapters(x, ids, down, up, scale, (("dy", dy),), (("dx_base", dx_base),))
    dx = torch.empty((fields[0], fields[1]), dtype=x.dtype, device=x.device)
    d_down, d_up = torch.empty_like(down), torch.empty_like(up)
    plan = _lowrank(*fields, _row_stride(x, "x"), 0 if dx_base is None else _row_stride(dx_base, "dx_base"),
                    _row_stride(dy, "dy"), 0)
    space = _bytes(plan.backward_bytes, x.device)
    _call(x.device, "sfc_lowrank_backward", plan.at, x.data_ptr(), dy.data_ptr(), ids.data_ptr(), down.data_ptr(),
          up.data_ptr(), _ptr(scale), _ptr(dx_base), dx.data_ptr(), d_down.data_ptr(), d_up.data_ptr(), _ptr(space),
          plan.backward_bytes)
    return dx, d_down, d_up


class _Adapters(torch.autograd.Function):
    @staticmethod
    def forward(ctx, base, x, ids, down, up, scale):
        ctx.save_for_backward(x, ids, down, up, scale)
        ctx.with_base = base is not None
        return add_adapters(base, x, ids, down, up, scale)

    @staticmethod
    def backward(ctx, dy):
        x, ids, down, up, scale = ctx.saved_tensors
        dy = dy.contiguous()
        dx, d_down, d_up = add_adapters_backward(dy, x, ids, down, up, scale)
        return dy if ctx.with_base else None, dx, None, d_down, d_up, None


def adapters(base, x, ids, down, up, scale=None):
    """y of add_adapters; differentiable in base, x, down and up."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (base, x, down, up)):
        return _Adapters.apply(base, x, ids, down, up, scale)
    return add_adapters(base, x, ids, down, up, scale)


# ---- distillation from a teacher's top logits ----

@lru_cache(maxsize=1024)
def _distill(rows, classes, top, dtype, wide, tail, temperature, logits_stride, grad_stride, values_stride, index_stride):
    return binding.DistillDesc(rows, classes, top, _TYPE[dtype], int(wide), int(tail), temperature,
                               logits_stride, grad_stride, values_stride, index_stride)


def _check_distill(logits, values, index, row_scale, temperature, tail, grad=None):
    _require(logits.is_cuda and logits.dim() == 2 and logits.shape[1] > 0,
             f"logits: [rows, classes] on the GPU, not {tuple(logits.shape)} on {logits.device}")
    _require(logits.dtype in _TYPE and logits.dtype != torch.int8,
             f"logits: float32, float16 or bfloat16, not {logits.dtype}")
    rows, classes = logits.shape
    _require(values.dim() == 2 and values.shape[0] == rows and values.dtype == torch.float32
             and values.device == logits.device, f"values: float32 [{rows}, top] on {logits.device}")
    _require(index.shape == values.shape and index.dtype in (torch.int32, torch.int64) and index.device == logits.device,
             f"index: int32 or int64 {tuple(values.shape)} on {logits.device}")
    if row_scale is not None:
        _require(row_scale.shape == (rows,) and row_scale.dtype == torch.float32 and row_scale.is_contiguous()
                 and row_scale.device == logits.device, f"row_scale: float32 [{rows}] on {logits.device}, contiguous")
    desc = _distill(rows, classes, values.shape[1], logits.dtype, index.dtype == torch.int64, tail, temperature,
                    _row_stride(logits, "logits"), 0 if grad is None else _row_stride(grad, "grad"),
                    _row_stride(values, "values"), _row_stride(index, "index"))
    return C.addressof(desc)


def distill_loss(logits, values, index, row_scale=None, temperature=1.0, tail=False):
    """(loss, stats) of each row: the divergence of q = softmax(logits / temperature) from the teacher's p, times
    temperature^2, float32 [rows]; stats, float32 [rows, 4], for distill_grad.

    values, float32 [rows, top], and index, int32 or int64, are the teacher's top logits and their places; p is
    their softmax at the temperature.  tail: the values are log-probabilities at the temperature instead, and what
    they leave is one more outcome, against the student's mass outside the places.  A place outside the classes
    is padding.  row_scale, float32 [rows]: rows of 0 are masked (loss 0, not read)."""
    at = _check_distill(logits, values, index, row_scale, temperature, tail)
    loss = torch.empty(logits.shape[0], dtype=torch.float32, device=logits.device)
    stats = torch.empty((logits.shape[0], 4), dtype=torch.float32, device=logits.device)
    _call(logits.device, "sfc_distill_loss", at, logits.data_ptr(), values.data_ptr(), index.data_ptr(), _ptr(row_scale),
          loss.data_ptr(), stats.data_ptr())
    return loss, stats


def distill_grad(logits, values, index, stats, row_scale=None, temperature=1.0, tail=False, out=None):
    """The gradient of sum(row_scale loss) in the logits, in their type, from distill_loss's stats.  `out` may be
    the logits themselves."""
    grad = torch.empty_like(logits, memory_format=torch.contiguous_format) if out is None else out
    _require(grad.shape == logits.shape and grad.dtype == logits.dtype and grad.device == logits.device,
             f"out: as the logits, {tuple(logits.shape)} {logits.dtype}")
    _require(stats.shape == (logits.shape[0], 4) and stats.dtype == torch.float32 and stats.is_contiguous()
             and stats.device == logits.device, f"stats: float32 [{logits.shape[0]}, 4], as distill_loss gave them")
    at = _check_distill(logits, values, index, row_scale, temperature, tail, grad)
    _call(logits.device, "sfc_distill_grad", at, logits.data_ptr(), values.data_ptr(), index.data_ptr(), _ptr(row_scale),
          stats.data_ptr(), grad.data_ptr())
    return grad


def distill_loss_and_grad(logits, values, index, row_scale=None, temperature=1.0, tail=False, out=None):
    """(loss, gradient) as of distill_loss and distill_grad, the logits read once: for a training step whose loss
    is sum(row_scale loss)."""
    grad = torch.empty_like(logits, memory_format=torch.contiguous_format) if out is None else out
    _require(grad.shape == logits.shape and grad.dtype == logits.dtype and grad.device == logits.device,
             f"out: as the logits, {tuple(logits.shape)} {logits.dtype}")
    at = _check_distill(logits, values, index, row_scale, temperature, tail, grad)
    loss = torch.empty(logits.shape[0], dtype=torch.float32, device=logits.device)
    _call(logits.device, "sfc_distill_loss_grad", at, logits.data_ptr(), values.data_ptr(), index.data_ptr(),
          _ptr(row_scale), loss.data_ptr(), grad.data_ptr())
    return loss, grad


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, values, index, mask, temperature, tail):
        loss, stats = distill_loss(logits, values, index, mask, temperature, tail)
        ctx.save_for_backward(logits, values, index, mask, stats)
        ctx.how = temperature, tail
        return loss

    @staticmethod
    def backward(ctx, dloss):
        logits, values, index, mask, stats = ctx.saved_tensors
        scale = dloss.contiguous() if mask is None else torch.where(mask != 0, dloss, 0.0)
        return (distill_grad(logits, values, index, stats, scale, *ctx.how),) + (None,) * 5


def distill(logits, values, index, mask=None, temperature=1.0, tail=False):
    """loss of distill_loss, float32 [rows]; differentiable in the logits.  mask, float32 [rows]: rows of 0 have
    loss and gradient 0."""
    return _Distill.apply(logits, values, index, mask, temperature, tail)
