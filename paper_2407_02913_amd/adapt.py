"""Operators around the frozen int8 convolutions: what is tuned and served beside them.

Functions of torch tensors on the GPU over the library's C entry points (``include/sfc.h``); every
numeric step runs in its HIP kernels.  They work on the tensors' device and its current stream, return
new tensors and never synchronize.  Descriptions are checked by the library (:class:`binding.SfcError`),
shapes, types and devices here (``ValueError``).

* ``group_norm``: group norm with an activation, channels last or planes; ``group_norm_i8`` hands on the
  next convolution's int8 activations.
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
