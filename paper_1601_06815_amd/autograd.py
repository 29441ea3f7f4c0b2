"""torch.autograd binding of the OaA convolution layer, of group normalisation
with an activation, of the gated unit and dropout, and the clipping of a network's
gradients.

Training needs the forward convolution and the two backward convolutions
(arXiv:1601.06815, Section 3.2); ``OaAConv2dFunction`` connects them to
autograd and ``OaAConv2d`` holds a weight like a layer. Argument marshalling
only: every pass runs in the library's kernels through ``binding.Plan``.

The layer computes a true convolution (the kernel flipped), valid output,
stride 1: y = OaAConv2d(x) equals torch's cross-correlation
``conv2d(x, w.flip(-1, -2))``.

Spectra cached by a plan belong to the last pass it ran. The backward pass
reuses the kernel and input spectra of its own forward pass when the plan has
run nothing since (its ``generation`` counter, which every pass of the plan
advances, is unchanged), and recomputes them from the saved tensors
otherwise.

``group_norm`` (``GroupNorm`` as a layer) takes the convolution's output in
planes, or tensors in torch's channels_last layout, and so do ``gated``
(``GatedUnit``), which mixes the channels at each position (tokens [T, C] are
positions too), and ``dropout`` (``Dropout``), which adds a residual in the same
pass; ``clip_grad_norm_`` clips the gradients that the backward passes left in a
network's parameters.
"""

import functools
import math

import torch
from torch.autograd import forward_ad

from . import binding


class OaAConv2dFunction(torch.autograd.Function):
    """y = conv(x, w) through ``plan`` (a binding.Plan of matching shape)."""

    @staticmethod
    def forward(ctx, x, w, plan):
        x, w = x.contiguous(), w.contiguous()
        y = plan.forward(x, w)
        ctx.generation = plan.generation
        ctx.plan = plan
        ctx.save_for_backward(x, w)
        return y

    @staticmethod
    def backward(ctx, gy):
        x, w = ctx.saved_tensors
        plan = ctx.plan
        gy = gy.contiguous()
        need_x, need_w = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        if not (need_x or need_w):
            return None, None, None
        fresh = plan.generation == ctx.generation
        # both gradients start from the gradient windows transformed here
        # (which the fused passes do not keep: they transform them again)
        dx = plan.backward_data(gy, None if fresh else w)
        dw = (plan.backward_filter(None if fresh else x, None if plan.caches_grad_spectra else gy)
              if need_w else None)
        return (dx if need_x else None), dw, None


class OaAConv2d(torch.nn.Module):
    """Convolution layer with K = out_channels kernels of side kernel_size over
    C = in_channels channels; one plan (and device workspace) per input shape.
    ``tiling`` is passed to binding.Plan ("auto", "paper" or (L, b))."""

    def __init__(self, in_channels, out_channels, kernel_size, tiling="auto", device="cuda"):
        super().__init__()
        self.C, self.K, self.n = in_channels, out_channels, kernel_size
        self.tiling = tiling
        std = math.sqrt(1.0 / (in_channels * kernel_size * kernel_size))
        self.weight = torch.nn.Parameter(
            torch.randn(out_channels, in_channels, kernel_size, kernel_size, device=device) * std)
        self._plans = {}

    def plan_for(self, B, N):
        key = (B, N, self.weight.device)
        if key not in self._plans:
            self._plans[key] = binding.Plan(B, self.C, self.K, N, self.n, device=self.weight.device,
                                            tiling=self.tiling)
        return self._plans[key]

    def forward(self, x):
        B, C, N, N2 = x.shape
        if C != self.C or N != N2:
            raise ValueError(f"expected x[B,{self.C},N,N], got {tuple(x.shape)}")
        return OaAConv2dFunction.apply(x, self.weight, self.plan_for(B, N))


@functools.lru_cache(maxsize=4096)
def _layout(shape, strides, want=None):
    """The layout (`want`, if one is given) of a tensor's strides; None if the library
    does not take them."""
    try:
        return binding._layout_of(shape, strides, "x", want)[0]
    except ValueError:
        return None


def _laid_out(t, layout=None):
    """t if the library takes its strides (in `layout`, if one is given), or a
    dense copy of it."""
    if _layout(t.shape, t.stride(), layout) is not None:
        return t
    if layout == binding.LAYOUT_CHANNELS_LAST:
        return t.movedim(1, -1).contiguous().movedim(-1, 1)
    return t.contiguous()


class GroupNormFunction(torch.autograd.Function):
    """y = act(group_norm(x) weight + bias)."""

    @staticmethod
    def forward(ctx, x, weight, bias, num_groups, eps, activation):
        record = binding.GroupNormRecord(x, num_groups, weight, bias, eps, activation)
        y, buffer = record.y, record.buffer
        record.y = record.buffer = None  # autograd keeps what the backward pass needs
        ctx.record = record
        ctx.save_for_backward(x, weight, bias, buffer)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, buffer = ctx.saved_tensors
        if dy.stride() != x.stride():
            dy = _laid_out(dy, binding._norm_layout(x, "x")[0])
        need_x, need_weight, need_bias = ctx.needs_input_grad[:3]
        dx, dweight, dbias = ctx.record.backward(dy, x, weight, bias, buffer, need_x, need_weight, need_bias)
        return dx, dweight, dbias, None, None, None


def group_norm(x, num_groups, weight=None, bias=None, eps=1e-5, activation="none"):
    """Group normalisation of x[B, C, ...] over num_groups groups of neighbouring
    channels, with weight[C] and bias[C], then the activation ("none", "relu",
    "silu", "gelu"). x is float32, bfloat16 or float16 in planes or channels
    last, and y like it; parameters are float32 or of x's type."""
    if not x.is_contiguous():
        x = _laid_out(x)
    # forward-mode derivatives are refused by the function, not dropped
    if forward_ad._current_level >= 0 or torch.is_grad_enabled() and (
            x.requires_grad or (weight is not None and weight.requires_grad) or
            (bias is not None and bias.requires_grad)):
        return GroupNormFunction.apply(x, weight, bias, num_groups, eps, activation)
    return binding.group_norm_forward(x, num_groups, weight, bias, eps, activation, stats=False)[0]


class GroupNorm(torch.nn.Module):
    """Group normalisation layer over num_channels channels in num_groups groups,
    with its activation; ``affine`` gives it a weight and a bias."""

    def __init__(self, num_groups, num_channels, eps=1e-5, affine=True, activation="none", device="cuda",
                 dtype=torch.float32):
        super().__init__()
        if num_groups < 1 or num_channels % num_groups:
            raise ValueError(f"{num_channels} channels do not divide into {num_groups} groups")
        if activation not in binding.ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(binding.ACTIVATIONS)}, got {activation!r}")
        self.G, self.C, self.eps, self.activation = num_groups, num_channels, eps, activation
        for name, value in (("weight", 1.0), ("bias", 0.0)):
            self.register_parameter(name, torch.nn.Parameter(torch.full((num_channels,), value, device=device,
                                                                        dtype=dtype)) if affine else None)

    def forward(self, x):
        if x.dim() < 2 or x.shape[1] != self.C:
            raise ValueError(f"expected x[B,{self.C},...], got {tuple(x.shape)}")
        return group_norm(x, self.G, self.weight, self.bias, self.eps, self.activation)


def _rows(weight):
    """weight[F, C], or a copy, with rows of neighbouring values."""
    if weight.dim() == 2 and weight.stride(1) == 1 and weight.stride(0) >= weight.shape[1]:
        return weight
    return weight.contiguous()


def _recorded(*tensors):
    """Whether autograd has to see a call: forward-mode derivatives are refused by the
    functions, not dropped."""
    return forward_ad._current_level >= 0 or torch.is_grad_enabled() and any(
        t is not None and t.requires_grad for t in tensors)


class GatedFunction(torch.autograd.Function):
    """h = act(gate_weight x + gate_bias) (up_weight x + up_bias)."""

    @staticmethod
    def forward(ctx, x, gate_weight, up_weight, gate_bias, up_bias, activation):
        x = _laid_out(x)
        h, gate, up = binding.gated_forward(x, gate_weight, up_weight, gate_bias, up_bias, activation)
        ctx.activation = activation
        ctx.save_for_backward(x, gate_weight, up_weight, gate, up)
        return h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        x, gate_weight, up_weight, gate, up = ctx.saved_tensors
        # hooks on saved tensors may bring them back with other strides than they had
        x = _laid_out(x)
        layout = _layout(x.shape, x.stride())
        dh, gate, up = (t if t.dim() == 1 else _laid_out(t, layout) for t in (dh, gate, up))
        need = ctx.needs_input_grad
        grads = binding.gated_backward(dh, x, _rows(gate_weight), _rows(up_weight), gate, up, ctx.activation, need[0],
                                       need[1] or need[2], need[3] or need[4])
        return (*(g if n else None for g, n in zip(grads, need)), None)


def gated(x, gate_weight, up_weight, gate_bias=None, up_bias=None, activation="silu"):
    """act(gate_weight x + gate_bias) (up_weight x + up_bias) over the channels of
    x[B, C, ...] at each position: [B, F, ...] for weights [F, C], in x's layout.
    Tokens are x[T, C]. float32, bfloat16 or float16, all of one type."""
    gate_weight, up_weight = _rows(gate_weight), _rows(up_weight)
    gate_bias, up_bias = (b if b is None or b.is_contiguous() else b.contiguous() for b in (gate_bias, up_bias))
    if _recorded(x, gate_weight, up_weight, gate_bias, up_bias):
        return GatedFunction.apply(x, gate_weight, up_weight, gate_bias, up_bias, activation)
    return binding.gated_forward(_laid_out(x), gate_weight, up_weight, gate_bias, up_bias, activation, keep=False)[0]


class GatedUnit(torch.nn.Module):
    """The gated unit from in_channels to hidden_channels as a layer."""

    def __init__(self, in_channels, hidden_channels, bias=True, activation="silu", device="cuda", dtype=torch.float32):
        super().__init__()
        if activation not in binding.ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(binding.ACTIVATIONS)}, got {activation!r}")
        self.C, self.F, self.activation = in_channels, hidden_channels, activation
        for name in ("gate", "up"):
            weight = torch.randn(hidden_channels, in_channels, device=device) / math.sqrt(in_channels)
            self.register_parameter(name + "_weight", torch.nn.Parameter(weight.to(dtype)))
            self.register_parameter(name + "_bias", torch.nn.Parameter(
                torch.zeros(hidden_channels, device=device, dtype=dtype)) if bias else None)

    def forward(self, x):
        if x.dim() < 2 or x.shape[1] != self.C:
            raise ValueError(f"expected x[B,{self.C},...], got {tuple(x.shape)}")
        return gated(x, self.gate_weight, self.up_weight, self.gate_bias, self.up_bias, self.activation)


class DropoutFunction(torch.autograd.Function):
    """y = residual + x / (1 - p) where the mask of seed keeps x."""

    @staticmethod
    def forward(ctx, x, p, seed, residual):
        x = _laid_out(x)
        ctx.layout = _layout(x.shape, x.stride())
        ctx.p, ctx.dtype = p, x.dtype
        # (without a mask any seed will do, and one that a layer advances would be found changed)
        ctx.save_for_backward(seed if p > 0.0 else seed.clone())
        return binding.dropout(x, p, seed, None if residual is None else _laid_out(residual, ctx.layout))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        seed, = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            dx = binding.dropout(_laid_out(dy, ctx.layout), ctx.p, seed, dtype=ctx.dtype)
        return dx, None, None, dy if ctx.needs_input_grad[3] else None


def dropout(x, p, seed, residual=None):
    """residual + x / (1 - p) where the mask of ``seed`` keeps x, residual elsewhere.
    seed is an int64 tensor [key, call] on the device (``Dropout`` keeps one); equal
    seeds give equal masks. x[B, C, ...] is float32, bfloat16 or float16 in planes or
    channels last (element i of the mask is element i of that layout); residual and
    the result are of x's type or float32."""
    if _recorded(x, residual):
        return DropoutFunction.apply(x, p, seed, residual)
    x = _laid_out(x)
    if residual is not None:
        residual = _laid_out(residual, _layout(x.shape, x.stride()))
    return binding.dropout(x, p, seed, residual)


class Dropout(torch.nn.Module):
    """Dropout with probability p while training. Its state (a key and the number of
    calls) is a buffer on the device that every call advances there, so that a
    captured graph draws another mask at each replay. A call that is made again for the
    backward pass, as by torch.utils.checkpoint, draws another one too: there, draw the
    seed once (``binding.dropout_next(state)``) and call ``dropout`` with it. Copies of a
    layer have its key and draw the same masks, and so do the ranks of a distributed job whose
    torch generators were seeded alike, or whose wrapper sends rank 0's buffers to the others
    (``broadcast_buffers=True``): give each rank another ``seed``, and keep its buffers."""

    def __init__(self, p=0.5, seed=None, device="cuda"):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"the probability must be in [0, 1], not {p!r}")
        self.p = p
        key = int(torch.randint(0, 1 << 62, (1,))) if seed is None else seed
        self.register_buffer("state", torch.tensor([key, 0], dtype=torch.int64, device=device))

    def forward(self, x, residual=None):
        if self.training and self.p > 0.0:
            return dropout(x, self.p, binding.dropout_next(self.state), residual)
        return x if residual is None else dropout(x, 0.0, self.state, residual)


@torch.no_grad()
def clip_grad_norm_(parameters, max_norm, norm_type=2.0):
    """Scale the gradients of the parameters in place so that their norm is at
    most max_norm; returns the norm before, a scalar on the device (nothing
    waits for it). Parameters without a gradient are left out."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    return binding.grad_clip([p.grad for p in parameters if p.grad is not None], max_norm, norm_type)
