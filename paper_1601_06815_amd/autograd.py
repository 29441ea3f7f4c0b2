"""torch.autograd binding of the OaA convolution layer, of group normalisation
with an activation, and the clipping of a network's gradients.

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
planes, or tensors in torch's channels_last layout; ``clip_grad_norm_`` clips
the gradients that the backward passes left in a network's parameters.
"""

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


def _laid_out(t, layout=None):
    """t if the library takes its strides (in `layout`, if one is given), or a
    dense copy of it."""
    try:
        binding._norm_layout(t, "x", layout)
    except ValueError:
        if layout == binding.LAYOUT_CHANNELS_LAST:
            return t.movedim(1, -1).contiguous().movedim(-1, 1)
        return t.contiguous()
    return t


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


@torch.no_grad()
def clip_grad_norm_(parameters, max_norm, norm_type=2.0):
    """Scale the gradients of the parameters in place so that their norm is at
    most max_norm; returns the norm before, a scalar on the device (nothing
    waits for it). Parameters without a gradient are left out."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    return binding.grad_clip([p.grad for p in parameters if p.grad is not None], max_norm, norm_type)
