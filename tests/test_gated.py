"""The gated unit through the public calls, against the fp64 oracle.

Bounds, value by value, from the arithmetic: with e = 2^-23 for a product or a sum
of the matrix cores (which round toward one side), a sum of K terms is off by at most
(K + 8) e times the sum of their magnitudes. The activations are within 1e-6 of
themselves (GELU's Phi within 2e-7), their first and second derivatives are at most
1.2 and 0.8, and an output adds half a step of its type. dg and du add half a step of
x's type where they enter dx and dW. What these worst cases allow, random signs do
not reach, so that the norm of all errors is held to far less.
"""

import ctypes

import numpy as np
import pytest
import torch
from scipy import special
from torch.autograd import forward_ad

from oracle import block as oracle
from oracle.norm import _act
from paper_1601_06815_amd import autograd, binding

DEV = "cuda:0"
E = 2.0 ** -23
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
# of the norm: half a step of the result and of dg and du is at most 2 steps in all;
# in float32 sums of n terms of either sign gather about sqrt(n) e
NORM = {torch.float32: 4e-6, torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10}
ACTS = sorted(binding.ACTIVATIONS)
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAMES = ("dx", "dgate_weight", "dup_weight", "dgate_bias", "dup_bias")


def wide(t):
    return None if t is None else t.detach().cpu().double().numpy()


def lay(t, layout):
    return t.contiguous() if layout == "planes" else t.movedim(1, -1).contiguous().movedim(-1, 1)


def make(shape, F, layout="planes", dtype=torch.float32, bias=True, seed=0):
    """x, dh, the weights and the biases (or None)."""
    rng = np.random.default_rng(seed)
    C = shape[1]
    x = rng.standard_normal(shape)
    dh = rng.standard_normal((shape[0], F, *shape[2:])) * 0.1
    x, dh = (lay(torch.from_numpy(a).to(DEV, dtype), layout) for a in (x, dh))
    w = [torch.from_numpy(rng.standard_normal((F, C)) / np.sqrt(C)).to(DEV, dtype) for _ in range(2)]
    b = [torch.from_numpy(rng.standard_normal(F) * 0.3).to(DEV, dtype) if bias else None for _ in range(2)]
    return x, dh, *w, *b


class Bounds:
    """The results in float64 and how far float32 or 16-bit ones may be off."""

    def __init__(self, x, gw, uw, gb, ub, act, dtype, dh=None):
        step, least = STEP[dtype], LEAST[dtype]
        C, F = x.shape[1], gw.shape[0]
        V = np.abs(oracle._flat(x))
        g, u = oracle.gated_preactivations(x, gw, uw, gb, ub)
        a, slope = _act(act, g)
        off = []
        for w, b in ((gw, gb), (uw, ub)):
            off.append((C + 8) * E * (V @ np.abs(w).T + (0 if b is None else np.abs(b))))
        G, U = np.abs(g), np.abs(u)
        self.g = g
        of_a = 1.2 * off[0] + 1e-6 * np.abs(a) + 2e-7 * G
        self.h = oracle.gated_forward(x, gw, uw, gb, ub, act)
        h_off = of_a * (U + off[1]) + np.abs(a) * off[1]
        self.h_off = oracle._back(h_off + step * (np.abs(a * u) + h_off) + least, x, F)
        if dh is None:
            return
        self.grads = oracle.gated_backward(dh, x, gw, uw, gb, ub, act)
        D = np.abs(oracle._flat(dh))
        T = D.shape[0]
        dg, du = np.abs(D * u * slope), D * np.abs(a)
        # before dg and du are rounded, for the biases
        og = D * (0.8 * off[0] * (U + off[1]) + 1.2 * off[1] + 3e-6 * U)
        ou = D * (of_a + 1e-6 * np.abs(a))
        rg, ru = (o + step * (v + o) + least for o, v in ((og, dg), (ou, du)))
        W = np.abs(gw), np.abs(uw)
        size = (dg + rg) @ W[0] + (du + ru) @ W[1]
        dx = rg @ W[0] + ru @ W[1] + (2 * F + 8) * E * size
        self.offs = [oracle._back(dx + step * (size + dx) + least, x, C)]
        for r, v in ((rg, dg), (ru, du)):
            size = (v + r).T @ V
            o = r.T @ V + (T + 8) * E * size
            self.offs.append(o + step * (np.abs(self.grads[len(self.offs)]) + o) + least)
        for o, v in ((og, dg), (ou, du)):
            o = o.sum(axis=0) + 300 * E * (v + o).sum(axis=0)
            self.offs.append(o + step * (np.abs(self.grads[len(self.offs)]) + o) + least)


def near(got, ref, off, dtype, what, terms=1):
    got = wide(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert not np.isnan(got).any(), what
    d = np.abs(got - ref)
    assert np.all(d <= off), (what, float(np.max(d / off)), np.unravel_index(np.argmax(d / off), d.shape))
    norm = np.linalg.norm(ref)
    bar = NORM[dtype] + (np.sqrt(terms) * E if dtype == torch.float32 else 0.0)
    # (few values: one of them may be what is left of much larger terms)
    if ref.size >= 256:
        assert np.linalg.norm(d) <= bar * norm + LEAST[dtype] * np.sqrt(ref.size), (what, np.linalg.norm(d) / norm)


def check(x, dh, gw, uw, gb, ub, act="silu", forward_only=False):
    dtype = x.dtype
    W = [wide(t) for t in (gw, uw, gb, ub)]
    if act == "relu" and not forward_only:
        # zero where the pre-activation is so near 0 that rounding decides its side
        g = oracle.gated_preactivations(wide(x), *W)[0]
        corner = torch.from_numpy(oracle._back(np.abs(g) < 1e-3, x, gw.shape[0])).to(DEV)
        dh = dh.clone().masked_fill_(corner, 0.0)
    h, gate, up = binding.gated_forward(x, gw, uw, gb, ub, act)
    alone = binding.gated_forward(x, gw, uw, gb, ub, act, keep=False)
    assert alone[1:] == (None, None) and torch.equal(alone[0], h)
    b = Bounds(wide(x), *W, act, dtype, None if forward_only else wide(dh))
    near(h, b.h, b.h_off, dtype, "h", x.shape[1])
    if forward_only:
        return h
    grads = binding.gated_backward(dh, x, gw, uw, gate, up, act)
    positions = x.numel() // x.shape[1]
    terms = (2 * gw.shape[0], positions, positions, positions, positions)
    for name, got, ref, off, n in zip(NAMES, grads, b.grads, b.offs, terms):
        assert got.dtype == dtype
        near(got, ref, off, dtype, name, n)
    return h, gate, up, grads


SHAPES = [  # (B, C, ...), F: one of each, odd and ragged, multiples, more than a tile of each
    ((1, 1), 1), ((1, 8), 3), ((1, 64), 64), ((2, 33), 65), ((3, 27, 5, 3), 71), ((1, 16, 1, 1), 40),
    ((5, 96), 200), ((17, 130), 129), ((130, 64), 33), ((300, 72), 136), ((2, 5, 31, 17), 9), ((257, 100, 1, 1), 50),
    ((2, 128, 12, 11), 256), ((1, 200, 23, 29), 70), ((3, 64, 7, 7), 130), ((16, 512), 384), ((40, 260, 2, 1), 31),
    ((1, 3, 70, 64), 6), ((2, 6, 3, 5, 7), 10), ((700, 40), 48), ((64, 1030), 24), ((33, 24), 1500),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape,F", SHAPES, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else f"f{v}")
def test_both_passes(gpu_lib, shape, F, layout, dtype):
    i = [s for s, _ in SHAPES].index(shape)
    act = ACTS[(i + (layout == "last") + TYPES.index(dtype)) % 4]
    print(shape, F, layout, dtype, act, flush=True)
    x, *rest = make(shape, F, layout, dtype, bias=i % 3 != 0, seed=i)
    h, gate, up, grads = check(x, *rest, act)
    if shape[1] > 1 and F > 1 and np.prod(shape[2:]) > 1:
        assert grads[0].stride() == x.stride()
        assert binding._norm_layout(h, "h")[0] == binding._norm_layout(x, "x")[0]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_types_and_activations(gpu_lib, layout, dtype, act):
    check(*make((2, 24, 17, 19), 40, layout, dtype, seed=3), act)
    x, _, gw, uw, gb, ub = make((2, 24, 17, 19), 40, layout, dtype, seed=5)
    check(x, None, gw, uw, gb, None, act, forward_only=True)
    check(x, None, gw, uw, None, ub, act, forward_only=True)


# Sizes at which another tile, another way to cut the sum or another kernel takes over.
REACH = [
    ("last", (1, 2048), 300, torch.bfloat16), ("last", (4, 1000), 2000, torch.float16), ("last", (15, 700), 1000, torch.bfloat16),
    ("last", (16, 333), 1000, torch.float16), ("last", (17, 512), 1024, torch.bfloat16), ("last", (31, 256), 600, torch.float32),
    ("last", (48, 640), 512, torch.bfloat16), ("last", (64, 512), 1024, torch.float32), ("last", (65, 300), 700, torch.float16),
    ("last", (128, 512), 512, torch.bfloat16), ("last", (200, 1024), 260, torch.bfloat16), ("last", (513, 256), 384, torch.float32),
    ("last", (2500, 64), 512, torch.bfloat16), ("last", (4100, 128), 256, torch.float16), ("last", (9000, 48), 40, torch.bfloat16),
    ("last", (3, 32, 40, 41), 64, torch.float32), ("planes", (3, 32, 40, 41), 64, torch.float32),
    ("planes", (2, 128, 53, 53), 96, torch.bfloat16), ("planes", (1, 64, 90, 90), 512, torch.float16),
    ("planes", (70, 40, 7, 7), 72, torch.bfloat16), ("planes", (600, 16, 3, 2), 24, torch.float32),
    ("planes", (1, 300, 64, 64), 300, torch.bfloat16), ("last", (20000, 16), 24, torch.float32),
    ("planes", (2, 16, 100, 101), 24, torch.float32), ("last", (1030, 520), 1100, torch.bfloat16),
    ("last", (1500, 700), 520, torch.float32), ("planes", (4, 256, 30, 30), 600, torch.float16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("layout,shape,F,dtype", REACH, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_sizes(gpu_lib, layout, shape, F, dtype):
    print(layout, shape, F, dtype, flush=True)
    check(*make(shape, F, layout, dtype, seed=F))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape,F", [((12, 1001, 40, 41), 770), ((2, 2045, 19, 27), 4091), ((9, 100, 60, 61), 1001),
                                     ((70, 50, 21, 23), 129)])
def test_large_tiles(gpu_lib, shape, F, layout, dtype):
    """Sizes that are multiples of nothing at which each product takes its largest tiles, and
    many of them with short sums, beside each other: h and dx at some positions, the weights'
    and biases' gradients of some hidden channels, which need nothing of the others."""
    x, dh, gw, uw, gb, ub = make(shape, F, layout, dtype, seed=31)
    B, C, H, W = shape
    h, gate, up = binding.gated_forward(x, gw, uw, gb, ub)
    dx, dgw, duw, dgb, dub = binding.gated_backward(dh, x, gw, uw, gate, up)
    T = B * H * W
    rng = np.random.default_rng(1)
    some = np.unique(np.concatenate([rng.integers(0, T, 40), [0, 1, T - 2, T - 1]]))

    def rows(t):
        return t.movedim(1, -1).reshape(T, -1)[torch.from_numpy(some).to(DEV)].contiguous()

    b = Bounds(wide(rows(x)), *map(wide, (gw, uw, gb, ub)), "silu", dtype, wide(rows(dh)))
    near(rows(h), b.h, b.h_off, dtype, "h", C)
    near(rows(dx), b.grads[0], b.offs[0], dtype, "dx", 2 * F)
    few = torch.tensor([k for k in (0, 1, 63, 64, 255, 256, F - 2, F - 1) if k < F], device=DEV)
    b = Bounds(wide(x), *(wide(t[few]) for t in (gw, uw, gb, ub)), "silu", dtype, wide(dh[:, few]))
    for name, got, ref, off in zip(NAMES[1:], (dgw, duw, dgb, dub), b.grads[1:], b.offs[1:]):
        near(got[few], ref, off, dtype, name, T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape,F", [((3, 40, 9, 8), 56), ((2, 70, 31, 5), 150), ((1, 260, 21, 1), 131)])
def test_stored_or_made_again(gpu_lib, shape, F, layout, dtype):
    """Both ways of the backward pass, whichever is the faster: g and u that the forward
    pass stored, and made again."""
    x, dh, gw, uw, gb, ub = make(shape, F, layout, dtype, seed=33)
    B, C, H, W = shape
    last = layout == "last"
    d = desc(B=B, C=C, F=F, S=H * W, layout=int(last), dtype=binding._dtype_codes()[dtype])
    stream = torch.cuda.current_stream().cuda_stream
    ws = [torch.empty(max(1, binding.oaa_gated_workspace_bytes(d, back, 0)), dtype=torch.uint8, device=DEV)
          for back in (0, 1)]
    h = torch.empty_like(dh)
    kept = [torch.full(dh.shape, float("nan"), device=DEV) for _ in range(2)]
    weights = [t.data_ptr() for t in (gw, uw, gb, ub)]
    binding.oaa_gated_forward(d, x.data_ptr(), *weights, h.data_ptr(), *(t.data_ptr() for t in kept),
                              ws[0].data_ptr(), ws[0].numel(), stream)
    assert torch.equal(h, binding.gated_forward(x, gw, uw, gb, ub, keep=False)[0])
    b = Bounds(wide(x), *map(wide, (gw, uw, gb, ub)), "silu", dtype, wide(dh))
    for addresses in ([t.data_ptr() for t in kept], [None, None]):
        grads = [torch.empty_like(t) for t in (x, gw, uw, gb, ub)]
        binding.oaa_gated_backward(d, dh.data_ptr(), x.data_ptr(), *weights, *addresses, *(t.data_ptr() for t in grads),
                                   ws[1].data_ptr(), ws[1].numel(), stream)
        terms = (2 * F, *[x.numel() // C] * 4)
        for name, got, ref, off, n in zip(NAMES, grads, b.grads, b.offs, terms):
            near(got, ref, off, dtype, name, n)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,F", [((150, 300), 260), ((2, 40, 31, 5), 66), ((9, 100), 130)])
@pytest.mark.parametrize("k", [-55, 60])
def test_range_of_float32(gpu_lib, shape, F, k):
    """x times 2^k and the weights over 2^k give the same g and u, and gradients that
    differ by those factors: scaling by a power of two rounds nowhere."""
    x, dh, gw, uw, gb, ub = make(shape, F, dtype=torch.float32, seed=35)
    ref = binding.gated_forward(x, gw, uw, gb, ub)
    grads = binding.gated_backward(dh, x, gw, uw, *ref[1:])
    s = 2.0 ** k
    far = binding.gated_forward(x * s, gw / s, uw / s, gb, ub)
    assert all(torch.equal(a, b) for a, b in zip(ref, far))
    for got, want, scale in zip(binding.gated_backward(dh, x * s, gw / s, uw / s, *far[1:]), grads,
                                (1 / s, s, s, 1.0, 1.0)):
        assert torch.equal(got, want * scale)


def both_backwards(x, dh, gw, uw, gb, ub, act, need=(True,) * 5):
    """The gradients (or None) with g and u stored, and made again: through the C entries."""
    B, C, S = x.shape[0], x.shape[1], int(np.prod(x.shape[2:]))
    F, dtype = gw.shape[0], x.dtype
    last = binding._norm_layout(x, "x")[0]
    d = desc(B=B, C=C, F=F, S=S, layout=last, dtype=binding._dtype_codes()[dtype], activation=binding.ACTIVATIONS[act])
    stream = torch.cuda.current_stream().cuda_stream
    ws = [torch.empty(max(1, binding.oaa_gated_workspace_bytes(d, back, 0)), dtype=torch.uint8, device=DEV)
          for back in (0, 1)]
    h, kept = torch.empty_like(dh), [torch.empty_like(dh, dtype=torch.float32) for _ in range(2)]
    weights = [binding._pointer(t) for t in (gw, uw, gb, ub)]
    binding.oaa_gated_forward(d, x.data_ptr(), *weights, h.data_ptr(), *(t.data_ptr() for t in kept), ws[0].data_ptr(),
                              ws[0].numel(), stream)
    for addresses in ([t.data_ptr() for t in kept], [None, None]):
        shapes = (x, gw, uw, gw[:, 0], uw[:, 0])
        grads = [torch.empty_like(t) if n else None for t, n in zip(shapes, need)]
        binding.oaa_gated_backward(d, dh.data_ptr(), x.data_ptr(), *weights, *addresses, *map(binding._pointer, grads),
                                   ws[1].data_ptr(), ws[1].numel(), stream)
        yield grads


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape,F", [((3, 24, 5, 7), 40), ((2, 70, 31, 5), 150)])
def test_large_gradients_of_small_slopes(gpu_lib, shape, F, layout, dtype, act):
    """dh u is beyond float32 (1e40) where act'(g) is so small that dg is not, or 0.

    The values are of one sign, so that a sum's bound is relative. g, down to -60, or to -8 for
    GELU, is off by (C + 8) 2^-23 of itself, 6e-4 at most; act(g) and act'(g) then by as much
    for SiLU and eight times as much of 8e-5 for GELU; their own errors (below 1e-4 there) and
    a sum of 2 F + 8 terms add 2e-4: 1e-3 in all. Besides, half a step of dg or du and of the
    result."""
    rng = np.random.default_rng(45)
    B, C = shape[:2]
    far = 8.0 if act == "gelu" else 60.0
    x = lay(torch.from_numpy(rng.uniform(0.5, 1.0, shape)).to(DEV, dtype), layout)
    dh = lay(torch.from_numpy(rng.uniform(0.5, 1.0, (B, F, *shape[2:])) * 1e20).to(DEV, dtype), layout)
    gw = torch.from_numpy(-far / C * rng.uniform(0.9, 1.0, (F, C))).to(DEV, dtype)
    uw = torch.from_numpy(1e20 * rng.uniform(0.5, 1.0, (F, C))).to(DEV, dtype)
    values = [wide(t) for t in (x, gw, uw)]
    g, u = oracle.gated_preactivations(*values)
    low = {"relu": 0.0 * g, "silu": np.exp(g) / (1.0 + np.exp(g)), "gelu": special.ndtr(g)}[act]
    slope = {"relu": 0.0 * g, "silu": low * (1.0 + g * (1.0 - low)),
             "gelu": low + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)}[act]
    D, V = oracle._flat(wide(dh)), oracle._flat(values[0])
    dg, du = D * u * slope, D * g * low
    dx = dg @ values[1] + du @ values[2]
    size = np.abs(dg) @ np.abs(values[1]) + np.abs(du) @ np.abs(values[2])  # terms of either sign
    ref = (oracle._back(dx, wide(x), C), dg.T @ V, du.T @ V, dg.sum(axis=0), du.sum(axis=0))
    for grads in both_backwards(x, dh, gw, uw, None, None, act):
        for name, got, r in zip(NAMES, grads, ref):
            scale = oracle._back(size, wide(x), C) if name == "dx" else np.abs(r)
            assert np.isfinite(r).all() and np.isfinite(wide(got)).all(), name
            assert np.all(np.abs(wide(got) - r) <= (1e-3 + 2 * STEP[dtype]) * scale), name


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("shape,F", [((3, 40, 9, 8), 56), ((2, 70, 31, 5), 150), ((1, 260, 21, 1), 131), ((700, 40), 48),
                                     ((9, 24, 29, 31), 700), ((12, 1200), 40)])
@pytest.mark.parametrize("wanted", ["dx", "weights"])
@pytest.mark.parametrize("k", [14, -20])
def test_range_of_float16(gpu_lib, k, wanted, shape, F, act, layout):
    """dg and du that float16 does not hold (beyond 65504, or of no more than four digits),
    where dx or dW is in its range: x and the weights make up for it by powers of two.

    As in Bounds, but the least step of dg and du is that of float16 scaled so that their largest is 2^14 or
    more: half of it is 2^-39 of that."""
    far = 2.0 ** {("dx", 14): 8, ("dx", -20): -10, ("weights", 14): -12, ("weights", -20): 10}[wanted, k]
    x, dh, gw, uw, *_ = make(shape, F, layout, torch.float64, bias=False, seed=47)
    more = 4.0 if k > 0 else 1.0  # (of g and u, so that many are beyond)
    x, gw, uw = x * more * far, gw / far, uw / far
    x, gw, uw, dh = (t.half() for t in (x, gw, uw, dh.clamp(-0.4, 0.4) * 10 * 2.0 ** (k - 1)))
    assert bool(torch.isfinite(dh).all())
    values = [wide(t) for t in (x, gw, uw)]
    g, u = oracle.gated_preactivations(*values)
    a, slope = _act(act, g)
    D, V = np.abs(oracle._flat(wide(dh))), np.abs(oracle._flat(values[0]))
    og, ou = ((shape[1] + 8) * E * (V @ np.abs(w).T) for w in values[1:])
    dg, du = np.abs(D * u * slope), D * np.abs(a)
    most = max(dg.max(), du.max())
    assert most > 65504 if k > 0 else most < 2.0 ** -4
    G, U, step = np.abs(g), np.abs(u), STEP[torch.float16]
    rg = D * (0.8 * og * (U + ou) + 1.2 * ou + 3e-6 * U)
    ru = D * (1.2 * og + 2e-6 * np.abs(a) + 2e-7 * G)
    rg, ru = (o + step * (v + o) + 2.0 ** -39 * most for o, v in ((rg, dg), (ru, du)))
    if wanted == "dx":
        size = (dg + rg) @ np.abs(values[1]) + (du + ru) @ np.abs(values[2])
        offs = [oracle._back(rg @ np.abs(values[1]) + ru @ np.abs(values[2]) + (2 * F + 8) * E * size, wide(x), shape[1])]
    else:
        offs = [r.T @ V + (len(V) + 8) * E * ((v + r).T @ V) for r, v in ((rg, dg), (ru, du))]
    names = ("dx",) if wanted == "dx" else NAMES[1:3]
    refs = dict(zip(NAMES, oracle.gated_backward(wide(dh), *values, activation=act)))
    for grads in both_backwards(x, dh, gw, uw, None, None, act, [n in names for n in NAMES]):
        for name, off in zip(names, offs):
            ref, got = refs[name], grads[NAMES.index(name)]
            assert np.abs(ref).max() < 65504 and np.abs(ref).max() > 2.0 ** -12
            near(got, ref, off + step * (np.abs(ref) + off) + LEAST[torch.float16], torch.float16, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("view", ["channels", "channels last", "rows last", "images", "one image many times",
                                  "one position many times", "odd address", "odd address last"])
def test_strided_tensors(gpu_lib, view, dtype):
    """Slices of larger tensors are read in place, or copied where a row is no whole
    number of 4 bytes, and written in place through h."""
    last = "last" in view or "position" in view
    base, other, *_ = make((4, 12, 9, 7), 20, "last" if last else "planes", dtype, seed=7)
    cut = {"channels": lambda t, n: t[:, 3:3 + n], "channels last": lambda t, n: t[:, 3:3 + n],
           "rows last": lambda t, n: t[:, :n, 2:6], "images": lambda t, n: t[::2, :n],
           "one image many times": lambda t, n: t[:1, :n].expand(3, n, 9, 7),
           "one position many times": lambda t, n: t[:, :n, :1, :1].expand(4, n, 9, 7),
           "odd address": lambda t, n: t.flatten()[1:1 + 2 * n * 63].view(2, n, 9, 7),
           "odd address last": lambda t, n: t.movedim(1, -1).flatten()[1:1 + 126 * n].view(2, 9, 7, n).movedim(-1, 1)}[view]
    x, dh = cut(base, 6), cut(other, 10)
    gw, uw, gb, ub = make((1, 6), 10, dtype=dtype, seed=8)[2:]
    h, gate, up, _ = check(x, dh, gw, uw, gb, ub, "gelu")
    # a slice as the output: what lies around it stays
    B, _, H, W = h.shape
    if last:
        room = torch.full((B, H + 2, W, 15), 7.0, device=DEV, dtype=dtype)
        y = room[:, 1:1 + H, :, 3:13].movedim(-1, 1)
    else:
        room = torch.full((B, 15, H * W), 7.0, device=DEV, dtype=dtype)
        y = room[:, 3:13].unflatten(2, (H, W))
    got = binding.gated_forward(x, gw, uw, gb, ub, "gelu", h=y)[0]
    assert got is y and torch.equal(y, h)
    y.fill_(7.0)
    assert bool((room == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_weights_in_one_tensor(gpu_lib, dtype):
    """Both weights as halves or as columns of one matrix, at any address and any
    distance of their rows."""
    x, dh, *_ = make((37, 20), 24, dtype=dtype, seed=11)
    both = make((1, 40), 48, dtype=dtype, seed=12)[2]
    flat = make((1, 21), 60, dtype=dtype, seed=13)[2].flatten()
    pairs = [(both[:24, :20], both[24:, :20]), (both[::2, :20], both[::2, 20:]), (both[:24, 1:21], both[24:, 19:39]),
             (flat[1:481].view(24, 20), flat[502:982].view(24, 20)), (both[:24, :20], flat[:480].view(24, 20))]
    for gw, uw in pairs:
        check(x, dh, gw, uw, None, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("S,F", [(7, 900), (150, 700), (150, 12)])
def test_input_gradient_with_gaps(gpu_lib, S, F, layout, dtype):
    """dx with values between its rows and images, left as they were: in one piece, and
    joined from parts of a long sum."""
    B, C, last = 3, 20, layout == "last"
    x, dh, gw, uw, *_ = make((B, C, S, 1), F, layout, dtype, bias=False, seed=21)
    h, gate, up = binding.gated_forward(x, gw, uw, keep=False)
    row, image = (C + 3, S * (C + 3) + 5) if last else (S, C * S + 6)
    d = desc(B=B, C=C, F=F, S=S, layout=int(last), dtype=binding._dtype_codes()[dtype], dx=(image, row))
    flat = torch.full((B * image,), 3.0, dtype=dtype, device=DEV)
    ws = torch.empty(binding.oaa_gated_workspace_bytes(d, 1, 0), dtype=torch.uint8, device=DEV)
    binding.oaa_gated_backward(d, dh.data_ptr(), x.data_ptr(), gw.data_ptr(), uw.data_ptr(), None, None, None, None,
                               flat.data_ptr(), None, None, None, None, ws.data_ptr(), ws.numel(),
                               torch.cuda.current_stream().cuda_stream)
    got = flat.as_strided((B, S, C) if last else (B, C, S), (image, row, 1))
    b = Bounds(wide(x), wide(gw), wide(uw), None, None, "silu", dtype, wide(dh))
    near((got.movedim(-1, 1) if last else got)[..., None], b.grads[0], b.offs[0], dtype, "dx", 2 * F)
    got.fill_(3.0)
    assert bool((flat == 3.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_nothing_to_do(gpu_lib, layout):
    for shape in ((0, 6, 3, 2), (2, 6, 0, 4), (0, 6)):
        x, dh, gw, uw, gb, ub = make(shape, 10, layout, seed=1)
        h, gate, up = binding.gated_forward(x, gw, uw, gb, ub)
        assert h.shape == (shape[0], 10, *shape[2:])
        dx, *rest = binding.gated_backward(dh, x, gw, uw, gate, up)
        assert dx.shape == x.shape and all(bool((t == 0).all()) for t in rest)
    x, dh, gw, uw, gb, ub = make((2, 6, 3, 2), 10, layout, seed=1)
    h, gate, up = binding.gated_forward(x, gw, uw, gb, ub)
    assert binding.gated_backward(dh, x, gw, uw, gate, up, need_x=False, need_weights=False,
                                  need_biases=False) == (None,) * 5


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_gradients_one_at_a_time(gpu_lib, layout):
    x, dh, gw, uw, gb, ub = make((3, 40, 9, 8), 56, layout, torch.bfloat16, seed=15)
    h, gate, up = binding.gated_forward(x, gw, uw, gb, ub)
    full = binding.gated_backward(dh, x, gw, uw, gate, up)
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        got = binding.gated_backward(dh, x, gw, uw, gate, up, "silu", *need)
        for g, f, n in zip(got, full, (need[0], need[1], need[1], need[2], need[2])):
            assert torch.equal(g, f) if n else g is None


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_one_bad_value_reaches(gpu_lib, value, dtype, layout):
    """Its own position of h and dx; all others keep their bits, in tiles with edges
    in every direction."""
    for shape, F in (((2, 27, 9, 7), 71), ((2, 64, 16, 10), 96), ((70, 130), 40)):
        x, dh, gw, uw, gb, ub = make(shape, F, layout, dtype, seed=17)
        clean = binding.gated_forward(x, gw, uw, gb, ub)
        ref = binding.gated_backward(dh, x, gw, uw, *clean[1:])
        bad = x.clone()
        at = (1, shape[1] - 1) + (0,) * (len(shape) - 2)
        bad[at] = value
        h, gate, up = binding.gated_forward(bad, gw, uw, gb, ub)
        dx, dgw, duw, *_ = binding.gated_backward(dh, bad, gw, uw, gate, up)
        spot = torch.zeros((shape[0], 1, *shape[2:]), dtype=torch.bool, device=DEV)
        spot[(1, 0) + (0,) * (len(shape) - 2)] = True
        for got, good in ((h, clean[0]), (dx, ref[0])):
            spots = spot.expand(got.shape)
            assert torch.equal(got[~spots], good[~spots]) and not bool(torch.isfinite(got[spots]).all())
        assert bool(torch.isnan(dgw).any())
        if clean[1].dim() == 1:  # g and u are made again, from the bad value
            continue
        # with g, u and dh of that position fine, its channel of x is all that reaches dW
        dh0 = dh.clone().masked_fill_(spot.expand(dh.shape), 0.0)
        _, dgw, duw, *_ = binding.gated_backward(dh0, bad, gw, uw, *clean[1:])
        for g in (dgw, duw):
            assert bool(torch.isfinite(g[:, :-1]).all()) and bool(torch.isnan(g[:, -1]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_equal_calls_give_equal_bits(gpu_lib, layout):
    for shape, F, dtype in (((3, 48, 31, 20), 72, torch.bfloat16), ((1900, 80), 100, torch.float32)):
        args = make(shape, F, layout, dtype, seed=19)
        def both():
            h, gate, up = binding.gated_forward(args[0], *args[2:])
            return (h, gate, up, *binding.gated_backward(args[1], args[0], *args[2:4], gate, up))
        first = both()
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, both()))


@pytest.mark.gpu
def test_finite_differences(gpu_lib):
    """The derivative along a random direction of every argument: differences of h's
    float64 oracle, whose own error is about (1e-4)^2, against the gradients."""
    args = make((2, 12, 5, 4), 10, seed=21)
    x, dh, *params = args
    h, gate, up = binding.gated_forward(x, *params, activation="gelu")
    grads = binding.gated_backward(dh, x, *params[:2], gate, up, "gelu")
    rng = np.random.default_rng(22)
    values = [wide(t) for t in (x, *params)]
    for k, g in enumerate(grads):
        step = rng.standard_normal(values[k].shape)
        ends = []
        for sign in (1e-4, -1e-4):
            moved = list(values)
            moved[k] = values[k] + sign * step
            ends.append(float((oracle.gated_forward(*moved, activation="gelu") * wide(dh)).sum()))
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(slope - float((wide(g) * step).sum())) <= 1e-4 * float(np.abs(wide(g) * step).sum())


# ---- through autograd -----------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_autograd(gpu_lib, layout, dtype):
    x, dh, *params = make((2, 20, 9, 6), 28, layout, dtype, seed=23)
    plain = binding.gated_forward(x, *params)
    ref = binding.gated_backward(dh, x, *params[:2], *plain[1:])
    leaves = [t.requires_grad_() for t in (x, *params)]
    h = autograd.gated(*leaves)
    assert torch.equal(h, plain[0])
    for upstream in (dh, lay(dh, "planes"), lay(dh, "last")):
        for got, r in zip(torch.autograd.grad(h, leaves, upstream, retain_graph=True), ref):
            assert torch.equal(got, r)
    with torch.no_grad():
        assert torch.equal(autograd.gated(*leaves), plain[0])
    # one leaf at a time, and a gradient that is one number everywhere
    for k, leaf in enumerate(leaves):
        frozen = [t.detach() for t in leaves]
        frozen[k] = leaf
        (got,) = torch.autograd.grad(autograd.gated(*frozen), leaf, dh)
        assert torch.equal(got, ref[k])
    (got,) = torch.autograd.grad(autograd.gated(*leaves).sum(), leaves[:1])
    (r,) = binding.gated_backward(torch.ones_like(dh), x.detach(), *(p.detach() for p in params[:2]), *plain[1:])[:1]
    assert torch.equal(got, r)


@pytest.mark.gpu
def test_other_strides(gpu_lib):
    """Tensors that the direct calls refuse are laid out first."""
    x, dh, *params = make((2, 6, 8, 7), 10, seed=25)
    turned = x.transpose(2, 3).contiguous().transpose(2, 3)
    gw = params[0].t().contiguous().t()
    for call in (lambda: binding.gated_forward(turned, *params), lambda: binding.gated_forward(x, gw, *params[1:])):
        with pytest.raises(ValueError):
            call()
    ref = binding.gated_forward(x, *params)[0]
    assert torch.equal(autograd.gated(turned, gw, *params[1:]), ref)
    leaves = [t.requires_grad_() for t in (turned, gw)]
    h = autograd.gated(*leaves, *params[1:])
    grads = torch.autograd.grad(h, leaves, dh)
    assert torch.equal(h, ref) and grads[0].shape == x.shape and grads[1].shape == gw.shape


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["pinned", "pageable", "repacked"])
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_saved_tensors_elsewhere(gpu_lib, layout, how):
    x, dh, *params = make((3, 12, 11, 10), 20, layout, seed=27)
    leaves = [t.requires_grad_() for t in (x, *params)]
    ref = torch.autograd.grad(autograd.gated(*leaves), leaves, dh)

    def pack(t):
        room = torch.empty(t.numel() + 4, dtype=t.dtype, device=DEV)
        return room[4:].view(t.shape).copy_(t)

    hooks = {"pinned": lambda: torch.autograd.graph.save_on_cpu(pin_memory=True),
             "pageable": lambda: torch.autograd.graph.save_on_cpu(),
             "repacked": lambda: torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t)}[how]
    with hooks():
        h = autograd.gated(*leaves)
    got = torch.autograd.grad(h, leaves, dh)
    for g, r in zip(got, ref):
        # another layout sums in another order
        assert float((g - r).abs().max()) <= 3e-5 * float(r.abs().max())


@pytest.mark.gpu
def test_biases_of_any_strides(gpu_lib):
    """Columns of a matrix, and one value for all channels: with their gradients."""
    x, dh, gw, uw, gb, ub = make((70, 12), 40, seed=17)
    both = torch.stack((gb, ub), 1).requires_grad_()
    one = torch.full((1,), 0.25, device=DEV, requires_grad=True)
    h = autograd.gated(x, gw, uw, both[:, 0], both[:, 1])
    assert torch.equal(h, autograd.gated(x, gw, uw, gb, ub))
    (grad,) = torch.autograd.grad(h, both, dh)
    ref = binding.gated_backward(dh, x, gw, uw, *binding.gated_forward(x, gw, uw, gb, ub)[1:])[3:]
    assert torch.equal(grad, torch.stack(ref, 1))
    full = one.detach().repeat(40)
    h = autograd.gated(x, gw, uw, one.expand(40), ub)
    assert torch.equal(h, autograd.gated(x, gw, uw, full, ub))
    (grad,) = torch.autograd.grad(h, one, dh)
    ref = binding.gated_backward(dh, x, gw, uw, *binding.gated_forward(x, gw, uw, full, ub)[1:])[3]
    # torch adds the 40 values up in float32
    torch.testing.assert_close(grad[0].double(), ref.double().sum(), rtol=0, atol=40 * E * float(ref.abs().sum()))


@pytest.mark.gpu
def test_writes_are_seen(gpu_lib):
    """A saved tensor that changed before the backward pass is an error, not a wrong
    gradient; writing through h is announced."""
    x, dh, *params = make((4, 12), 20, seed=29)
    leaves = [t.requires_grad_() for t in (x, *params)]
    h = autograd.gated(*leaves)
    with torch.no_grad():
        leaves[1].mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        torch.autograd.grad(h, leaves, dh)
    out = torch.empty(4, 20, device=DEV)
    before = out._version
    binding.gated_forward(x.detach(), *(p.detach() for p in params), h=out)
    assert out._version == before + 1


@pytest.mark.gpu
def test_forward_mode_and_second_derivatives_are_refused(gpu_lib):
    x, dh, *params = make((4, 12), 20, seed=31)
    with forward_ad.dual_level():
        for k in range(5):
            args = [x, *params]
            args[k] = forward_ad.make_dual(args[k], torch.ones_like(args[k]))
            with pytest.raises(NotImplementedError):
                autograd.gated(*args)
    x.requires_grad_()
    (dx,) = torch.autograd.grad(autograd.gated(x, *params), x, dh.requires_grad_(), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.sum(), x)


@pytest.mark.gpu
def test_layer(gpu_lib):
    unit = autograd.GatedUnit(12, 20, activation="gelu", device=DEV)
    x, dh, *_ = make((2, 12, 5, 6), 20, seed=33)
    assert torch.equal(unit(x), binding.gated_forward(x, unit.gate_weight, unit.up_weight, unit.gate_bias, unit.up_bias,
                                                      "gelu")[0])
    assert len(list(autograd.GatedUnit(3, 4, bias=False, device=DEV, dtype=torch.bfloat16).parameters())) == 2
    with pytest.raises(ValueError, match="expected x"):
        unit(x[:, :11])
    with pytest.raises(ValueError, match="activation"):
        autograd.GatedUnit(3, 4, activation="tanh", device=DEV)


# ---- streams, graphs, large offsets ---------------------------------------------------

@pytest.mark.gpu
def test_another_stream(gpu_lib):
    args = make((2, 64, 40, 40), 96, seed=35)
    ref = binding.gated_forward(args[0], *args[2:])
    refs = binding.gated_backward(args[1], args[0], *args[2:4], *ref[1:])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            h, gate, up = binding.gated_forward(args[0], *args[2:])
            results.append((h, *binding.gated_backward(args[1], args[0], *args[2:4], gate, up)))
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(a, b) for a, b in zip(got, (ref[0], *refs)))


@pytest.mark.gpu
@pytest.mark.parametrize("shape,F,dtype", [((2, 27, 13, 11), 71, torch.bfloat16), ((300, 64), 96, torch.float32),
                                           ((3, 512), 700, torch.float16)], ids=str)
def test_graph_replays(gpu_lib, shape, F, dtype):
    """Both passes captured, replayed on other values with eager calls between."""
    x, dh, *params = make(shape, F, dtype=dtype, seed=37)
    leaves = [t.requires_grad_() for t in (x, *params)]

    def step():
        h = autograd.gated(*leaves)
        return (h, *torch.autograd.grad(h, leaves, dh))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        other = make(shape, F, dtype=dtype, seed=40 + k)
        with torch.no_grad():
            for t, v in zip((x, dh, *params), other):
                t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(out, step()):
            assert torch.equal(got, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("layout,shape,F", [("last", (16500, 24), 1900), ("planes", (40, 24, 12, 30), 300),
                                            ("last", (3, 40, 700, 9), 800), ("planes", (300, 16, 40, 26), 70)])
@pytest.mark.parametrize("k", [14, -20])
def test_range_of_float16_over_many_workgroups(gpu_lib, k, layout, shape, F):
    """The same where each workgroup takes several rows or tiles, by what some positions
    and some hidden channels need."""
    gen = torch.Generator(device=DEV).manual_seed(53)

    def normal(*size):
        return torch.randn(size, generator=gen, device=DEV)

    B, C = shape[:2]
    step = STEP[torch.float16]
    dh = lay((normal(B, F, *shape[2:]).clamp(-4.0, 4.0) * 2.0 ** (k - 1)).half(), layout)
    x0, gw0, uw0 = normal(*shape) * (4.0 if k > 0 else 1.0), *(normal(F, C) / C ** 0.5 for _ in range(2))
    T = x0.numel() // C
    some = torch.tensor(sorted({0, 1, T // 3, T // 2, T - 66, T - 2, T - 1}), device=DEV)
    few = torch.tensor([0, 1, 31, 63, F - 2, F - 1], device=DEV)

    def rows(t):
        return t.movedim(1, -1).reshape(T, -1)

    for wanted in ("dx", "weights"):
        far = 2.0 ** {("dx", 14): 8, ("dx", -20): -10, ("weights", 14): -14, ("weights", -20): 8}[wanted, k]
        x, gw, uw = lay((x0 * far).half(), layout), (gw0 / far).half(), (uw0 / far).half()
        d, W = (rows(dh)[some], (gw, uw)) if wanted == "dx" else (rows(dh)[:, few], (gw[few], uw[few]))
        v, d = wide(rows(x)[some] if wanted == "dx" else rows(x)), wide(d)
        W = [wide(w) for w in W]
        g, u = (v @ w.T for w in W)
        a, slope = _act("silu", g)
        D, V = np.abs(d), np.abs(v)
        og, ou = ((C + 8) * E * (V @ np.abs(w).T) for w in W)
        rg = D * (0.8 * og * (np.abs(u) + ou) + 1.2 * ou + 3e-6 * np.abs(u))
        ru = D * (1.2 * og + 2e-6 * np.abs(a) + 2e-7 * np.abs(g))
        whole = [(rows(x).double() @ w.double().t()) for w in (gw, uw)]
        s = torch.sigmoid(whole[0])
        y = rows(dh).double().abs()
        most = float(max((y * (whole[1] * s * (1 + whole[0] * (1 - s))).abs()).max(), (y * (whole[0] * s).abs()).max()))
        del whole, s, y
        assert most > 65504 if k > 0 else most < 2.0 ** -4
        rg, ru = (o + step * (np.abs(t) + o) + 2.0 ** -39 * most for o, t in ((rg, d * u * slope), (ru, d * a)))
        dg, du = d * u * slope, d * a
        if wanted == "dx":
            size = (np.abs(dg) + rg) @ np.abs(W[0]) + (np.abs(du) + ru) @ np.abs(W[1])
            refs = [dg @ W[0] + du @ W[1]]
            offs = [rg @ np.abs(W[0]) + ru @ np.abs(W[1]) + (2 * F + 8) * E * size]
        else:
            refs = [dg.T @ v, du.T @ v]
            offs = [r.T @ V + (T + 8) * E * ((np.abs(t) + r).T @ V) for r, t in ((rg, dg), (ru, du))]
        for grads in both_backwards(x, dh, gw, uw, None, None, "silu", [n in (("dx",) if wanted == "dx" else NAMES[1:3]) for n in NAMES]):
            got = [rows(grads[0])[some]] if wanted == "dx" else [t[few] for t in grads[1:3]]
            for t, ref, off in zip(got, refs, offs):
                assert 2.0 ** -12 < np.abs(ref).max() < 65504
                near(t, ref, off + step * (np.abs(ref) + off) + LEAST[torch.float16], torch.float16, wanted)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_replays_of_another_range(gpu_lib, layout):
    """Float16's dg and du in range, above and below it, from one replay to the next."""
    x, dh, *params = make((3, 40, 9, 8), 56, layout, torch.float16, seed=49)
    leaves = [t.requires_grad_() for t in (x, *params)]
    base = dh.clone()

    def step():
        h = autograd.gated(*leaves)
        return torch.autograd.grad(h, leaves, dh)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in (0, 17, 0, -12, 17, -12, 0):
        dh.copy_(base * 2.0 ** k)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(out, step()):
            assert bool(((got == ref) | (torch.isnan(got) & torch.isnan(ref))).all())
        # of a power of two the digits are the same, but for what lies among the smallest numbers
        if k == -12:
            for got, ref in zip(out, plain):
                ref = ref.float() * 2.0 ** k
                assert float((got.float() - ref).abs().max()) <= 2.0 ** -24 + 2.0 ** -8 * float(ref.abs().max())
        elif k == 0:
            plain = [t.clone() for t in out]


@pytest.mark.gpu
def test_many_small_images(gpu_lib):
    """More images than the limit of squares would allow one by one: the bits of their
    positions as tokens."""
    gen = torch.Generator(device=DEV).manual_seed(39)
    x, dh = (torch.randn((1 << 18, 2, n), generator=gen, device=DEV, dtype=torch.bfloat16).movedim(-1, 1)
             for n in (64, 2048))
    params = make((1, 64), 2048, dtype=torch.bfloat16, seed=39)[2:]

    def rows(t):
        return t.movedim(1, -1).reshape(-1, t.shape[1])

    h, *kept = binding.gated_forward(x, *params)
    got = (h, *binding.gated_backward(dh, x, *params[:2], *kept))
    ref, *kept = binding.gated_forward(rows(x), *params)
    refs = (ref, *binding.gated_backward(rows(dh), rows(x), *params[:2], *kept))
    for g, r in zip(got, refs):
        assert torch.equal(rows(g) if g.dim() == 3 else g, r)


@pytest.mark.gpu
def test_offsets_past_32_bits(gpu_lib):
    """h of 2^31 values and more, its last rows against the oracle."""
    T, C, F = (1 << 20) + 3, 16, 2056
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((T, C), generator=gen, device=DEV).bfloat16()
    gw, uw, gb, ub = make((1, C), F, dtype=torch.bfloat16, seed=41)[2:]
    h = binding.gated_forward(x, gw, uw, gb, ub, keep=False)[0]
    assert h.numel() > 1 << 31
    for rows in (slice(0, 5), slice(T // 2, T // 2 + 5), slice(T - 5, T)):
        b = Bounds(wide(x[rows]), wide(gw), wide(uw), wide(gb), wide(ub), "silu", torch.bfloat16)
        near(h[rows], b.h, b.h_off, torch.bfloat16, "h", C)
    del h
    # the backward pass, its gradients of the weights from a known sum
    few = 8
    h, gate, up = binding.gated_forward(x, gw[:few], uw[:few], None, None)
    dh = torch.zeros_like(h)
    dh[-1] = 1.0
    dx, dgw, duw, dgb, dub = binding.gated_backward(dh, x, gw[:few], uw[:few], gate, up)
    ref = oracle.gated_backward(wide(dh[-1:]), wide(x[-1:]), wide(gw[:few]), wide(uw[:few]))
    assert not bool(dx[:-1].any())
    for got, r in zip((dx[-1:], dgw, duw, dgb, dub), ref):
        assert np.abs(wide(got) - r).max() <= 2.0 ** -6 * np.abs(r).max()


@pytest.mark.gpu
@pytest.mark.parametrize("layout,B,C,S,F,dtype", [
    ("last", 1, 16, (1 << 20) + 3, 2056, torch.bfloat16),   # h, dh, g, u, dg and du
    ("last", 3, 2056, 349529, 16, torch.bfloat16),          # x and dx
    ("planes", 3, 16, (1 << 19) + 5, 1400, torch.float16),  # h, dh, g, u, dg and du; x is copied
    ("planes", 2, 1030, (1 << 20) + 4, 16, torch.bfloat16),  # x and dx
], ids=str)
def test_backward_past_32_bits(gpu_lib, layout, B, C, S, F, dtype):
    """Tensors of more than 2^31 values in both passes, g and u stored and made again. dh is 0
    but at the first, the last and some other positions, which are all that the gradients of the
    weights and biases then come from."""
    assert B * S * max(C, F) > 1 << 31
    print(layout, B, C, S, F, dtype, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(51)

    def tensor(make, n):
        return make((B, n, S)) if layout == "planes" else make((B, S, n)).movedim(-1, 1)

    x = tensor(lambda size: torch.randn(size, generator=gen, device=DEV, dtype=dtype), C)
    dh = tensor(lambda size: torch.zeros(size, device=DEV, dtype=dtype), F)
    gw, uw, gb, ub = make((1, C), F, dtype=dtype, seed=51)[2:]
    spots = [(b, s) for b in sorted({0, B - 1}) for s in (0, 1, S // 3, S - 65, S - 2, S - 1)]
    for b, s in spots:
        dh[b, :, s] = (torch.randn(F, generator=gen, device=DEV) * 0.1).to(dtype)

    def rows(t):
        return torch.stack([t[b, :, s] for b, s in spots])

    bounds = Bounds(wide(rows(x)), *map(wide, (gw, uw, gb, ub)), "silu", dtype, wide(rows(dh)))
    h = binding.gated_forward(x, gw, uw, gb, ub, keep=False)[0]
    near(rows(h), bounds.h, bounds.h_off, dtype, "h", C)
    del h
    terms = (2 * F, *[len(spots)] * 4)
    for dx, *rest in both_backwards(x, dh, gw, uw, gb, ub, "silu"):
        for name, got, ref, off, n in zip(NAMES, (rows(dx), *rest), bounds.grads, bounds.offs, terms):
            near(got, ref, off, dtype, name, n)
        for b, s in spots:
            dx[b, :, s] = 0.0
        assert not bool(dx.any())


# ---- refusals, without a GPU ----------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    import os

    from paper_1601_06815_amd import build
    if not os.path.exists(build.LIB_PATH):
        build.build()
    return binding.load()


def desc(**change):
    d = dict(B=2, C=6, F=10, S=10, layout=0, dtype=0, activation=2, gate_row=0, up_row=0, x=(0, 0), h=(0, 0), dh=(0, 0),
             dx=(0, 0))
    d.update(change)
    return binding.GatedDesc(*[binding.Strides(*v) if isinstance(v, tuple) else v for v in d.values()])


M = 1 << 20  # addresses far from each other; nothing is launched


def forward(d, x=M, gw=2 * M, uw=3 * M, gb=4 * M, ub=5 * M, h=6 * M, gate=7 * M, up=8 * M, ws=1 << 40, size=1 << 30):
    return binding.oaa_gated_forward(d, x, gw, uw, gb, ub, h, gate, up, ws, size, None)


def backward(d, dh=M, x=2 * M, gw=3 * M, uw=4 * M, gate=5 * M, up=6 * M, dx=7 * M, dgw=8 * M, duw=9 * M, dgb=10 * M,
             dub=11 * M, gb=12 * M, ub=13 * M, ws=1 << 40, size=1 << 30):
    return binding.oaa_gated_backward(d, dh, x, gw, uw, gb, ub, gate, up, dx, dgw, duw, dgb, dub, ws, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), 1), (dict(C=0), 1), (dict(F=0), 1), (dict(S=-1), 1), (dict(layout=2), 1), (dict(dtype=3), 1),
    (dict(activation=4), 1), (dict(gate_row=5), 1), (dict(up_row=-6), 1), (dict(x=(-1, 0)), 1), (dict(x=(0, -1)), 1),
    (dict(h=(9, 10)), 1), (dict(dx=(9, 10)), 1), (dict(layout=1, h=(100, 9)), 1), (dict(x=(60, 11)), 2),
    (dict(C=(1 << 20) + 1), 2), (dict(F=(1 << 20) + 1), 2), (dict(S=1 << 21), 2), (dict(B=1 << 30, S=2), 2),
    (dict(layout=1, S=1 << 31), 2), (dict(layout=1, S=1 << 30, F=1 << 10), 2), (dict(C=1 << 20, F=1 << 20), 2),
    (dict(gate_row=1 << 62), 2),
])
def test_refused_descriptions(lib, change, status):
    for call in (forward, backward):
        with pytest.raises(binding.OaaError) as e:
            call(desc(**change))
        assert e.value.status == status, e.value
    assert binding.oaa_gated_workspace_bytes(desc(**change), True, True) == 0


@pytest.mark.parametrize("change,match", [
    (dict(x=0), "x must"), (dict(gw=None), "gate_weight must"), (dict(uw=None), "up_weight must"), (dict(h=None), "h must"),
    (dict(gate=None), "together"), (dict(up=None), "together"), (dict(x=M + 2), "aligned"), (dict(gb=M + 1), "aligned"),
    (dict(h=M + 4), "h overlaps x"), (dict(h=M - 8), "h overlaps x"), (dict(h=2 * M + 4 * 59), "h overlaps gate_weight"),
    (dict(h=5 * M), "h overlaps up_bias"), (dict(gate=M + 4 * 119), "gate overlaps x"),
    (dict(up=7 * M + 796), "up overlaps gate"), (dict(gate=6 * M, up=9 * M), "gate overlaps h"),
])
def test_refused_forward_arguments(lib, change, match):
    with pytest.raises(binding.OaaError, match=match) as e:
        forward(desc(), **change)
    assert e.value.status == 1


@pytest.mark.parametrize("change,match", [
    (dict(dh=None), "dh must"), (dict(x=None), "x must"), (dict(gw=None), "gate_weight must"), (dict(gate=None), "together"),
    (dict(up=None), "together"), (dict(gate=None, up=None, dgw=None, duw=None, x=None), "x must"),
    (dict(gate=None, up=None, dx=None, uw=None), "up_weight must"), (dict(gate=None, up=None, dx=13 * M), "dx overlaps up_bias"),
    (dict(dgw=None), "together"), (dict(duw=None), "together"),
    (dict(dx=None, dgw=None, duw=None, dgb=None, dub=None), "all five"), (dict(dx=M), "dx overlaps dh"),
    (dict(dx=2 * M + 4), "dx overlaps x"), (dict(dgw=3 * M), "dgate_weight overlaps gate_weight"),
    (dict(duw=8 * M + 4 * 59), "dup_weight overlaps dgate_weight"), (dict(dgb=6 * M + 796), "dgate_bias overlaps up"),
    (dict(dub=10 * M), "dup_bias overlaps dgate_bias"), (dict(dub=10 * M + 2), "aligned"),
])
def test_refused_backward_arguments(lib, change, match):
    with pytest.raises(binding.OaaError, match=match) as e:
        backward(desc(), **change)
    assert e.value.status == 1


def test_refused_workspaces(lib):
    d = desc()
    need = binding.oaa_gated_workspace_bytes(d, True, False)
    assert need % 256 == 0 and need >= 2 * 4 * 200
    for ws, size, status in ((None, 0, 3), (1 << 40, 2 * 4 * 200 - 1, 3), ((1 << 40) + 8, need, 1)):
        with pytest.raises(binding.OaaError) as e:
            backward(d, ws=ws, size=size)
        assert e.value.status == status
    # float32 is read in place; 16 bits with rows of odd length, or at odd addresses, are not
    assert binding.oaa_gated_workspace_bytes(d, False, True) == 0
    assert binding.oaa_gated_workspace_bytes(desc(dtype=1), False, False) == 0
    assert binding.oaa_gated_workspace_bytes(desc(dtype=1, S=20), False, True) > 0
    assert binding.oaa_gated_workspace_bytes(desc(dtype=1, C=7, S=20), False, False) > 0
    with pytest.raises(binding.OaaError) as e:
        forward(desc(dtype=2), x=M + 2, ws=None, size=0)
    assert e.value.status == 3


def test_size_of_images_that_follow_each_other(lib):
    """Positions are counted as they run: evenly spaced, those of all images are one's."""
    sizes = dict(layout=1, dtype=1, C=64, F=2048)
    many, one = desc(B=1 << 18, S=2, **sizes), desc(B=1, S=1 << 19, **sizes)
    need = binding.oaa_gated_workspace_bytes(many, True, False)
    assert need == binding.oaa_gated_workspace_bytes(one, True, False) > 4 * 2048 << 19
    assert binding.oaa_gated_keeps(many) == binding.oaa_gated_keeps(one)
    with pytest.raises(binding.OaaError) as e:
        backward(many, dh=1 << 40, x=1 << 44, dx=1 << 45, gate=None, up=None, ws=None, size=0)
    assert e.value.status == 3, e.value
    # 16-bit rows of odd length are copied
    assert binding.oaa_gated_workspace_bytes(desc(B=1 << 18, S=2, layout=1, dtype=1, C=63, F=2048), False, False) > 64 << 19
    # gaps between the images of a tensor that the pass reads or writes: each is one
    gaps = (2 * 2048 + 8, 2048)
    for change, back, fits in ((dict(x=(136, 64)), False, False), (dict(h=gaps), False, False), (dict(h=gaps), True, True),
                               (dict(dh=gaps), True, False), (dict(dx=(136, 64)), True, False), (dict(dh=gaps), False, True)):
        d = desc(B=1 << 18, S=2, **sizes, **change)
        if back:
            assert (binding.oaa_gated_workspace_bytes(d, True, False) > 0) == fits
        with pytest.raises(binding.OaaError) as e:
            if back:
                backward(d, dh=1 << 40, x=1 << 44, dx=1 << 45, gate=None, up=None, ws=None, size=0)
            else:
                forward(d, x=1 << 40, gw=None, h=1 << 45, gate=None, up=None)
        assert e.value.status == ((3 if back else 1) if fits else 2), e.value


def test_slices_beside_each_other(lib):
    """x and h as columns of one tensor pass the check of overlaps (and then fail for
    want of a workspace); one column in common does not."""
    for layout, strides, width in ((0, (320, 20), 100), (1, (320, 16), 5)):
        d = desc(layout=layout, dtype=1, C=5, S=20, x=strides, h=strides)
        x = M + 2
        with pytest.raises(binding.OaaError) as e:
            forward(d, x=x, h=x + 2 * width, ws=None, size=0)
        assert e.value.status == 3
        for h in (x + 2 * width - 2, x + 2):
            with pytest.raises(binding.OaaError, match="h overlaps x"):
                forward(d, x=x, h=h)


def test_refused_tensors(lib):
    """The checks of the torch wrapper, on descriptions alone."""
    t = torch.float32
    weights = ((t, (10, 6), (6, 1)), (t, (10, 6), (6, 1)))
    good = ((2, 6, 4), (24, 4, 1), t, weights, (None, None), None, None, "silu")
    assert binding._GatedCall(*good).out_shape == (2, 10, 4)
    for k, v, match in [(2, torch.float64, "x must"), (7, "tanh", "activation"), (1, (48, 8, 2), "planes or channels"),
                        (3, (weights[0], (t, (10, 5), (5, 1))), "up_weight"), (3, (weights[0], (t, (9, 6), (6, 1))), "up_weight"),
                        (3, ((torch.float16, (10, 6), (6, 1)), weights[1]), "gate_weight"),
                        (3, ((t, (6,), (1,)), weights[1]), "gate_weight"), (3, ((t, (10, 6), (1, 10)), weights[1]), "strides"),
                        (3, ((t, (10, 6), (5, 1)), weights[1]), "strides"),
                        (4, ((t, (9,)), None), "gate_bias"), (4, (None, (torch.float16, (10,))), "up_bias"),
                        (5, (40, 1, 10), "h"), (6, (40, 1, 10), "dh")]:
        args = list(good)
        args[k] = v
        with pytest.raises(ValueError, match=match):
            binding._GatedCall(*args)
    with pytest.raises(ValueError, match="on the GPU"):
        binding.gated_forward(torch.zeros(2, 6), torch.zeros(10, 6), torch.zeros(10, 6))
    assert ctypes.sizeof(binding.GatedDesc) == 120


def test_oracle_matches_autograd():
    """The oracle against torch's float64 operations and their derivatives."""
    gen = torch.Generator().manual_seed(3)
    x, gw, uw, gb, ub, dh = (torch.randn(s, generator=gen, dtype=torch.float64, requires_grad=True)
                             for s in ((2, 5, 3, 4), (7, 5), (7, 5), (7,), (7,), (2, 7, 3, 4)))
    acts = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
    for name, f in acts.items():
        rows = x.movedim(1, -1)
        h = (f(rows @ gw.t() + gb) * (rows @ uw.t() + ub)).movedim(-1, 1)
        values = [t.detach().numpy() for t in (x, gw, uw, gb, ub)]
        assert np.allclose(h.detach().numpy(), oracle.gated_forward(*values, activation=name), atol=1e-12)
        refs = torch.autograd.grad(h, (x, gw, uw, gb, ub), dh)
        for r, o in zip(refs, oracle.gated_backward(dh.detach().numpy(), *values, activation=name)):
            assert np.allclose(r.numpy(), o, atol=1e-10)
