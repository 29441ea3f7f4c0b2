"""Dropout through the public calls, against the fp64 oracle with the generator's
own mask.

The mask is exact. A kept value is multiplied by 1 / (1 - p), a float32 (half a step
of it, 2^-24, and another for the product), added to the residual (2^-24 of the
sum) and rounded to its type (half a step): a value may be off by 3 2^-24 of the two
terms' magnitudes and half a step of the result.
"""

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from oracle import block as oracle
from paper_1601_06815_amd import autograd, binding

DEV = "cuda:0"
STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
F32, BF16, F16 = TYPES = [torch.float32, torch.bfloat16, torch.float16]
PAIRS = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32), (F32, BF16), (F32, F16)]
SEED = (-0x123456789ABCDEF0, 0x1FEDCBA987654321)


def wide(t):
    return None if t is None else t.detach().cpu().double().numpy()


def lay(t, layout):
    return t.contiguous() if layout == "planes" else t.movedim(1, -1).contiguous().movedim(-1, 1)


def seed_of(key=SEED[0], call=SEED[1]):
    return torch.tensor([key, call], dtype=torch.int64, device=DEV)


def make(shape, layout="planes", dtype=F32, seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    return lay(torch.from_numpy(rng.standard_normal(shape) * scale).to(DEV, dtype), layout)


def near(y, x, p, seed, residual, layout):
    ref = oracle.dropout(wide(x), p, seed, wide(residual), layout)
    terms = np.abs(wide(x)) / (1.0 - p if p < 1.0 else 1.0) + (0 if residual is None else np.abs(wide(residual)))
    bound = 3 * 2.0 ** -24 * terms * (1 + STEP[y.dtype]) + STEP[y.dtype] * np.abs(ref) + LEAST[y.dtype]
    off = np.abs(wide(y) - ref)
    assert np.all(off <= bound), (float(np.max(off / bound)), np.unravel_index(np.argmax(off / bound), off.shape))
    return oracle.dropout_mask(x.shape, p, seed, layout)


def check(x, p, residual=None, dtype=None, layout="planes", seed=SEED, y=None):
    got = binding.dropout(x, p, seed_of(*seed), residual, y=y, dtype=dtype)
    kept = near(got, x, p, seed, residual, layout)
    if residual is None:
        assert not wide(got)[~kept].any()
    return got


SHAPES = [(1, 1), (1, 3), (5, 1), (2, 7), (1, 4, 28, 28), (3, 27, 13, 11), (5, 6, 1, 1), (1000, 33), (2, 64, 40, 41),
          (1, 5, 3, 1, 7), (4, 2048), (300, 1027), (7, 96, 52, 52)]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(gpu_lib, shape, layout):
    print(shape, layout, flush=True)
    i = SHAPES.index(shape)
    for k in range(3):
        tx, ty = PAIRS[(2 * i + 3 * k) % len(PAIRS)]
        x = make(shape, layout, tx, i)
        check(x, (0.1, 0.5, 0.9)[k], None, ty, layout)
        y = check(x, 0.25, make(shape, layout, ty, i + 50), None, layout)
        if np.prod(shape[2:]) > 1 and shape[1] > 1:
            assert y.stride() == x.stride()


@pytest.mark.gpu
@pytest.mark.parametrize("tx,ty", PAIRS, ids=str)
@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 1e-6, 0.3, 0.999, 1.0 - 2.0 ** -40, 1.0])
def test_types_and_probabilities(gpu_lib, p, tx, ty):
    x = make((3, 5, 77), "planes", tx, 1)
    if p > 0.9999999:  # 1 / (1 - p) of nothing that is kept
        y = binding.dropout(x, p, seed_of(), dtype=ty)
        assert not bool(y.any())
        r = make((3, 5, 77), "planes", ty, 2)
        assert torch.equal(binding.dropout(x, p, seed_of(), r), r)
        return
    check(x, p, None, ty)
    check(x, p, make((3, 5, 77), "planes", ty, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("seed", [(0, 0), (-1, -1), (1 << 62, 5), (7, -(1 << 63)), ((1 << 32) + 3, 1 << 32)], ids=str)
def test_seeds(gpu_lib, seed):
    """Every bit of key and call counts."""
    x = make((3, 1001), seed=3)
    y = check(x, 0.5, seed=seed)
    for other in ((seed[0] ^ 1, seed[1]), (seed[0] ^ (1 << 40), seed[1]), (seed[0], seed[1] ^ 1), (seed[0], seed[1] ^ (1 << 40))):
        differ = float(((check(x, 0.5, seed=other) == 0) != (y == 0)).double().mean())
        assert abs(differ - 0.5) < 5 * 0.5 / np.sqrt(3003)


@pytest.mark.gpu
@pytest.mark.parametrize("tx,ty", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16)], ids=str)
@pytest.mark.parametrize("view", ["channels", "channels last", "rows last", "images", "one image many times", "odd address",
                                  "images between rows"])
def test_strided_tensors(gpu_lib, view, tx, ty):
    """Slices have the mask of a dense tensor; one in place of the output leaves what
    is around it."""
    layout = "last" if "last" in view or "rows" in view else "planes"
    cut = {"channels": lambda t: t[:, 3:9], "channels last": lambda t: t[:, 3:9], "rows last": lambda t: t[:, :6, 2:6],
           "images": lambda t: t[::2, :6], "one image many times": lambda t: t[:1, :6].expand(3, 6, 9, 7),
           "odd address": lambda t: t.flatten()[1:1 + 2 * 6 * 63].view(2, 6, 9, 7),
           "images between rows": lambda t: t.movedim(1, -1).reshape(-1)[:9 * 7 * 4 * 12].view(63, 4, 12)[:, :, 1:7].permute(1, 2, 0)}[view]
    x = cut(make((4, 12, 9, 7), layout, tx, 5))
    r = cut(make((4, 12, 9, 7), layout, ty, 6))
    check(x, 0.3, None, ty, layout)
    ref = check(x, 0.3, r, None, layout)
    check(x, 0.3, lay(r, layout), None, layout)
    if "many times" in view:
        return
    room = torch.full((4, 12, 9, 7), 7.0, device=DEV, dtype=ty)
    room = lay(room, layout)
    y = cut(room)
    got = check(x, 0.3, r, None, layout, y=y)
    assert got is y and torch.equal(y, ref)
    y.fill_(7.0)
    assert bool((room == 7.0).all())


@pytest.mark.gpu
def test_in_place(gpu_lib):
    x, r = make((3, 40, 11), seed=7), make((3, 40, 11), seed=8)
    ref = binding.dropout(x, 0.4, seed_of(), r)
    for target in (x.clone(), r.clone()):
        args = (target, r) if target.equal(x) else (x, target)
        version = target._version
        assert torch.equal(binding.dropout(args[0], 0.4, seed_of(), args[1], y=target), ref)
        assert target._version == version + 1


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_dropped_values_are_gone(gpu_lib, layout):
    """NaN and infinities where x is dropped do not come through; kept ones do."""
    for shape in ((2, 6, 5, 4), (3, 4, 1001)):
        x = make(shape, layout, seed=9)
        kept = torch.from_numpy(oracle.dropout_mask(shape, 0.5, SEED, layout)).to(DEV)
        clean = binding.dropout(x, 0.5, seed_of(), x)
        for value in (float("nan"), float("inf")):
            assert torch.equal(binding.dropout(lay(x.masked_fill(~kept, value), layout), 0.5, seed_of(), x), clean)
            assert not bool(torch.isfinite(binding.dropout(lay(x.masked_fill(kept, value), layout), 0.5, seed_of())[kept]).any())


@pytest.mark.gpu
def test_nothing_to_do(gpu_lib):
    for shape in ((0, 4), (2, 3, 0), (0, 3, 5)):
        x = torch.empty(shape, device=DEV)
        assert binding.dropout(x, 0.5, seed_of(), x).shape == x.shape


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_share_of_kept_values(gpu_lib, p):
    """Five deviations of a binomial count, in every quarter of a counter and in every
    one of 16 stretches; neighbours are independent."""
    n = 1 << 22
    kept = (binding.dropout(torch.ones((1, n), device=DEV), p, seed_of()) != 0).reshape(-1).double()
    for part in [kept[k::4] for k in range(4)] + list(kept.split(n // 16)):
        share = 5 * np.sqrt(p * (1 - p) / part.numel())
        assert abs(float(part.mean()) - (1 - p)) < share
    both = float((kept[1:] * kept[:-1]).mean())
    assert abs(both - (1 - p) ** 2) < 5 * np.sqrt(3 * p / n)


@pytest.mark.gpu
def test_offsets_past_32_bits(gpu_lib):
    """2^31 elements and more: the index of the mask and the addresses."""
    n = (1 << 31) + 4096 + 5
    for dtype, shape in ((BF16, (1, 1, n)), (BF16, (n // 64, 64))):
        x = torch.ones(shape, dtype=dtype, device=DEV)
        if shape[1] == 64:  # rows apart: the strided kernel
            x = torch.ones((shape[0], 65), dtype=dtype, device=DEV)[:, :64]
        y = binding.dropout(x, 0.5, seed_of())
        m = x.numel()
        for start in (0, (1 << 31) - 8, (m - 4000) // 64 * 64):
            count = min(4000, m - start) // 64 * 64
            words = oracle.dropout_words(count, SEED, start)
            got = y.reshape(-1)[start:start + count].cpu().double().numpy()
            assert np.array_equal(got, np.where(words >= 1 << 31, 2.0, 0.0))
        del x, y


# ---- through autograd -----------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("tx,ty", PAIRS[:5], ids=str)
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_autograd(gpu_lib, layout, tx, ty):
    x, r = make((2, 20, 9, 6), layout, tx, 11), make((2, 20, 9, 6), layout, ty, 12)
    dy = make((2, 20, 9, 6), layout, ty, 13)
    x.requires_grad_()
    r.requires_grad_()
    seed = seed_of()
    y = autograd.dropout(x, 0.3, seed, r)
    near(y, x, 0.3, SEED, r, layout)
    for upstream in (dy, lay(dy, "planes"), lay(dy, "last")):
        dx, dr = torch.autograd.grad(y, (x, r), upstream, retain_graph=True)
        assert dx.dtype == tx and torch.equal(dr, upstream)
        near(dx, upstream, 0.3, SEED, None, layout)
    (dx,) = torch.autograd.grad(y.sum(), x)
    near(dx, torch.ones_like(dy), 0.3, SEED, None, layout)
    with torch.no_grad():
        assert torch.equal(autograd.dropout(x, 0.3, seed, lay(r, "planes")), y)
    for leaf, args in ((x, (x, r.detach())), (r, (x.detach(), r))):
        y = autograd.dropout(args[0], 0.3, seed, args[1])
        torch.autograd.grad(y, leaf, dy)


@pytest.mark.gpu
def test_gradient_by_differences(gpu_lib):
    """y is linear in x: differences are exact up to rounding."""
    x, d = make((3, 50), seed=15), make((3, 50), seed=16)
    x.requires_grad_()
    y = autograd.dropout(x, 0.4, seed_of())
    (dx,) = torch.autograd.grad(y, x, d)
    t = make((3, 50), seed=17)
    moved = autograd.dropout((x + t).detach(), 0.4, seed_of())
    change = ((moved - y.detach()).double() * d.double()).sum()
    assert abs(float(change - (dx.double() * t.double()).sum())) <= 150 * 2.0 ** -22 * 30


@pytest.mark.gpu
def test_seed_that_changed(gpu_lib):
    """The seed of a call is part of its gradient: changed in between it is refused."""
    x = make((3, 50), seed=18).requires_grad_()
    state = seed_of()
    y = autograd.dropout(x, 0.4, state)
    binding.dropout_next(state)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


@pytest.mark.gpu
def test_layer_between_modes(gpu_lib):
    """The gradient of a call in evaluation mode, after the layer has trained on."""
    layer = autograd.Dropout(0.5, seed=3, device=DEV).eval()
    x, r = (make((4, 6), seed=n).requires_grad_() for n in (1, 2))
    y = layer(x, r)
    layer.train()
    layer(x.detach())
    dy = make((4, 6), seed=5)
    dx, dr = torch.autograd.grad(y, (x, r), dy)
    assert torch.equal(dx, dy) and torch.equal(dr, dy) and torch.equal(y, x + r)


@pytest.mark.gpu
def test_forward_mode_is_refused(gpu_lib):
    x = make((3, 50), seed=19)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for args in ((dual, 0.3, seed_of()), (x, 0.3, seed_of(), dual)):
            with pytest.raises(NotImplementedError):
                autograd.dropout(*args)


@pytest.mark.gpu
def test_layer(gpu_lib):
    layer = autograd.Dropout(0.4, seed=5, device=DEV)
    x, r = make((3, 400), seed=20), make((3, 400), seed=21)
    for call in range(3):
        y = layer(x, r)
        near(y, x, 0.4, (5, call), r, "planes")
        assert layer.state.tolist() == [5, call + 1]
    layer.eval()
    assert layer(x) is x and torch.equal(layer(x, r), x + r) and layer.state.tolist() == [5, 3]
    assert torch.equal(autograd.Dropout(0.0, device=DEV)(x), x)
    other = autograd.Dropout(0.4, device=DEV)
    other.load_state_dict(layer.state_dict())
    near(other(x), x, 0.4, (5, 3), None, "planes")
    with pytest.raises(ValueError, match="probability"):
        autograd.Dropout(1.5, device=DEV)


@pytest.mark.gpu
def test_graph_replays_draw_new_masks(gpu_lib):
    """A captured layer advances its state at each replay, and its gradient has that
    replay's mask."""
    layer = autograd.Dropout(0.5, seed=9, device=DEV)
    x = make((4, 1000), seed=22).requires_grad_()

    def step():
        y = layer(x)
        return y, torch.autograd.grad(y, x, torch.ones_like(y))[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = step()
    for call in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        near(y, x, 0.5, (9, call), None, "planes")
        near(dx, torch.ones_like(x), 0.5, (9, call), None, "planes")
        eager = binding.dropout(x.detach(), 0.5, seed_of(9, call))
        assert torch.equal(eager, y)
    assert layer.state.tolist() == [9, 5]


@pytest.mark.gpu
def test_another_stream(gpu_lib):
    x = make((40, 3001), seed=23)
    ref = binding.dropout(x, 0.5, seed_of())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = binding.dropout(x, 0.5, seed_of())
    s.synchronize()
    assert torch.equal(got, ref)


# ---- refusals and the generator, without a GPU ----------------------------------------

@pytest.fixture(scope="module")
def lib():
    import os

    from paper_1601_06815_amd import build
    if not os.path.exists(build.LIB_PATH):
        build.build()
    return binding.load()


def desc(**change):
    d = dict(B=2, C=6, S=10, layout=0, x_dtype=0, y_dtype=0, x=(0, 0), residual=(0, 0), y=(0, 0))
    d.update(change)
    return binding.DropoutDesc(*[binding.Strides(*v) if isinstance(v, tuple) else v for v in d.values()])


M = 1 << 20


def call(d, x=M, residual=2 * M, y=3 * M, p=0.5, seed=4 * M):
    return binding.oaa_dropout(d, x, residual, y, p, seed, None)


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), 1), (dict(C=0), 1), (dict(S=-1), 1), (dict(layout=2), 1), (dict(x_dtype=3), 1), (dict(y_dtype=-1), 1),
    (dict(x_dtype=1, y_dtype=2), 1), (dict(x=(-1, 0)), 1), (dict(y=(9, 10)), 1), (dict(layout=1, y=(100, 5)), 1),
    (dict(residual=(60, 11)), 2), (dict(S=1 << 34), 2), (dict(B=1 << 30, S=1 << 5), 2),
])
def test_refused_descriptions(lib, change, status):
    with pytest.raises(binding.OaaError) as e:
        call(desc(**change))
    assert e.value.status == status, e.value


@pytest.mark.parametrize("change,match", [
    (dict(x=None), "x and y"), (dict(y=None), "x and y"), (dict(seed=None), "seed must"), (dict(seed=M + 4), "seed must"),
    (dict(p=-0.1), "probability"), (dict(p=1.1), "probability"), (dict(p=float("nan")), "probability"),
    (dict(x=M + 2), "aligned"), (dict(y=M + 4), "y overlaps x"), (dict(y=M - 4 * 119), "y overlaps x"),
    (dict(y=2 * M + 4), "y overlaps residual"),
])
def test_refused_arguments(lib, change, match):
    with pytest.raises(binding.OaaError, match=match) as e:
        call(desc(), **change)
    assert e.value.status == 1


def test_refused_overlaps_of_types(lib):
    for change in (dict(y=M), dict(y=M + 236), dict(y=M - 476)):
        with pytest.raises(binding.OaaError, match="y overlaps x"):
            call(desc(x_dtype=1), **change)
    for state, used in ((None, M), (M, None), (M, M), (M, M + 8), (M, M - 8), (M + 4, 2 * M)):
        with pytest.raises(binding.OaaError):
            binding.oaa_dropout_next(state, used, None)


def test_refused_tensors(lib):
    t = torch.float32
    good = ((2, 6, 4), (24, 4, 1), t, (t, (24, 4, 1)), t, None)
    binding._DropoutCall(*good)
    for k, v, match in [(2, torch.float64, "x must"), (4, torch.int32, "y must"), (3, (torch.float16, (24, 4, 1)), "residual"),
                        (3, (t, (24, 1, 6)), "residual"), (5, (24, 1, 6), "y"), (1, (48, 8, 2), "planes or channels")]:
        args = list(good)
        args[k] = v
        with pytest.raises(ValueError, match=match):
            binding._DropoutCall(*args)
    with pytest.raises(ValueError, match="on the GPU"):
        binding.dropout(torch.zeros(2, 6), 0.5, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="on the GPU"):
        binding.dropout_next(torch.zeros(2, dtype=torch.int64))


def test_generator():
    """The published known answers of Philox4x32-10: all words 0, all ones, digits of pi."""
    pi = [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]
    for counter, key, words in (
            ([0] * 4, (0, 0), [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
            ([0xFFFFFFFF] * 4, (0xFFFFFFFF, 0xFFFFFFFF), [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
            (pi, (0xA4093822, 0x299F31D0), [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert oracle.philox([counter], key)[0].tolist() == words


def test_generator_of_the_library(tmp_path):
    """csrc/philox.hpp, compiled for the host, against the oracle."""
    import shutil
    import subprocess

    from paper_1601_06815_amd import build
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text("#define __host__\n#define __device__\n#define __forceinline__ inline\n")
    (tmp_path / "t.cpp").write_text(
        '#include "philox.hpp"\n#include <cstdio>\n'
        'int main() { unsigned long long at, call, key;\n'
        '  while (std::scanf("%llu%llu%llu", &at, &call, &key) == 3) {\n'
        '    const oaa::Words w = oaa::philox(at, call, key);\n'
        '    std::printf("%u %u %u %u\\n", w.w[0], w.w[1], w.w[2], w.w[3]); } }\n')
    subprocess.run([cxx, "-std=c++17", "-I", str(tmp_path), "-I", build.CSRC, str(tmp_path / "t.cpp"), "-o",
                    str(tmp_path / "t")], check=True)
    rng = np.random.default_rng(3)
    lines = rng.integers(0, 2 ** 64, (200, 3), dtype=np.uint64, endpoint=False)
    out = subprocess.run([str(tmp_path / "t")], input="\n".join(" ".join(map(str, v)) for v in lines),
                         capture_output=True, text=True, check=True).stdout.split("\n")
    for (at, c, key), line in zip(lines.tolist(), out):
        counter = [at & 0xFFFFFFFF, at >> 32, c & 0xFFFFFFFF, c >> 32]
        assert [int(v) for v in line.split()] == oracle.philox([counter], (key & 0xFFFFFFFF, key >> 32))[0].tolist()
