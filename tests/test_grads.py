"""The norm of many gradients and clipping by it, through the public calls,
against the fp64 oracle.

Sums are held in 64 bits, so the float32 norm is within two of its roundings of
the exact one (2e-7); a clipped value adds the coefficient's roundings and its
own: 4e-7 in float32, half a step in 16 bits.
"""

import numpy as np
import pytest
import torch

from oracle import norm as oracle
from paper_1601_06815_amd import autograd, binding

DEV = "cuda:0"
INF = float("inf")
STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def wide(t):
    return t.detach().cpu().double().numpy()


def make(sizes, types=TYPES, seed=0):
    """One tensor a size, the types in turn, each at a magnitude of its own."""
    rng = np.random.default_rng(seed)
    out = []
    for i, n in enumerate(sizes):
        a = rng.standard_normal(n if isinstance(n, tuple) else (n,)).astype(np.float32) * 0.01 * 2.0 ** (i % 5)
        out.append(torch.from_numpy(a).to(DEV, types[i % len(types)]))
    return out


def check(grads, max_norm, p=2.0, out=None, in_place=False):
    ref_norm, refs = oracle.grad_clip([wide(g) for g in grads], max_norm, p)
    norm = binding.grad_norm(grads, p)
    targets = [torch.empty_like(g) for g in grads] if not in_place else [g.clone() for g in grads]
    clipped = binding.grad_clip(targets if in_place else grads, max_norm, p, out=None if in_place else targets)
    torch.cuda.synchronize()
    for got in (norm, clipped):
        assert got.shape == () and got.dtype == torch.float32
        assert abs(float(got) - ref_norm) <= 2e-7 * ref_norm, (float(got), ref_norm)
    for t, r in zip(targets, refs):
        off = np.abs(wide(t) - r)
        assert np.all(off <= 4e-7 * np.abs(r) + STEP[t.dtype] * np.abs(r) * 1.001 + LEAST[t.dtype])
    return targets


LISTS = [
    [1], [300, 4, 4], [0], [0, 5, 0, 0, 7], [16384], [16385, 1], [16383, 16384, 3], [100003, 7, 65536, 1],
    [(8, 3, 7, 7), 8, 8] * 5, [17] * 300, [40000] * 130, [3000000, 1, 5], [1 << 20] * 9, [25000000, 7],
]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("p", [1.0, 2.0, INF])
def test_norm_and_clip(gpu_lib, sizes, p):
    print(len(sizes), sizes[0], p, flush=True)
    grads = make(sizes, seed=len(sizes))
    size = oracle.grad_norm([wide(g) for g in grads], p)
    check(grads, 0.3 * size, p)
    check(grads, 0.3 * size, p, in_place=True)
    check(grads, 2 * size + 1, p)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("count", [5, 20000, 700001])
def test_types_and_odd_addresses(gpu_lib, dtype, count):
    """Tensors that start at any element."""
    whole = make([count + 16], [dtype], seed=3)[0]
    for start in (1, 3, 8):
        view = whole[start:start + count]
        room = torch.full((count + 16,), 3.0, device=DEV, dtype=dtype)
        norm = binding.grad_clip([view], 0.01, out=[room[start + 1:start + 1 + count]])
        ref_norm, (ref,) = oracle.grad_clip([wide(view)], 0.01)
        assert abs(float(norm) - ref_norm) <= 2e-7 * ref_norm
        got = wide(room)
        assert np.all(got[:start + 1] == 3.0) and np.all(got[start + 1 + count:] == 3.0)
        off = np.abs(got[start + 1:start + 1 + count] - ref)
        assert np.all(off <= 4e-7 * np.abs(ref) + STEP[dtype] * np.abs(ref) * 1.001 + LEAST[dtype])


@pytest.mark.gpu
def test_no_tensors(gpu_lib):
    assert float(binding.grad_norm([])) == 0.0 and float(binding.grad_clip([], 1.0)) == 0.0
    assert float(autograd.clip_grad_norm_([torch.nn.Parameter(torch.ones(3, device=DEV))], 1.0)) == 0.0


@pytest.mark.gpu
def test_nothing_is_scaled_below_the_bound(gpu_lib):
    """k = 1: copies are exact, and in place every bit stays, also where a
    product would change it (a NaN's payload is not looked at)."""
    for sizes in ([7, 300], [100000, 3]):
        grads = make(sizes, seed=5)
        before = [g.clone() for g in grads]
        out = [torch.empty_like(g) for g in grads]
        binding.grad_clip(grads, 1e9, out=out)
        binding.grad_clip(grads, 1e9)
        assert all(torch.equal(a, b) and torch.equal(a, o) for a, b, o in zip(grads, before, out))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[50, 60], [50000, 60, 70000]], ids=str)
@pytest.mark.parametrize("p", [1.0, 2.0, INF])
def test_values_that_are_not_finite(gpu_lib, sizes, p):
    for value in (float("nan"), INF, -INF):
        grads = make(sizes, [torch.float32], seed=7)
        grads[0][-1] = value
        out = [torch.empty_like(g) for g in grads]
        norm = float(binding.grad_clip(grads, 1.0, p, out=out))
        if np.isnan(value):
            assert np.isnan(norm) and np.isnan(float(binding.grad_norm(grads, p)))
            assert all(bool(torch.isnan(o).all()) for o in out)
        else:
            assert norm == INF and float(binding.grad_norm(grads, p)) == INF
            assert bool(torch.isnan(out[0][-1])) and bool((out[0][:-1] == 0).all()) and bool((out[1] == 0).all())
        # both at once: the NaN shows
        grads[1][3] = INF if np.isnan(value) else float("nan")
        assert np.isnan(float(binding.grad_norm(grads, p)))


@pytest.mark.gpu
@pytest.mark.parametrize("value", [3e38, 1e25, 1e-25, 1e-44])
def test_range_of_float32(gpu_lib, value):
    """Squares far beyond float32 on either side."""
    g = torch.full((1000,), value, device=DEV)
    exact = float(g[0].double()) * np.sqrt(1000.0)
    got = float(binding.grad_norm([g]))
    assert got == INF if exact > 3.4028235e38 else abs(got - exact) <= max(2e-7 * exact, 2.0 ** -149)


@pytest.mark.gpu
def test_orders_of_dimensions(gpu_lib):
    """Dense tensors in any order of dimensions."""
    a, b = make([(8, 6, 5, 3), (12, 10)], [torch.float32], seed=9)
    a, b = a.contiguous(memory_format=torch.channels_last), b.t()
    out = [torch.empty_like(a), torch.empty_like(b)]
    assert out[1].stride() == b.stride()
    check([a, b], 0.1)
    binding.grad_clip([a, b], 0.1, out=out)
    _, refs = oracle.grad_clip([wide(a), wide(b)], 0.1)
    assert all(np.abs(wide(o) - r).max() <= 1e-7 for o, r in zip(out, refs))


@pytest.mark.gpu
def test_equal_calls_give_equal_bits(gpu_lib):
    grads = make([700001, 3, 90000, 64], seed=11)
    runs = [torch.stack([binding.grad_norm(grads, p) for p in (1.0, 2.0, INF)]) for _ in range(4)]
    assert all(torch.equal(runs[0], r) for r in runs)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[300, 4, 4], [700001, 3, 90000]], ids=str)
def test_other_stream_and_graph(gpu_lib, sizes):
    grads = make(sizes, seed=13)
    out = [torch.empty_like(g) for g in grads]
    norm = binding.grad_clip(grads, 0.1, out=out)
    ref = [o.clone() for o in out]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = binding.grad_clip(grads, 0.1, out=out)
    side.synchronize()
    assert torch.equal(norm, other) and all(torch.equal(a, r) for a, r in zip(out, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = binding.grad_clip(grads, 0.1, out=out)
    for k in range(4):
        for g in grads:
            g.mul_(1.5)
        eager_out = [torch.empty_like(g) for g in grads]
        eager = binding.grad_clip(grads, 0.1, out=eager_out)
        for o in out:
            o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, eager) and all(torch.equal(a, r) for a, r in zip(out, eager_out)), k


@pytest.mark.gpu
def test_past_32_bit_offsets(gpu_lib):
    n = (1 << 31) + 70001
    g = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    g[-3:] = 300.0
    exact = float(np.sqrt(n - 3 + 3 * 300.0 ** 2))
    norm = binding.grad_clip([g], exact / 4)
    assert abs(float(norm) - exact) <= 2e-7 * exact
    assert bool((g[:-3] == 0.25).all()) and bool((g[-3:] == 75.0).all())


@pytest.mark.gpu
def test_parameters_of_a_network(gpu_lib):
    layer = autograd.GroupNorm(2, 6, device=DEV)
    conv = autograd.OaAConv2d(3, 6, 3, device=DEV)
    params = list(conv.parameters()) + list(layer.parameters()) + [torch.nn.Parameter(torch.zeros(4, device=DEV))]
    layer(conv(torch.rand(2, 3, 9, 9, device=DEV))).square().sum().backward()
    grads = [p.grad.clone() for p in params if p.grad is not None]
    assert len(grads) == 3
    norm = autograd.clip_grad_norm_(params, 0.5)
    ref_norm, refs = oracle.grad_clip([wide(g) for g in grads], 0.5)
    assert abs(float(norm) - ref_norm) <= 2e-7 * ref_norm
    for p, r in zip(params, refs):
        assert np.all(np.abs(wide(p.grad) - r) <= 4e-7 * np.abs(r) + 2.0 ** -149)
    again = float(autograd.clip_grad_norm_(params, 0.5))
    assert abs(again - 0.5) < 1e-5


@pytest.mark.gpu
def test_binding_refuses(gpu_lib):
    a, b = make([8, 9], [torch.float32])
    with pytest.raises(ValueError, match="norm_type"):
        binding.grad_norm([a], 3.0)
    with pytest.raises(ValueError, match="gradient 1"):
        binding.grad_norm([a, b.double()])
    with pytest.raises(ValueError, match="gradient 1"):
        binding.grad_norm([a, b.cpu()])
    with pytest.raises(ValueError, match="gaps"):
        binding.grad_norm([a[::2]])
    with pytest.raises(ValueError, match="gaps"):
        binding.grad_clip([a[:1].expand(5)], 1.0)
    with pytest.raises(ValueError, match="outputs"):
        binding.grad_clip([a, b], 1.0, out=[a])
    with pytest.raises(ValueError, match="output 0"):
        binding.grad_clip([a], 1.0, out=[b])
    with pytest.raises(ValueError, match="output 0"):
        binding.grad_clip([a], 1.0, out=[a.bfloat16()])
    with pytest.raises(ValueError, match="written twice"):
        binding.grad_clip([a, b, a], 1.0)
    assert float(binding.grad_norm([a, a])) > 0  # reading one twice is well defined
    empty = a[:0]
    binding.grad_clip([empty, a, empty], 1.0)
    one = torch.nn.Parameter(torch.ones(4, device=DEV))
    one.grad = torch.full((4,), 2.0, device=DEV)
    assert float(autograd.clip_grad_norm_(one, 1.0)) == 4.0 and abs(float(one.grad[0]) - 0.5) < 1e-6
    for bad in (-1.0, float("nan")):
        with pytest.raises(binding.OaaError, match="max_norm"):
            binding.grad_clip([a], bad)


# ---- no GPU ---------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    import os

    from paper_1601_06815_amd import build
    if not os.path.exists(build.LIB_PATH):
        build.build()
    return binding.load()


@pytest.mark.parametrize("p", [1.0, 2.0, INF])
def test_oracle_matches_torch(p):
    rng = np.random.default_rng(17)
    grads = [rng.standard_normal(s) for s in ((3, 4), 5, (2, 2, 2))]
    params = [torch.nn.Parameter(torch.zeros(g.shape, dtype=torch.float64)) for g in (np.asarray(g) for g in grads)]
    for q, g in zip(params, grads):
        q.grad = torch.from_numpy(np.asarray(g)).clone()
    ref = torch.nn.utils.clip_grad_norm_(params, 0.7, p)
    norm, clipped = oracle.grad_clip(grads, 0.7, p)
    assert abs(norm - float(ref)) < 1e-12
    assert all(np.allclose(c, q.grad.numpy(), rtol=1e-12) for c, q in zip(clipped, params))


def arrays(ptrs, sizes, kinds):
    import array
    return array.array("Q", ptrs), array.array("q", sizes), array.array("i", kinds)


@pytest.mark.parametrize("change,status", [
    (dict(count=-1), 1), (dict(type=0), 1), (dict(type=4), 1), (dict(norm=None), 1), (dict(norm=258), 1),
    (dict(ptrs=(0, 256)), 1), (dict(ptrs=(257, 256)), 1), (dict(sizes=(-1, 4)), 1), (dict(kinds=(0, 3)), 1),
    (dict(sizes=(1 << 60, 4)), 2), (dict(ws=None), 3), (dict(bytes=64), 3), (dict(ws=264), 1), (dict(max=-1.0), 1),
    (dict(out=(0, 256)), 1), (dict(out=(256, 257)), 1), (dict(null=True), 1),
])
def test_refused_lists(lib, change, status):
    """Refused before any launch."""
    k = dict(count=2, type=2, norm=256, ptrs=(256, 256), sizes=(4, 4), kinds=(0, 1), ws=256, bytes=1 << 20, max=1.0,
             out=(256, 256), null=False)
    k.update(change)
    src, sizes, kinds = arrays(k["ptrs"], k["sizes"], k["kinds"])
    out = arrays(k["out"], (), ())[0]
    at = [None if k["null"] else a.buffer_info()[0] for a in (src, sizes, kinds)]
    with pytest.raises(binding.OaaError) as e:
        binding.oaa_grad_clip(k["count"], at[0], out.buffer_info()[0], at[1], at[2], k["type"], k["max"], k["norm"],
                              k["ws"], k["bytes"], None)
    assert e.value.status == status and e.value.detail
    if "out" not in change and "max" not in change:
        with pytest.raises(binding.OaaError) as e:
            binding.oaa_grad_norm(k["count"], at[0], at[1], at[2], k["type"], k["norm"], k["ws"], k["bytes"], None)
        assert e.value.status == status


def test_workspace_grows_with_the_tensors(lib):
    sizes = [binding.oaa_grad_workspace_bytes(n) for n in (0, 1, 100, 100000)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and all(s % 256 == 0 for s in sizes)


def test_dense_in_any_order():
    t = torch.zeros(4, 6, 5, 3)
    for ok in (t, t.permute(3, 1, 0, 2), t.contiguous(memory_format=torch.channels_last), t[2], t[:0], t[:, :, :1, :1][:1, :1]):
        assert binding._dense(ok)
    for bad in (t[:, ::2], t[:, :3], t[:1, :1, :1, :1].expand(4, 1, 1, 1), t.as_strided((3, 3), (2, 1))):
        assert not binding._dense(bad)


def test_binding_refuses_on_the_cpu():
    with pytest.raises(ValueError, match="on the GPU"):
        binding.grad_norm([torch.zeros(3)])


@pytest.mark.gpu
def test_writes_are_seen_by_autograd(gpu_lib):
    """A tensor that a graph has saved, clipped in place or written as an output,
    must not be used changed."""
    for write in (lambda h: binding.grad_clip([h], 0.01),
                  lambda h: binding.grad_clip([torch.ones_like(h)], 0.01, out=[h]),
                  lambda h: binding.group_norm_forward(torch.ones_like(h), 1, y=h)):
        h = torch.ones((2, 3, 4), device=DEV, requires_grad=True) * 2
        z = (h * h).sum()
        version = h._version
        write(h.detach())
        assert h._version > version
        with pytest.raises(RuntimeError, match="inplace"):
            z.backward()
    read = torch.ones(5, device=DEV)
    version = read._version
    binding.grad_norm([read])
    binding.grad_clip([read], 1.0, out=[torch.empty_like(read)])
    assert read._version == version
    with torch.inference_mode():  # such tensors have no versions
        inside = torch.ones(5, device=DEV)
        binding.grad_clip([inside], 1.0)
        binding.group_norm_forward(torch.ones((2, 3, 4), device=DEV), 1, y=torch.empty((2, 3, 4), device=DEV))
    assert float(inside[0]) < 0.5


@pytest.mark.parametrize("src,out,sizes,kinds", [
    ((4096, 8192), (8192, 4096), (4, 4), (0, 0)),  # exchanged
    ((4096, 8192), (16384, 4096), (4, 4), (0, 0)),  # the second into the first
    ((4096, 8192), (4096, 4096 + 8), (4, 4), (0, 1)),  # an output inside another
    ((4096, 4096 + 12), (4096, 4096 + 12), (4, 4), (0, 0)),  # in place, one value in common
    ((4096, 8192), (4096 + 4, 16384), (4, 4), (0, 0)),  # a step beside its own gradient
    ((4096, 4096), (4096, 16384), (4, 4), (0, 0)),  # the same gradient, read once in place and once not
    ((4096, 1 << 20, 8192), (1 << 21, 1 << 22, 4096 + 398), (100, 7, 3), (0, 0, 1)),  # the last value's half
    ((1 << 20, 4096), (4096 + 8, 1 << 21), (64, 64), (1, 1)),
    ((4096, 0, 8192), (1 << 20, 0, (1 << 20) + 14), (8, 0, 8), (1, 0, 1)),  # an empty one between
])
def test_refused_overlaps(lib, src, out, sizes, kinds):
    """A tensor that one workgroup would write while another still reads it."""
    count = len(sizes)
    (a, n, k), o = arrays(src, sizes, kinds), arrays(out, (), ())[0]
    with pytest.raises(binding.OaaError, match="overlap") as e:
        binding.oaa_grad_clip(count, a.buffer_info()[0], o.buffer_info()[0], n.buffer_info()[0], k.buffer_info()[0], 2,
                              1.0, 256, 512, 1 << 20, None)
    assert e.value.status == 1


@pytest.mark.gpu
def test_neighbours_are_no_overlap(gpu_lib):
    """Outputs right beside gradients and each other, in any order, some in place."""
    room = make([64], [torch.float32], seed=19)[0]
    refs = wide(room).copy()
    grads = [room[40:48], room[8:16], room[24:24], room[16:23], room[8:16]]
    out = [room[40:48], room[23:31], room[12:12], room[0:7], room[48:56]]
    norm, clipped = oracle.grad_clip([wide(g) for g in grads], 0.1)
    assert abs(float(binding.grad_clip(grads, 0.1, out=out)) - norm) <= 2e-7 * norm
    for at, c in zip((40, 23, 12, 0, 48), clipped):
        refs[at:at + len(c)] = c
    assert np.all(np.abs(wide(room) - refs) <= 4e-7 * np.abs(refs))
    with pytest.raises(binding.OaaError, match="overlap"):
        binding.grad_clip([room[:8], room[8:16]], 0.1, out=[room[8:16], room[:8]])
    with pytest.raises(binding.OaaError, match="overlap"):
        binding.grad_clip([room[:8], room[4:12]], 0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[50, 60], [50000, 60, 70000]], ids=str)
def test_infinite_bound(gpu_lib, sizes):
    """No bound: nothing changes, unless the norm is infinite too, where inf / inf
    has no value."""
    grads = make(sizes, [torch.float32], seed=23)
    before = [g.clone() for g in grads]
    assert np.isfinite(float(binding.grad_clip(grads, INF)))
    assert all(torch.equal(g, r) for g, r in zip(grads, before))
    grads[1][2] = INF
    assert float(binding.grad_clip(grads, INF)) == INF and all(bool(torch.isnan(g).all()) for g in grads)
