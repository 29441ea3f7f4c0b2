"""The gated unit and dropout together with the operators beside them, as programs use
them: a feed-forward block in a network that trains, and over tokens in a captured
step."""

import json
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import block as oracle
from paper_1601_06815_amd import autograd, train_example

DEV = "cuda:0"


def plain(p, net, seed, layout, x):
    """The same network of torch's float64 operations on the CPU, with parameters p and
    the mask of `seed`."""
    F = torch.nn.functional

    def norm(x, name, layer):
        return F.group_norm(x, layer.G, p[name + ".weight"], p[name + ".bias"], layer.eps)

    for i in range(2):
        x = F.conv2d(x, p[f"convs.{i}.weight"].flip(-1, -2))
        x = F.silu(norm(x, f"norms.{i}", net.norms[i]))
    z = norm(x, "block.norm", net.block.norm)
    g, u = (torch.einsum("fc,bchw->bfhw", p[f"block.unit.{n}_weight"], z) + p[f"block.unit.{n}_bias"][:, None, None]
            for n in ("gate", "up"))
    d = F.conv2d(F.silu(g) * u, p["block.down.weight"])
    # down's result is in planes, whatever the layout of the block's input
    kept = torch.from_numpy(oracle.dropout_mask(tuple(d.shape), net.block.dropout.p, seed, "planes"))
    x = x + torch.where(kept, d / (1.0 - net.block.dropout.p), 0.0)
    return F.linear(x.mean((2, 3)), p["head.weight"], p["head.bias"])


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_gradients_of_a_network(gpu_lib, layout, p):
    """Every parameter's gradient against float64. Each layer adds 1e-6 (the convolution's
    measured error) or less of its largest value, and eight layers' worth of them pass
    back through the network: 1e-4 of the largest."""
    torch.manual_seed(4)
    net = train_example.Net(layout=layout, device=DEV, hidden=88, dropout=p)
    (x, label), = train_example.batches(1, 8, 32, 4, 6, DEV)
    seed = tuple(net.block.dropout.state.tolist())
    torch.nn.functional.cross_entropy(net(x), label).backward()
    assert net.block.dropout.state.tolist() == [seed[0], seed[1] + (p > 0)]
    names = [n for n, _ in net.named_parameters()]
    values = [v.detach().cpu().double().requires_grad_() for v in net.parameters()]
    logits = plain(dict(zip(names, values)), net, seed, layout, x.cpu().double())
    grads = torch.autograd.grad(torch.nn.functional.cross_entropy(logits, label.cpu()), values)
    for name, v, g in zip(names, net.parameters(), grads):
        off = (v.grad.cpu().double() - g).abs().max()
        assert float(off) < 1e-4 * float(g.abs().max()), name


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_training_runs(gpu_lib, layout):
    history = train_example.train(steps=5, layout=layout, hidden=64, dropout=0.2)
    assert all(np.isfinite(h["loss"]) and 0 < h["grad_norm"] < float("inf") for h in history)


@pytest.mark.gpu
def test_the_command(gpu_lib):
    run = subprocess.run([sys.executable, "-m", "paper_1601_06815_amd.train_example", "--steps", "2", "--hidden", "40",
                          "--dropout", "0.5"], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stderr
    assert [json.loads(line)["step"] for line in run.stdout.splitlines()] == [0, 1]


def test_without_a_block_nothing_is_added():
    """The network's parameters, and the numbers it draws for them, are what they were."""
    torch.manual_seed(0)
    a = train_example.Net(device="cpu")
    left = torch.rand(1)
    torch.manual_seed(0)
    b = train_example.Net(device="cpu", hidden=16)
    names = [n for n, _ in a.named_parameters()]
    assert not any(n.startswith("block") for n in names)
    own = dict(b.named_parameters())
    assert all(torch.equal(v, own[n]) for n, v in a.named_parameters())
    torch.manual_seed(0)
    train_example.Net(device="cpu")
    assert torch.equal(torch.rand(1), left)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_captured_step_over_tokens(gpu_lib, dtype):
    """x + dropout(gated unit(norm(x))) forward and backward over tokens in a graph: each
    replay draws the next mask, and gives the bits of the eager calls with that seed."""
    torch.manual_seed(1)
    T, C, p = 150, 48, 0.3
    norm = autograd.GroupNorm(1, C, device=DEV, dtype=dtype)
    unit = autograd.GatedUnit(C, C, device=DEV, dtype=dtype)
    drop = autograd.Dropout(p, seed=9, device=DEV)
    x = torch.randn(T, C, device=DEV).to(dtype).requires_grad_()
    dy = torch.randn(T, C, device=DEV).to(dtype)
    leaves = [x, *norm.parameters(), *unit.parameters()]

    def step():
        y = drop(unit(norm(x)), x)
        return (y, *torch.autograd.grad(y, leaves, dy))

    def eager(call):
        seed = torch.tensor([9, call], dtype=torch.int64, device=DEV)
        y = autograd.dropout(unit(norm(x)), p, seed, x)
        return (y, *torch.autograd.grad(y, leaves, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    first = int(drop.state[1])
    assert first == 2
    for replay in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = eager(first + replay)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), replay
        with torch.no_grad():  # the next replay sees another input
            x.mul_(0.9)
    assert int(drop.state[1]) == first + 4
