"""The operators together, as a program trains with them."""

import pytest
import torch

from paper_1601_06815_amd import autograd, train_example

DEV = "cuda:0"


def plain(p, G, eps, x):
    """The same network of torch's float64 operations on the CPU, with parameters p."""
    for i in range(2):
        x = torch.nn.functional.conv2d(x, p[f"convs.{i}.weight"].flip(-1, -2))
        z = torch.nn.functional.group_norm(x, G, p[f"norms.{i}.weight"], p[f"norms.{i}.bias"], eps)
        x = torch.nn.functional.silu(z)
    return torch.nn.functional.linear(x.mean((2, 3)), p["head.weight"], p["head.bias"])


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_gradients_of_a_network(gpu_lib, layout):
    """Every parameter's clipped gradient against float64. Each layer adds 1e-6
    (the convolution's measured error) or less of its largest value, and four
    layers' worth of them pass back through the network: 1e-4 of the largest."""
    torch.manual_seed(3)
    net = train_example.Net(layout=layout, device=DEV)
    (x, label), = train_example.batches(1, 8, 32, 4, 5, DEV)
    torch.nn.functional.cross_entropy(net(x), label).backward()
    names = [n for n, _ in net.named_parameters()]
    values = [p.detach().cpu().double().requires_grad_() for p in net.parameters()]
    held = dict(zip(names, values))

    logits = plain(held, net.norms[0].G, net.norms[0].eps, x.cpu().double())
    grads = torch.autograd.grad(torch.nn.functional.cross_entropy(logits, label.cpu()), values)
    exact = torch.sqrt(sum(g.square().sum() for g in grads))
    norm = autograd.clip_grad_norm_(net.parameters(), float(exact) / 2)
    assert abs(float(norm) - float(exact)) < 1e-4 * float(exact)
    for name, p, g in zip(names, net.parameters(), grads):
        off = (p.grad.cpu().double() - g / 2).abs().max()
        assert float(off) < 1e-4 * float(g.abs().max()), name


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["planes", "last"])
def test_training_learns(gpu_lib, layout):
    history = train_example.train(steps=25, layout=layout)
    assert all(h["grad_norm"] > 0 for h in history)
    assert sum(h["loss"] for h in history[-5:]) < 0.5 * sum(h["loss"] for h in history[:5])


def test_batches_are_reproducible():
    a, b = (list(train_example.batches(2, 3, 8, 4, 1, "cpu")) for _ in range(2))
    assert all(torch.equal(x, u) and torch.equal(y, v) for (x, y), (u, v) in zip(a, b))
    assert a[0][0].shape == (3, 3, 8, 8) and int(a[0][1].max()) < 4
