"""A small image network of this library's parts, trained on synthetic data:
convolution (``OaAConv2d``), group normalisation with SiLU (``GroupNorm``),
convolution, group normalisation, a mean over the positions and a linear
classifier; every step clips the gradients (``clip_grad_norm_``) before SGD
applies them. With ``--hidden`` a feed-forward block follows the convolutions: group
normalisation, the gated unit (``GatedUnit``), a 1 x 1 convolution back to the network's
channels, and ``Dropout``, which adds the result to the block's input.

    python -m paper_1601_06815_amd.train_example [--steps N] [--layout planes|last] [--hidden F] [--dropout P]

prints one JSON line per step: the loss and the gradients' norm before clipping.
``--layout last`` normalises in torch's channels_last layout, between two
changes of layout.
"""

import argparse
import json

import torch

from paper_1601_06815_amd.autograd import Dropout, GatedUnit, GroupNorm, OaAConv2d, clip_grad_norm_


class Block(torch.nn.Module):
    """x + dropout(down(gated unit(norm(x)))), at each position."""

    def __init__(self, width, hidden, p, groups, device):
        super().__init__()
        self.norm = GroupNorm(groups, width, device=device)
        self.unit = GatedUnit(width, hidden, device=device)
        self.down = OaAConv2d(hidden, width, 1, device=device)
        self.dropout = Dropout(p, device=device)

    def forward(self, x):
        return self.dropout(self.down(self.unit(self.norm(x)).contiguous()), x)


class Net(torch.nn.Module):
    def __init__(self, channels=3, width=32, classes=4, kernels=(5, 7), groups=8, layout="planes", device="cuda",
                 hidden=0, dropout=0.0):
        super().__init__()
        self.form = torch.channels_last if layout == "last" else torch.contiguous_format
        self.convs = torch.nn.ModuleList(
            OaAConv2d(c, width, n, device=device) for c, n in zip((channels, width), kernels))
        self.norms = torch.nn.ModuleList(
            GroupNorm(groups, width, activation="silu", device=device) for _ in kernels)
        self.head = torch.nn.Linear(width, classes, device=device)
        self.block = Block(width, hidden, dropout, groups, device) if hidden else None

    def forward(self, x):
        for conv, norm in zip(self.convs, self.norms):
            x = norm(conv(x).contiguous(memory_format=self.form))
        if self.block is not None:
            x = self.block(x)
        return self.head(x.mean((2, 3)))


def batches(steps, B, N, classes, seed, device):
    """Noise with a grating whose direction is the class."""
    gen = torch.Generator().manual_seed(seed)
    line = torch.arange(N, dtype=torch.float32)
    for _ in range(steps):
        label = torch.randint(classes, (B,), generator=gen)
        angle = label.float() * (torch.pi / classes)
        phase = line[None, None, :] * angle.cos()[:, None, None] + line[None, :, None] * angle.sin()[:, None, None]
        x = torch.randn((B, 3, N, N), generator=gen) + 2.0 * torch.sin(0.9 * phase)[:, None]
        yield x.to(device), label.to(device)


def train(steps=20, B=16, N=32, lr=0.5, max_norm=1.0, layout="planes", seed=0, device="cuda", report=None, hidden=0,
          dropout=0.0):
    """The losses and gradient norms of `steps` steps."""
    torch.manual_seed(seed)
    net = Net(layout=layout, device=device, hidden=hidden, dropout=dropout)
    optimiser = torch.optim.SGD(net.parameters(), lr=lr)
    history = []
    for step, (x, label) in enumerate(batches(steps, B, N, 4, seed, device)):
        optimiser.zero_grad()
        loss = torch.nn.functional.cross_entropy(net(x), label)
        loss.backward()
        norm = clip_grad_norm_(net.parameters(), max_norm)
        optimiser.step()
        history.append({"step": step, "loss": float(loss.detach()), "grad_norm": float(norm)})
        if report:
            report(history[-1])
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--layout", choices=("planes", "last"), default="planes")
    ap.add_argument("--hidden", type=int, default=0, help="channels inside of a feed-forward block; 0: no block")
    ap.add_argument("--dropout", type=float, default=0.0, help="of the block's result")
    a = ap.parse_args()
    train(steps=a.steps, layout=a.layout, hidden=a.hidden, dropout=a.dropout,
          report=lambda h: print(json.dumps(h), flush=True))


if __name__ == "__main__":
    main()
