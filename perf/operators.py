"""The calls that the normalisation and the gradient operators' speed is measured
by, over the ranges in which a program that trains or serves convolution layers
makes them.

Group normalisation with its activation, after a layer with output x[B,C,H,W]:

- "forward": ``autograd.group_norm`` with no gradient wanted, as in serving.
- "step": ``binding.group_norm_forward`` and ``binding.group_norm_backward``, as
  a training step calls them that keeps its own tensors.
- "autograd": ``autograd.group_norm`` and ``torch.autograd.grad`` with respect to
  the input, the weight and the bias.

x is laid out in planes, as the convolution returns it, or channels last.

The gradients of a whole network of convolution and normalisation layers (per
layer: a kernel w[K,C,n,n], a weight[K] and a bias[K]):

- "norm": ``binding.grad_norm``, one norm over all of them.
- "clip": ``binding.grad_clip`` into buffers that the program keeps, so that the
  same gradients can be clipped again.
"""

import math

import torch

own = False

EPS = 1e-5
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _norm(name, how, B, C, G, H, W, layout, dtype, act, params="float32"):
    return {"name": name, "op": "group_norm", "how": how, "B": B, "C": C, "G": G, "H": H, "W": W, "layout": layout,
            "dtype": dtype, "params": params, "act": act}


def _grads(name, how, layers, first, K, C, n, types, p="2", most=1.0):
    """Gradients of `layers` layers: the first K x first x n x n, the others K x C x n x n."""
    return {"name": name, "op": "gradients", "how": how, "layers": layers, "first": first, "K": K, "C": C, "n": n,
            "types": types, "p": p, "most": most}


def listed():
    return [
        # after the smallest layer of the tests (32 x 32, 5 x 5): one latency-bound call
        _norm("tiny28_forward", "forward", 1, 4, 2, 28, 28, "planes", "float32", "silu"),
        # a layer whose kernel covers its whole input: one position per image
        _norm("point_forward", "forward", 128, 256, 32, 1, 1, "last", "float32", "relu"),
        # one image of 100 kernels over a 256 x 256 plane: a few groups of 1.6 million values
        _norm("plane252_forward", "forward", 1, 100, 4, 252, 252, "planes", "float32", "silu"),
        # serving a middle layer in 16 bits, three channels a group
        _norm("infer52_forward", "forward", 8, 96, 32, 52, 52, "last", "float16", "silu", params="same"),
        # training a middle layer of many channels and small planes
        _norm("mid54_step", "step", 128, 128, 32, 54, 54, "planes", "float32", "silu"),
        # a small batch with no size a multiple of anything
        _norm("ragged53_step", "step", 5, 27, 3, 53, 53, "last", "float32", "gelu"),
        # after the RGB first layer of an image network, in 16 bits
        _norm("first218_step", "step", 64, 64, 8, 218, 218, "last", "bfloat16", "silu"),
        # after the large-kernel layer that the benchmark times: odd planes of 113 x 113
        _norm("large113_autograd", "autograd", 32, 256, 32, 113, 113, "planes", "float32", "silu"),
        # one small layer's gradients: launches and host work
        _grads("tiny_clip", "clip", 1, 3, 4, 4, 5, "float32"),
        # a network of twenty middle layers, kernels in 16 bits and the rest in 32
        _grads("mid_norm", "norm", 20, 3, 128, 128, 3, "mixed"),
        # a network of large kernels in 16 bits, clipped
        _grads("large_clip", "clip", 16, 3, 256, 96, 16, "mixed"),
        # the same in 32 bits, the norm alone
        _grads("large_norm", "norm", 20, 3, 256, 96, 16, "float32"),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over the logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        if rng.random() < 0.67:
            C = _log_int(rng, 4, 500)
            G = rng.choice([g for g in range(1, C + 1) if C % g == 0])
            H = _log_int(rng, 1, 252)
            W = H if rng.random() < 0.7 else _log_int(rng, 1, 252)
            how = rng.choice(["forward", "step", "autograd"])
            # in training, groups of four values at least: the input's gradient is zero for one value
            # and nothing but cancellation for two; and no ReLU, whose derivative jumps where rounding
            # decides the sign
            act = rng.choice(["none", "silu", "gelu"] + ["relu"] * (how == "forward"))
            if how != "forward" and C // G * H * W < 4:
                continue
            c = _norm("", how, _log_int(rng, 1, 128), C, G, H, W, rng.choice(["planes", "last"]),
                      rng.choice(sorted(TYPES)), act, rng.choice(["float32", "same"]))
        else:
            how = rng.choice(["norm", "clip"])
            c = _grads("", how, rng.randint(1, 20 if how == "clip" else 60), rng.randint(1, 4), _log_int(rng, 4, 256),
                       _log_int(rng, 4, 128), _log_int(rng, 1, 16), rng.choice(["float32", "bfloat16", "mixed"]),
                       rng.choice(["2", "2", "2", "1", "inf"]), rng.choice([1e-2, 1.0, 1e9]))
        del c["name"]
        if work(c)["bytes"] <= 0.5 * most:
            return c


def _shapes(c):
    first = [(c["K"], c["first"], c["n"], c["n"]), (c["K"],), (c["K"],)]
    return first + [(c["K"], c["C"], c["n"], c["n"]), (c["K"],), (c["K"],)] * (c["layers"] - 1)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if c["op"] == "gradients":
        kinds = {"mixed": (torch.bfloat16, torch.float32)}.get(c["types"]) or (TYPES[c["types"]],) * 2
        # each tensor at a magnitude of its own
        grads = [(normal(*s) * (0.003 * 1.5 ** (i % 7))).to(kinds[len(s) == 1]) for i, s in enumerate(_shapes(c))]
        out = [torch.empty_like(g) for g in grads] if c["how"] == "clip" else None
        return {"c": c, "grads": grads, "out": out}
    B, C, H, W = c["B"], c["C"], c["H"], c["W"]
    dtype = TYPES[c["dtype"]]
    params = dtype if c["params"] == "same" else torch.float32
    form = torch.channels_last if c["layout"] == "last" else torch.contiguous_format
    # channels of a layer's output differ in scale and offset
    x = normal(B, C, H, W) * (0.5 + normal(1, C, 1, 1).abs()) + 0.5 * normal(1, C, 1, 1)
    s = {"c": c, "x": x.to(dtype).contiguous(memory_format=form),
         "weight": (1 + 0.2 * normal(C)).to(params), "bias": (0.2 * normal(C)).to(params)}
    if c["how"] != "forward":
        s["dy"] = (normal(B, C, H, W) * 0.1).to(dtype).contiguous(memory_format=form)
    if c["how"] == "autograd":
        s.update({k: s[k].requires_grad_() for k in ("x", "weight", "bias")})
    return s


def _act(name, z):
    """The activation of z, and its derivative there."""
    if name == "relu":
        return z.clamp(min=0), (z > 0).float()
    if name == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return z * sig, sig * (1 + z * (1 - sig))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return z, torch.ones_like(z)


@torch.no_grad()
def _plain_norm(s):
    c = s["c"]
    B, C, G, H, W = c["B"], c["C"], c["G"], c["H"], c["W"]
    D, S = C // G, H * W
    last = c["layout"] == "last"

    def grouped(t):  # views of the layout: [B,S,G,D] or [B,G,D,S]
        return t.permute(0, 2, 3, 1).reshape(B, S, G, D).float() if last else t.reshape(B, G, D, S).float()

    def whole(t):
        return t.reshape(B, H, W, C).permute(0, 3, 1, 2) if last else t.reshape(B, C, H, W)

    axes, images = ((1, 3), (0, 1)) if last else ((2, 3), (0, 3))
    side = (1, 1, G, D) if last else (1, G, D, 1)
    w, b = s["weight"].float().reshape(side), s["bias"].float().reshape(side)
    x = grouped(s["x"])
    d = x - x.mean(axes, keepdim=True)
    rstd = 1 / torch.sqrt((d * d).mean(axes, keepdim=True) + EPS)
    xh = d * rstd
    dtype, params = s["x"].dtype, s["weight"].dtype
    if c["how"] == "forward":
        return {"y": whole(_act(c["act"], xh * w + b)[0].to(dtype))}
    y, slope = _act(c["act"], xh * w + b)
    dz = grouped(s["dy"]) * slope
    dw, db = (dz * xh).sum(images).reshape(C), dz.sum(images).reshape(C)
    t = dz * w
    dx = rstd * (t - t.mean(axes, keepdim=True) - xh * (t * xh).mean(axes, keepdim=True))
    return {"y": whole(y.to(dtype)), "dx": whole(dx.to(dtype)), "dweight": dw.to(params), "dbias": db.to(params)}


def _plain_grads(s):
    c, grads = s["c"], s["grads"]
    if c["p"] == "inf":
        norm = torch.stack([g.float().abs().max() for g in grads]).max()
    elif c["p"] == "1":
        norm = torch.stack([g.float().abs().sum() for g in grads]).sum()
    else:
        norm = torch.sqrt(torch.stack([g.float().square().sum() for g in grads]).sum())
    if c["how"] == "norm":
        return {"norm": norm}
    coefficient = (c["most"] / (norm + 1e-6)).clamp(max=1)
    return {"norm": norm, "grads": [o.copy_(g.float() * coefficient) for o, g in zip(s["out"], grads)]}


def run(state):
    s = state
    c = s["c"]
    if not own:
        return _plain_grads(s) if c["op"] == "gradients" else _plain_norm(s)
    from paper_1601_06815_amd import autograd, binding

    if c["op"] == "gradients":
        if c["how"] == "norm":
            return {"norm": binding.grad_norm(s["grads"], norm_type=float(c["p"]))}
        norm = binding.grad_clip(s["grads"], c["most"], norm_type=float(c["p"]), out=s["out"])
        return {"norm": norm, "grads": s["out"]}
    x, w, b = s["x"], s["weight"], s["bias"]
    if c["how"] == "step":
        y, mean, rstd = binding.group_norm_forward(x, c["G"], w, b, eps=EPS, activation=c["act"])
        dx, dw, db = binding.group_norm_backward(s["dy"], x, c["G"], w, b, mean, rstd, activation=c["act"])
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    y = autograd.group_norm(x, c["G"], w, b, eps=EPS, activation=c["act"])
    if c["how"] == "forward":
        return {"y": y}
    dx, dw, db = torch.autograd.grad(y, (x, w, b), s["dy"])
    return {"y": y, "dx": dx, "dweight": dw, "dbias": db}


def work(case):
    """Bytes: every operator's inputs read once and its outputs written once. A
    training step is two operators, the second of which is called after the
    layers above: x is an input of both. Flops: those of the formulas, an
    exponential or an error function counted as ten."""
    c = case
    if c["op"] == "gradients":
        count = [math.prod(s) for s in _shapes(c)]
        wide = {"float32": (4, 4), "bfloat16": (2, 2), "mixed": (2, 4)}[c["types"]]
        nbytes = sum(n * wide[len(s) == 1] for n, s in zip(count, _shapes(c)))
        clip = c["how"] == "clip"
        return {"bytes": float(nbytes * (2 if clip else 1) + 4), "flops": float(sum(count) * (3 if clip else 2))}
    size = 4 if c["dtype"] == "float32" else 2
    n = c["B"] * c["C"] * c["H"] * c["W"]
    params = 2 * c["C"] * (size if c["params"] == "same" else 4)
    act = {"none": 0, "relu": 1, "silu": 13, "gelu": 14}[c["act"]]
    if c["how"] == "forward":
        return {"bytes": float(2 * n * size + params), "flops": float(n * (8 + act))}
    return {"bytes": float(5 * n * size + 3 * params), "flops": float(n * (8 + act) + n * (18 + 2 * act))}


def exact(case, seed):
    """In float64: the forward definition with the variance as the mean of
    squared deviations, and the gradients by differentiating it; for gradients
    the norm over one long vector."""
    c = case
    s = prepare(case, seed)
    if c["op"] == "gradients":
        norm = torch.linalg.vector_norm(torch.cat([g.double().flatten() for g in s["grads"]]), float(c["p"]))
        if c["how"] == "norm":
            return {"norm": norm}
        k = min(1.0, c["most"] / (float(norm) + 1e-6))
        return {"norm": norm, "grads": [g.double() * k for g in s["grads"]]}
    B, C, G = c["B"], c["C"], c["G"]
    train = c["how"] != "forward"
    x, w, b = (s[k].detach().double().requires_grad_(train) for k in ("x", "weight", "bias"))
    flat = x.reshape(B, G, -1)
    var, mean = torch.var_mean(flat, 2, correction=0, keepdim=True)
    z = ((flat - mean) / (var + EPS).sqrt()).reshape(x.shape) * w.reshape(1, C, 1, 1) + b.reshape(1, C, 1, 1)
    if c["act"] == "relu":
        y = torch.where(z > 0, z, torch.zeros_like(z))
    elif c["act"] == "silu":
        y = z * torch.sigmoid(z)
    elif c["act"] == "gelu":
        y = z * (1 + torch.erf(z / math.sqrt(2))) / 2
    else:
        y = z
    if not train:
        return {"y": y}
    dx, dw, db = torch.autograd.grad(y, (x, w, b), s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dweight": dw, "dbias": db}
