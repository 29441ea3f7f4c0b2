"""fp64 numpy definitions of the gated unit, forward and backward, and of dropout
with its generator's mask.

Written from the formulas: the products as sums over channels position by
position; the generator Philox4x32-10 from its published description, in
unsigned 64-bit arithmetic.
"""

import numpy as np

from .norm import _act


def _flat(t):
    """[B, C, ...] as [positions, C]."""
    return np.moveaxis(t, 1, -1).reshape(-1, t.shape[1]).astype(np.float64)


def _back(t, like, channels):
    return np.moveaxis(t.reshape(like.shape[0], *like.shape[2:], channels), -1, 1)


def gated_preactivations(x, gate_weight, up_weight, gate_bias=None, up_bias=None):
    """g and u, [positions, F]."""
    v = _flat(x)
    out = []
    for w, b in ((gate_weight, gate_bias), (up_weight, up_bias)):
        z = v @ w.astype(np.float64).T
        out.append(z if b is None else z + b.astype(np.float64))
    return out


def gated_forward(x, gate_weight, up_weight, gate_bias=None, up_bias=None, activation="silu"):
    g, u = gated_preactivations(x, gate_weight, up_weight, gate_bias, up_bias)
    return _back(_act(activation, g)[0] * u, x, gate_weight.shape[0])


def gated_backward(dh, x, gate_weight, up_weight, gate_bias=None, up_bias=None, activation="silu"):
    """(dx, dgate_weight, dup_weight, dgate_bias, dup_bias)."""
    g, u = gated_preactivations(x, gate_weight, up_weight, gate_bias, up_bias)
    a, slope = _act(activation, g)
    d, v = _flat(dh), _flat(x)
    dg, du = d * u * slope, d * a
    dx = dg @ gate_weight.astype(np.float64) + du @ up_weight.astype(np.float64)
    return _back(dx, x, x.shape[1]), dg.T @ v, du.T @ v, dg.sum(axis=0), du.sum(axis=0)


def philox(counters, key):
    """Philox4x32-10 of counters [n, 4] under key (two words): [n, 4] words."""
    mask = np.uint64(0xFFFFFFFF)
    c = np.asarray(counters, dtype=np.uint64) & mask
    c0, c1, c2, c3 = c[:, 0], c[:, 1], c[:, 2], c[:, 3]
    k = [int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = ((p1 >> np.uint64(32)) ^ c1 ^ np.uint64(k[0]), p1 & mask,
                          (p0 >> np.uint64(32)) ^ c3 ^ np.uint64(k[1]), p0 & mask)
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack([c0, c1, c2, c3], axis=1)


def dropout_words(n, seed, start=0):
    """The words of elements start..start + n - 1 (start a multiple of 4) for a seed
    (key, call) of two signed 64-bit numbers."""
    key, call = (int(v) & (2 ** 64 - 1) for v in seed)
    i = np.arange(start // 4, start // 4 + (n + 3) // 4, dtype=np.uint64)
    counters = np.stack([i & np.uint64(0xFFFFFFFF), i >> np.uint64(32), np.full_like(i, call & 0xFFFFFFFF),
                         np.full_like(i, call >> 32)], axis=1)
    return philox(counters, (key & 0xFFFFFFFF, key >> 32)).reshape(-1)[:n]


def dropout_mask(shape, p, seed, layout="planes"):
    """Which elements of [B, C, ...] are kept; their order is the layout's."""
    kept = dropout_words(int(np.prod(shape)), seed) >= round(p * 2 ** 32)
    if layout == "planes":
        return kept.reshape(shape)
    return np.moveaxis(kept.reshape(shape[0], *shape[2:], shape[1]), -1, 1)


def dropout(x, p, seed, residual=None, layout="planes"):
    kept = dropout_mask(x.shape, p, seed, layout)
    y = np.where(kept, x.astype(np.float64), 0.0) / (1.0 - p if p < 1.0 else 1.0)
    return y if residual is None else y + residual.astype(np.float64)
