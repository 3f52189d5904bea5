"""The operators on a layer's rows, from their definitions in 64 bits (numpy): norm, its gradient, blocks of 8 bits with scales, the product of
them.  Each says beside its result what the errors of 32-bit arithmetic are measured by.  Test infrastructure only; shares nothing with the HIP library."""
from __future__ import annotations

import numpy as np

BLOCK, MOST, LEAST = 128, 448.0, 2.0 ** -126


def norm(h, weight, eps):
    """h [..., dim] -> h / sqrt(mean h^2 + eps) * weight."""
    return h / np.sqrt(np.square(h).mean(-1, keepdims=True) + eps) * weight


def norm_grad(h, weight, grad, eps, extra=None):
    """-> dx, dweight, and for each element of them the sum of sizes that their terms have: of dx that of its own term, and that of the row's common one."""
    r = 1.0 / np.sqrt(np.square(h).mean(-1, keepdims=True) + eps)
    t = grad * weight
    along = (t * h).sum(-1, keepdims=True) * r ** 2 / h.shape[-1]
    dx = r * (t - h * along)
    mass = r * np.abs(t), r * np.abs(h) * (np.abs(t * h).sum(-1, keepdims=True) * r ** 2 / h.shape[-1])
    axes = tuple(range(h.ndim - 1))
    return dx if extra is None else dx + extra, (grad * h * r).sum(axes), mass, np.abs(grad * h * r).sum(axes)


def gated(x, gate):
    with np.errstate(over="ignore"):
        return gate / (1.0 + np.exp(-gate)) * x


def blocks(y, tall):
    """y [rows, columns] -> (scale of each block, the scale of every element's block)."""
    rows, columns = y.shape
    scale = np.empty((-(-rows // tall), -(-columns // BLOCK)))
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            part = np.abs(y[i * tall:(i + 1) * tall, j * BLOCK:(j + 1) * BLOCK])
            finite = part[np.isfinite(part)]
            scale[i, j] = max(finite.max(initial=0.0) / MOST, LEAST)
    return scale, spread(scale, tall, rows, columns)


def spread(scale, tall, rows, columns):
    return np.repeat(np.repeat(scale, tall, 0)[:rows], BLOCK, 1)[:, :columns]


def product(a, a_scale, w, w_scale):
    """a [m, k], w [n, k] -> the product, and the sum of its terms' sizes."""
    x, y = a * spread(a_scale, 1, *a.shape), w * spread(w_scale, BLOCK, *w.shape)
    return x @ y.T, np.abs(x) @ np.abs(y).T


def largest_products(a, a_scale, w, w_scale, of):
    """The sum over each `of` neighbouring k of (at least) the size of their largest product."""
    def tops(x):
        x = np.abs(np.pad(x, ((0, 0), (0, -x.shape[1] % of))))
        return x.reshape(x.shape[0], -1, of).max(-1)
    return tops(a * spread(a_scale, 1, *a.shape)) @ tops(w * spread(w_scale, BLOCK, *w.shape)).T
