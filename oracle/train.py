"""CPU oracle of the retraining operators beside the convolution (test
infrastructure only, like the rest of ``oracle/``): group normalisation with
an activation and its gradient, the norm of all gradients with the factor
that clips them, and the AdamW step with moments in 32 or 8 bits.

Each function is the plain definition in fp64 (numpy), from the same fp32 or
fp16 inputs that the kernels get; none shares code with the HIP path.  Two
decisions are taken in the precision that include/psc.h names, since fp64
would decide otherwise next to a border: the ReLU's mask goes by u as fp32
rounds it after each operation, and 8-bit codes are taken against scales held
in fp32."""
from __future__ import annotations

import numpy as np

GROUP = 256      # elements that share the scales of 8-bit moments


def _grouped(x, groups):
    n, c, h, w = x.shape
    return np.asarray(x, dtype=np.float64).reshape(n, groups, c // groups, h * w)


def _per_channel(t, c, groups, fill):
    t = np.full(c, fill) if t is None else np.asarray(t, dtype=np.float64)
    return t.reshape(1, groups, c // groups, 1)


def _sigmoid(u):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-u))


def statistics(x, groups: int, eps: float):
    """mean and 1 / sqrt(variance + eps) of each image's groups, [n, groups]."""
    xg = _grouped(x, groups)
    mean = xg.mean(axis=(2, 3))
    var = ((xg - mean[:, :, None, None]) ** 2).mean(axis=(2, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def group_norm(x, groups: int, gamma, beta, eps: float, act: str):
    """y [n, c, h, w], mean and rstd [n, groups]."""
    mean, rstd = statistics(x, groups, eps)
    c = x.shape[1]
    u = (_grouped(x, groups) - mean[:, :, None, None]) * rstd[:, :, None, None]
    u = u * _per_channel(gamma, c, groups, 1.0) + _per_channel(beta, c, groups, 0.0)
    y = np.maximum(u, 0.0) if act == "relu" else u * _sigmoid(u) if act == "silu" else u
    return y.reshape(x.shape), mean, rstd


def relu_mask(x, groups: int, gamma, beta, mean, rstd):
    """u > 0, u rounded to fp32 after each of its four operations."""
    n, c, h, w = x.shape
    f = np.float32
    xh = (x.reshape(n, groups, c // groups, h * w).astype(f) - mean.astype(f)[:, :, None, None]) * \
        rstd.astype(f)[:, :, None, None]
    u = xh * _per_channel(gamma, c, groups, 1.0).astype(f) + _per_channel(beta, c, groups, 0.0).astype(f)
    return u > 0


def group_norm_back(x, dy, groups: int, gamma, beta, mean, rstd, act: str):
    """dx, dgamma, dbeta from the statistics that the forward kept."""
    n, c, h, w = x.shape
    ga, be = _per_channel(gamma, c, groups, 1.0), _per_channel(beta, c, groups, 0.0)
    r = np.asarray(rstd, dtype=np.float64)[:, :, None, None]
    xh = (_grouped(x, groups) - np.asarray(mean, dtype=np.float64)[:, :, None, None]) * r
    du = _grouped(dy, groups)
    if act == "relu":
        du = du * relu_mask(x, groups, gamma, beta, mean, rstd)
    elif act == "silu":
        u = xh * ga + be
        s = _sigmoid(u)
        du = du * s * (1.0 + u * (1.0 - s))
    e = du * ga
    dx = r * (e - e.mean(axis=(2, 3), keepdims=True) - xh * (e * xh).mean(axis=(2, 3), keepdims=True))
    return dx.reshape(x.shape), (du * xh).sum(axis=(0, 3)).reshape(c), du.sum(axis=(0, 3)).reshape(c)


def grad_norm(grads, scale: float = 1.0, max_norm: float = np.inf):
    """The norm of all gradients, and the factor that unscales and clips them."""
    norm = scale * np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    if not np.isfinite(norm):
        return norm, np.nan
    return norm, scale * (max_norm / norm if norm > max_norm else 1.0)


def decode_m(q, scale):
    """int8 codes [k] and scales [ceil(k/256), 2] -> the first moments they stand for."""
    q = np.asarray(q, dtype=np.float64)
    return np.sign(q) * (q / 127.0) ** 2 * np.repeat(np.asarray(scale, dtype=np.float64)[:, 0], GROUP)[:q.size]


def decode_v(c, scale):
    c = np.asarray(c, dtype=np.float64)
    return (c / 255.0) ** 4 * np.repeat(np.asarray(scale, dtype=np.float64)[:, 1], GROUP)[:c.size]


def encode(m, v):
    """Moments -> int8 codes, uint8 codes, scales: of each 256 in a row the
    largest magnitudes, held in fp32; the nearest code of sqrt|m| and of
    v^(1/4), a v above zero never at code 0."""
    m, v = np.asarray(m, dtype=np.float64), np.asarray(v, dtype=np.float64)
    groups = -(-m.size // GROUP)
    pad = lambda t: np.concatenate([t, np.zeros(groups * GROUP - t.size)]).reshape(groups, GROUP)   # noqa: E731
    scale = np.stack([np.abs(pad(m)).max(axis=1, initial=0), pad(v).max(axis=1, initial=0)], axis=1).astype(np.float32)
    top = np.repeat(scale.astype(np.float64), GROUP, axis=0)[:m.size]
    with np.errstate(divide="ignore", invalid="ignore"):
        cm = np.where(top[:, 0] > 0, np.floor(127.0 * np.sqrt(np.abs(m) / top[:, 0]) + 0.5), 0.0)
        cv = np.where(top[:, 1] > 0, np.floor(255.0 * np.sqrt(np.sqrt(v / top[:, 1])) + 0.5), 0.0)
    cv = np.where((v > 0) & (cv == 0), 1.0, cv)
    return (np.sign(m) * cm).astype(np.int8), cv.astype(np.uint8), scale


def adamw(p, g, m, v, step: int, lr, beta1, beta2, eps, weight_decay, factor=1.0):
    """New p, m, v (fp64) of step number ``step`` (from 1).  The betas are the
    fp32 values that the library is given."""
    p, m, v = (np.asarray(t, dtype=np.float64) for t in (p, m, v))
    b1, b2 = float(np.float32(beta1)), float(np.float32(beta2))
    g = float(np.float32(factor)) * np.asarray(g, dtype=np.float64)
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    update = m / (1.0 - b1 ** step) / (np.sqrt(v / (1.0 - b2 ** step)) + float(np.float32(eps)))
    lr, wd = float(np.float32(lr)), float(np.float32(weight_decay))
    return p - lr * wd * p - lr * update, m, v
