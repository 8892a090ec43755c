"""Plain definitions of the layer-and-step operators (NumPy): the activations and
their slopes, a linear layer around a PAM product, the gradient of what it adds,
the gradients' norm, and the AdamW step.  Everything is float64 but the 8-bit
states' codes, whose definition rounds each operation to float32 and takes what is
below 2^-126 for zero."""
from __future__ import annotations

import math

import numpy as np

from . import pam_ref

ACTIVATIONS = (None, "relu", "gelu", "gelu_tanh", "silu")
BLOCK = 256
_below = np.vectorize(lambda z: 0.5 * math.erfc(-z / math.sqrt(2)), otypes=[np.float64])
_T0, _T1 = math.sqrt(2 / math.pi), 0.044715


def normal_below(z):
    """P(N <= z) of a standard normal N."""
    return _below(np.asarray(z, np.float64))


def logistic(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-np.asarray(x, np.float64)))


def activation(z, name):
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        if name == "relu":
            return np.where(z <= 0, 0.0, z)
        if name == "gelu":
            return z * normal_below(z)
        if name == "gelu_tanh":
            return z * logistic(2 * _T0 * (z + _T1 * z ** 3))
        return z * logistic(z) if name == "silu" else z


def slope(z, name):
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if name is None:
        return np.ones_like(z)
    far = np.where(np.isnan(z), z, np.clip(z, -800, 800))     # the slopes' limits at infinity
    if name == "gelu":
        return normal_below(far) + far * np.exp(-far * far / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        s = logistic(2 * _T0 * (far + _T1 * far ** 3))
        return s + far * s * (1 - s) * 2 * _T0 * (1 + 3 * _T1 * far ** 2)
    s = logistic(far)
    return s + far * s * (1 - s)


def linear(x, w, bias, name, residual):
    """(y, z, S): the layer's outputs, and the sums of the product terms' magnitudes."""
    z, size = pam_ref.pam_gemm_ref(x, w, False, True)
    z = z if bias is None else z + bias.astype(np.float64)
    y = activation(z, name)
    return y if residual is None else y + residual.astype(np.float64), z, size


def activation_grad(dy, z, name):
    """(dz, db)."""
    dy = np.asarray(dy, np.float64)
    d = slope(z, name) if name is not None else 1.0
    with np.errstate(invalid="ignore"):
        dz = np.where(np.asarray(z) <= 0, 0.0, dy) if name == "relu" else dy * d
    return dz, dz.sum(0)


def grad_norm(grads):
    return math.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads))


def clip(norm, max_norm):
    return 1.0 if norm is None else min(1.0, max_norm / (norm + 1e-6))


def moved(p, avg, sq, step, lr, betas, eps, weight_decay):
    """Parameters after their averages, and the step alone."""
    c1, c2 = 1 - betas[0] ** step, 1 - betas[1] ** step
    by = lr / c1 * avg / (np.sqrt(sq) / math.sqrt(c2) + eps)
    return p * (1 - lr * weight_decay) - by, by


def adamw(p, g, avg, sq, step, lr, betas, eps, weight_decay, limit=1.0):
    """(p, avg, sq) of one tensor after a step with 32-bit states."""
    p, g, avg, sq = (np.asarray(t, np.float64) for t in (p, g, avg, sq))
    g = g * limit
    avg = betas[0] * avg + (1 - betas[0]) * g
    sq = betas[1] * sq + (1 - betas[1]) * g * g
    return moved(p, avg, sq, step, lr, betas, eps, weight_decay)[0], avg, sq


# 8-bit states ---------------------------------------------------------------

def mix(x):
    """A hash of 32 bits: C. Wellons, "Prospecting for Hash Functions", 2018."""
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, tensor, n):
    """The bits added below a code, for avg and for sq."""
    key = mix(int(mix((seed + step * 0x9E3779B9) & 0xFFFFFFFF)) + tensor)
    h = mix(np.arange(n, dtype=np.uint64) + key)
    return ((h & np.uint64(0xFFFF)) * np.uint64(16) + np.uint64(8),
            (h >> np.uint64(16)) * np.uint64(16) + np.uint64(8))


def normal(x):
    """x in float32, what is below 2^-126 as a zero of its sign."""
    x = np.asarray(x, np.float32)
    return np.where(np.abs(x) < np.float32(2.0 ** -126), np.copysign(np.float32(0), x), x)


def code_value(code, scales, most):
    """The float32 values of codes (most: 127 of avg, 255 of sq)."""
    size = code & most
    f = np.where(size > 0, (size.astype(np.uint32) + np.uint32(1016 - most)) << np.uint32(20), 0).astype(np.uint32)
    with np.errstate(invalid="ignore"):
        x = normal(f.view(np.float32) * np.repeat(normal(scales), BLOCK)[:len(code)])
    return np.where(code > most, -x, x).astype(np.float32)


def code_of(x, most, bits):
    """(codes, scales) of magnitudes x."""
    n = len(x)
    blocks = np.pad(x, (0, -n % BLOCK)).reshape(-1, BLOCK)
    scales = blocks.max(1)                                   # NaN where one is
    by = np.repeat(np.where(scales > 0, scales, np.float32(1)), BLOCK)[:n]
    with np.errstate(invalid="ignore"):
        part = np.abs((x / by).astype(np.float32))
    code = ((part.view(np.uint32).astype(np.int64) + bits.astype(np.int64)) >> 20) - (1016 - most)
    code = np.clip(code, 0, most)
    if most == 255:
        code = np.where(x != 0, np.maximum(code, 1), 0)
    return code.astype(np.uint8), scales.astype(np.float32)


def adamw8(p, g, avg, sq, avg_scale, sq_scale, step, lr, betas, eps, weight_decay, seed, tensor, limit=None):
    """(p, avg, sq, avg_scale, sq_scale, the step alone) of one tensor after a
    step with 8-bit states; limit: the float32 factor of the gradient."""
    f = np.float32
    g = normal(g)
    with np.errstate(invalid="ignore", over="ignore"):
        if limit is not None:
            g = normal(g * f(limit))
        m = normal(normal(code_value(avg, avg_scale, 127) * f(betas[0])) + normal(g * f(1 - betas[0])))
        v = normal(normal(code_value(sq, sq_scale, 255) * f(betas[1])) + normal(normal(g * f(1 - betas[1])) * g))
        assert m.dtype == v.dtype == f
        r1, r2 = random_bits(seed, step, tensor, len(g))
        code, scale = code_of(np.abs(m), 127, r1)
        code |= np.where((m < 0) & (code > 0), 128, 0).astype(np.uint8)
        code2, scale2 = code_of(v, 255, r2)
        new, by = moved(np.asarray(p, np.float64), m.astype(np.float64), v.astype(np.float64), step, lr, betas, eps,
                        weight_decay)
    return new, code, code2, scale, scale2, by
