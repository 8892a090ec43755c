"""Comparison rules of the layer-and-step operators' tests.

Tolerances follow from the operators' float32 steps, u = 2^-24 each (a unit in
the last place of an approximate exp2, reciprocal or square root is 2 u):

tail        Q(x) = exp(-x^2 / 2) t R(t): t is off by 3 u relatively, the ten steps
            of R by at most 0.25 u each where R >= 0.12 at t = 0 and more with t,
            and the tail's slope in t is at most 1: 3 + 5 + 2 u; the exponent's
            argument by 2 u of x^2 / 2, exp2 by 2 u, the products 2 u: (14 + x^2) u
gelu        z times Q or 1 - Q: |z| ((15 + z^2) Q + 3 P) u with Q the smaller, P the
            taken side
logistic    1 / (1 + e) off by (1 - s) (2 |x| + 4) + 3 u of s, where x itself is off
            by r u relatively another (1 - s) r |x|
slopes      the same errors in the sum of their two terms
sums        of n terms in any order: n u of the terms' magnitudes
A result in bfloat16 is off by another half step, 2^-8.
"""
from __future__ import annotations

import numpy as np

from oracle import training_ref as ref

U = 2.0 ** -24
TINY = 2.0 ** -120            # below it exponentials leave the float32 range


def half_step(bf16: bool) -> float:
    return 2.0 ** -8 if bf16 else U


def _logistic_error(x, r: float):
    """Relative error of logistic(x), x off by r u relatively."""
    s = ref.logistic(x)
    return ((1 - s) * ((2 + r) * np.abs(x) + 4) + 3) * U


def _tanh_argument(z):
    return 2 * ref._T0 * (z + ref._T1 * z ** 3)


def activation_error(z, name):
    """Of the activation of a float32 z, in float32."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        if name == "gelu":
            q = ref.normal_below(-np.abs(z))
            p = np.where(z < 0, q, 1 - q)
            return np.abs(z) * ((15 + z * z) * q + 3 * p) * U + TINY
        if name in ("gelu_tanh", "silu"):
            x = z if name == "silu" else _tanh_argument(z)
            return np.abs(z * ref.logistic(x)) * (_logistic_error(x, 0 if name == "silu" else 5) + 2 * U) + TINY
    return np.zeros_like(z)


def slope_error(z, name):
    z = np.clip(np.asarray(z, np.float64), -200, 200)
    if name == "gelu":
        q = ref.normal_below(-np.abs(z))
        bell = np.abs(z) * np.exp(-z * z / 2) * 0.4
        return ((15 + z * z) * q + 3 + bell * (8 + z * z)) * U + TINY
    if name in ("gelu_tanh", "silu"):
        x = z if name == "silu" else _tanh_argument(z)
        v = np.abs(z if name == "silu" else 2 * ref._T0 * z * (1 + 3 * ref._T1 * z * z))
        s, d = ref.logistic(x), _logistic_error(x, 0 if name == "silu" else 5)
        # s, and v s (1 - s), the last factor off by s d + u.
        return s * d + v * (s * (1 - s) * (d + 8 * U) + s * (s * d + U)) + 2 * U * np.abs(ref.slope(z, name)) + TINY
    return np.zeros_like(z)


def norm_limit(norm, max_norm):
    """The float32 factor the kernel takes, and its relative error against the definition."""
    f = np.float32
    c = f(max_norm) / (f(norm) + f(1e-6))
    return min(f(1), c), 4 * U


def step_errors(p, g, avg, sq, limit_error, step, lr, betas, eps, weight_decay, limit=1.0):
    """Errors of (p, avg, sq) after a step with 32-bit states: beta and 1 - beta are
    rounded, g' twice, each sum and product once; sqrt and reciprocal are
    approximate."""
    p, g, avg, sq = (np.asarray(t, np.float64) for t in (p, g, avg, sq))
    p1, m, v = ref.adamw(p, g, avg, sq, step, lr, betas, eps, weight_decay, limit)
    g = np.abs(g * limit)
    em = U * (2 * betas[0] * np.abs(avg) + 3 * (1 - betas[0]) * g + np.abs(m)) + limit_error * (1 - betas[0]) * g
    ev = U * (2 * betas[1] * sq + 5 * (1 - betas[1]) * g * g + v) + 2 * limit_error * (1 - betas[1]) * g * g
    return moved_error(p, m, v, em, ev, step, lr, betas, eps, weight_decay), em + TINY, ev + TINY


def moved_error(p, m, v, em, ev, step, lr, betas, eps, weight_decay):
    p1, by = ref.moved(p, m, v, step, lr, betas, eps, weight_decay)
    with np.errstate(divide="ignore", invalid="ignore"):
        relative = np.where(m != 0, em / np.abs(m), 0) + np.where(v > 0, ev / (2 * v), 0)
    return np.abs(by) * (12 * U + relative) + U * (2 * np.abs(p) + np.abs(p1)) + TINY
