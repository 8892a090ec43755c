"""Plain float64 definitions of the attention-side operators (NumPy): norm and
position rotation of heads, their gradient, the append to a paged cache, and
PAM attention over it.  Every PAM term is the oracle's (``pam_ref``), sums,
norms and softmax are float64; each definition comes with the scale its
float32 error grows with."""
from __future__ import annotations

import numpy as np

from . import pam_ref


def _pairs(rot: int, interleaved: bool):
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)


def rotate(y, positions, cos, sin, interleaved: bool, back: bool = False):
    """The first 2 * cos.shape[1] values of y (tokens, heads, d) turned by the
    angles of each token's position (NaN where the tables have no such row);
    also the sum of the magnitudes of each value's terms."""
    z, size = y.copy(), np.abs(y)
    if cos is None:
        return z, size
    a, b = _pairs(2 * cos.shape[1], interleaved)
    known = (positions >= 0) & (positions < cos.shape[0])
    at = np.where(known, positions, 0)
    c, s = (np.where(known[:, None], t[at].astype(np.float64), np.nan)[:, None] for t in (cos, sin))
    if back:
        s = -s
    z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    size[..., a] = np.abs(y[..., a] * c) + np.abs(y[..., b] * s)
    size[..., b] = np.abs(y[..., b] * c) + np.abs(y[..., a] * s)
    return z, size


def norm_rope(x, weight, positions, cos, sin, eps: float, interleaved: bool):
    """(z, size): norm and rotation of x (tokens, heads, d)."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    return rotate(y, positions, cos, sin, interleaved)


def norm_rope_grad(dz, x, weight, positions, cos, sin, eps: float, interleaved: bool):
    """(dx, its scale, dweight, its scale) from the formula."""
    g, size = rotate(np.asarray(dz, np.float64), positions, cos, sin, interleaved, back=True)
    if weight is None:
        return g, size, None, None
    x, w = np.asarray(x, np.float64), weight.astype(np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = g * w
    dx = r * (u - x * r * r * (u * x).mean(-1, keepdims=True))
    dx_size = r * (size * np.abs(w) + np.abs(x) * r * r * (size * np.abs(w * x)).mean(-1, keepdims=True))
    return dx, dx_size, (g * x * r).sum((0, 1)), (size * np.abs(x) * r).sum((0, 1))


def attention(q, k_cache, v_cache, table, kv_lens, q_starts, scale: float, causal: bool = True, window: int = 0):
    """(out, size, score_size): PAM attention of the tokens q (float32, tokens,
    heads, d) over the paged caches (float32), the sum of |P .^ v| of each
    output, and for each (token, head) the largest sum of |q .^ k| over its keys."""
    tokens, heads, d = q.shape
    pages, page, kv_heads, _ = k_cache.shape
    group = heads // kv_heads
    out = np.zeros((tokens, heads, d))
    size = np.zeros((tokens, heads, d))
    score_size = np.zeros((tokens, heads))
    for b, length in enumerate(kv_lens):
        first, last = int(q_starts[b]), int(q_starts[b + 1])
        for t in range(first, last):
            position = int(length) - (last - first) + t - first
            keys = np.arange(max(int(length), 0))
            if causal:
                keys = keys[keys <= position]
            if window > 0:
                keys = keys[keys > position - window]
            ids = table[b][keys // page]
            keys, ids = keys[(ids >= 0) & (ids < pages)], ids[(ids >= 0) & (ids < pages)]
            if len(keys) == 0:
                continue
            for h in range(heads):
                k = k_cache[ids, keys % page, h // group]
                v = v_cache[ids, keys % page, h // group]
                with np.errstate(all="ignore"):
                    terms = pam_ref.pam_mul_ref(np.broadcast_to(q[t, h], k.shape), k).astype(np.float64)
                    s = terms.sum(-1) * scale
                    score_size[t, h] = np.abs(terms).sum(-1).max() * abs(scale)
                    if np.all(s == -np.inf):
                        continue
                    p = np.exp(s - s.max())
                    p = p / p.sum()
                    if np.isnan(p).any():
                        out[t, h] = np.nan
                        continue
                    p32 = np.broadcast_to(p.astype(np.float32)[:, None], v.shape)
                    terms = pam_ref.pam_mul_ref(p32, v).astype(np.float64)
                    out[t, h] = terms.sum(0)
                    size[t, h] = np.abs(terms).sum(0)
    return out, size, score_size
