"""Inputs and comparison rules of the attention-side operators' tests.

Tolerances follow from the operators' float32 steps, u = 2^-24 each:

norm_rope   the mean of d squares is off by at most (d + 2) u relatively in
            any order, its square root's inverse by half that and 3 u; the
            products with r, w, the angle and the sum of two terms add 5 u, all
            relative to the terms' magnitudes: (d / 2 + 9) u size.  bfloat16
            results are off by another half unit of 2^-8.
gradient    dx: the two means again, each (d + 2) u and a few steps: 2 (d + 12) u
            of its terms' magnitudes.  dweight: a sum of n terms in any order:
            (n + d / 2 + 12) u of the sum of magnitudes.
attention   a score of d terms is off by (d + 3) u of the sum of its terms'
            magnitudes (times scale), the exponent's argument by another 3 u of
            itself; a probability relatively by twice that (numerator and sum)
            plus (n + 8) u for the sum and the division.  PAM's relative slope is
            at most 2.  The sum of n terms adds (n + 1) u, and what falls below
            the normal range n 2^-126.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def bf16(x: np.ndarray) -> np.ndarray:
    """x rounded to bfloat16 (nearest even), as float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where((u & 0x7FFFFFFF) > 0x7F800000, u, r).astype(np.uint32).view(np.float32)


def norm_rope_tolerance(size, d: int, to_bf16: bool):
    return (d / 2 + 9) * U * size * (1 + 2.0 ** -8) + (2.0 ** -8 * size if to_bf16 else 0.0) + 2.0 ** -126


def attention_tolerance(size, score_size, d: int, keys: int):
    score = (d + 6) * U * score_size * 2                      # |s| and its error, both ends of s - max
    relative = 2 * (2 * score + (keys + 8) * U) + (keys + 1) * U
    return np.expm1(relative)[..., None] * size + keys * 2.0 ** -126


def check(got: np.ndarray, want: np.ndarray, tol, what: str) -> None:
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN positions differ"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and np.array_equal(np.isinf(got), inf), f"{what}: infinities differ"
    fine = np.isfinite(want)
    tol = np.broadcast_to(tol, want.shape)[fine]
    err = np.abs(got[fine] - want[fine])
    if err.size:
        worst = int(np.argmax(err / np.maximum(tol, 1e-300)))
        assert np.all(err <= tol), (f"{what}: {int((err > tol).sum())} of {err.size} outside tolerance; worst "
                                    f"{err[worst]:.3e} against {tol[worst]:.3e}")


def tables(rows: int, rot: int):
    angle = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


class Paged:
    """A paged cache of sequences of given lengths, filled at random: pages in
    random order, unused slots and pages full of NaN."""

    def __init__(self, rng, kv_lens, page: int, heads: int, d: int, bf16_cache: bool, spare: int = 2):
        self.kv_lens = np.asarray(kv_lens, np.int32)
        need = [-(-max(int(n), 0) // page) for n in kv_lens]
        total = sum(need) + spare
        order = rng.permutation(total).astype(np.int32)
        self.table = np.full((len(kv_lens), max(need + [1])), -1, np.int32)
        self.k = np.full((total, page, heads, d), np.nan, np.float32)
        self.v = np.full((total, page, heads, d), np.nan, np.float32)
        at = 0
        for b, (n, pages) in enumerate(zip(kv_lens, need)):
            self.table[b, :pages] = order[at:at + pages]
            at += pages
            for j in range(int(n)):
                for c in (self.k, self.v):
                    c[self.table[b, j // page], j % page] = rng.standard_normal((heads, d))
        if bf16_cache:
            self.k, self.v = bf16(self.k), bf16(self.v)
