"""The float64 definitions of the attention-side operators, checked against
what does not come from their own formulas (CPU)."""
import numpy as np
import pytest

import attention_util as au
from oracle import attention_ref as ref
from oracle import pam_ref


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_rotation(interleaved):
    rng = np.random.default_rng(1)
    y = rng.standard_normal((5, 3, 16))
    cos, sin = au.tables(9, 12)
    pos = np.array([0, 8, 3, 3, 1])
    z, _ = ref.rotate(y, pos, cos, sin, interleaved)
    assert np.array_equal(z[..., 12:], y[..., 12:])
    assert np.allclose((z * z).sum(-1), (y * y).sum(-1), rtol=1e-6)
    assert np.allclose(z[0], y[0])
    back, _ = ref.rotate(z, pos, cos, sin, interleaved, back=True)
    assert np.allclose(back, y, atol=1e-6)
    # The complex form of one pair.
    a, b = (2, 3) if interleaved else (1, 7)
    angle = 3 * 10000.0 ** (-2 / 12)
    want = (y[2, 0, a] + 1j * y[2, 0, b]) * np.exp(1j * angle)
    assert np.allclose([z[2, 0, a], z[2, 0, b]], [want.real, want.imag], atol=1e-6)


def test_norm_gives_unit_mean_square():
    x = np.random.default_rng(2).standard_normal((4, 2, 32)) * 7
    z, _ = ref.norm_rope(x, np.ones(32, np.float32), None, None, None, 0.0, False)
    assert np.allclose((z * z).mean(-1), 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    """Central differences of the forward definition: their error is h^2 times a
    third derivative (values of order 1: below 1e-7 at h = 1e-4) and 1e-16 / h."""
    rng = np.random.default_rng(3)
    x, dz = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    w = (1 + 0.3 * rng.standard_normal(8)).astype(np.float32).astype(np.float64)
    cos, sin = (t.astype(np.float64) for t in au.tables(6, 6))
    pos = np.array([5, 0, 2])

    def loss(x, w):
        return (ref.norm_rope(x, w, pos, cos, sin, 1e-3, interleaved)[0] * dz).sum()

    dx, _, dw, _ = ref.norm_rope_grad(dz, x, w, pos, cos, sin, 1e-3, interleaved)
    h = 1e-4
    for value, grad in ((x, dx), (w, dw)):
        for i in np.ndindex(value.shape):
            old = value[i]
            value[i] = old + h
            up = loss(x, w)
            value[i] = old - h
            down = loss(x, w)
            value[i] = old
            assert abs((up - down) / (2 * h) - grad[i]) < 1e-6, i


def test_attention_by_hand():
    """One key: the probability is 1 and PAM with 1 is exact, so the output is
    the value; two equal keys: 0.5, a power of two, so their mean."""
    rng = np.random.default_rng(4)
    cache = au.Paged(rng, [1, 2], 4, 1, 8, False)
    cache.k[cache.table[1, 0], 1] = cache.k[cache.table[1, 0], 0]
    q = rng.standard_normal((2, 2, 8)).astype(np.float32)
    out, _, _ = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens, [0, 1, 2], 0.3)
    one, two = cache.v[cache.table[0, 0], 0, 0], cache.v[cache.table[1, 0], :2, 0].astype(np.float64)
    assert np.array_equal(out[0], np.stack([one, one]))
    assert np.allclose(out[1], two.mean(0), rtol=1e-12)


def test_attention_scores_are_pam_products():
    """Values that name their key, power-of-two queries: PAM is then the true
    product, and the outputs are those of ordinary attention (up to the second
    product, exact for values that are powers of two)."""
    rng = np.random.default_rng(5)
    cache = au.Paged(rng, [6], 4, 1, 8, False)
    for j in range(6):
        cache.v[cache.table[0, j // 4], j % 4] = 0.0
        cache.v[cache.table[0, j // 4], j % 4, 0, j] = 2.0 ** (j - 2)
    q = (2.0 ** rng.integers(-2, 2, (3, 1, 8))).astype(np.float32)
    k = cache.k[cache.table[0, np.arange(6) // 4], np.arange(6) % 4, 0].astype(np.float64)
    out, _, _ = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens, [0, 3], 1.0, window=3)
    for t in range(3):
        s = np.exp(q[t, 0] @ k.T)
        s[np.arange(6) > 3 + t] = 0
        s[np.arange(6) <= t] = 0
        assert np.allclose(out[t, 0, :6] / 2.0 ** (np.arange(6) - 2), s / s.sum(), rtol=1e-6)


def test_planted_mistakes_are_seen():
    """The unnormalised form - divide after the second product - is another
    function: far outside the tolerance the kernels are held to."""
    rng = np.random.default_rng(6)
    cache = au.Paged(rng, [40], 16, 1, 16, False)
    q = rng.standard_normal((1, 1, 16)).astype(np.float32)
    out, size, score = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens, [0, 1], 0.25)
    k, v = (c[cache.table[0, np.arange(40) // 16], np.arange(40) % 16, 0] for c in (cache.k, cache.v))
    s = pam_ref.pam_mul_ref(np.broadcast_to(q[0, 0], k.shape), k).astype(np.float64).sum(-1) * 0.25
    e = np.exp(s - s.max()).astype(np.float32)
    late = pam_ref.pam_mul_ref(np.broadcast_to(e[:, None], v.shape), v).astype(np.float64).sum(0) / e.sum()
    assert np.any(np.abs(late - out[0, 0]) > 10 * au.attention_tolerance(size, score, 16, 40)[0, 0])
    true = (np.exp(q[0, 0].astype(np.float64) @ k.T * 0.25)[None] @ v)[0]
    assert np.any(np.abs(true - out[0, 0]) > 10 * au.attention_tolerance(size, score, 16, 40)[0, 0])
