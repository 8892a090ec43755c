"""8-bit states of averages below 2^-126: the definition takes them for zero."""
import numpy as np

from oracle import training_ref as ref

KW = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, step=1, seed=0, tensor=0)


def step(g, avg_scale=0.0, sq_scale=0.0, code=0):
    n = len(g)
    codes = [np.full(n, code, np.uint8) for _ in "mv"]
    scales = [np.full(-(-n // ref.BLOCK), s, np.float32) for s in (avg_scale, sq_scale)]
    return ref.adamw8(np.ones(n, np.float32), np.asarray(g, np.float32), *codes, *scales, **KW)


def test_squares_below_the_normal_range():
    # g^2 (1 - beta2) crosses 2^-126 at |g| = 3.43e-18.
    p, m, v, ms, vs, by = step([3.4e-18, -3.4e-18, 1e-30])
    assert vs[0] == 0 and not v.any() and ms[0] > 0 and m[0] > 0 and m[1] == m[0] | 128
    assert np.allclose(by[:2], [1e-3 * 3.4e-18 / 1e-8, -1e-3 * 3.4e-18 / 1e-8], rtol=1e-6)
    p, m, v, ms, vs, by = step([3.5e-18, -3.4e-18])
    assert vs[0] > 0 and v[0] > 0 and v[1] == 0


def test_averages_below_the_normal_range():
    # g (1 - beta1) crosses 2^-126 at |g| = 1.18e-37.
    for g, held in ((1.1e-37, False), (1.2e-37, True), (1e-40, False), (-1e-40, False)):
        _, m, v, ms, vs, _ = step([g])
        assert (ms[0] > 0) == held == (m[0] > 0) and vs[0] == 0 and v[0] == 0


def test_scales_below_the_normal_range():
    _, m, v, ms, vs, by = step([0.0, 0.0], 1e-39, 1e-39, 100)
    assert ms[0] == 0 and vs[0] == 0 and not m.any() and not v.any() and not by.any()
    # A code's value is the scale times down to 2^-15.875 (avg), 2^-31.875 (sq).
    _, m, v, ms, vs, by = step([0.0, 0.0], 1e-35, 1e-35, 1)
    assert ms[0] == 0 and vs[0] == 0
