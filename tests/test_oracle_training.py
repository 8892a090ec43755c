"""The definitions of the layer-and-step operators against other facts than their
own formulas (CPU)."""
import math
from statistics import NormalDist

import numpy as np
import pytest

import training_util as tu
from oracle import training_ref as ref


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activations_by_hand(name):
    z = np.array([0.0, 1.0, -1.0, 3.0])
    c = math.sqrt(2 / math.pi)
    want = {None: z, "relu": [0, 1, 0, 3], "gelu": [x * NormalDist().cdf(x) for x in z],
            "gelu_tanh": [0.5 * x * (1 + math.tanh(c * (x + 0.044715 * x ** 3))) for x in z],
            "silu": [0.5 * x * (1 + math.tanh(x / 2)) for x in z]}[name]
    assert np.allclose(ref.activation(z, name), want, rtol=1e-12, atol=1e-15)


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_slopes_are_derivatives(name):
    z = np.linspace(-9, 9, 373) + 1e-3
    h = 1e-5
    d = (ref.activation(z + h, name) - ref.activation(z - h, name)) / (2 * h)
    assert np.allclose(ref.slope(z, name), d, rtol=1e-8, atol=1e-9)


def test_special_values():
    z = np.array([np.inf, -np.inf, np.nan])
    for name in ref.ACTIVATIONS:
        got, slope = ref.activation(z, name), ref.slope(z, name)
        assert got[0] == np.inf and np.isnan(got[2])
        assert slope[0] == 1 and slope[1] == (1 if name is None else 0)
        assert np.isnan(slope[2]) == (name in ("gelu", "gelu_tanh", "silu"))


def test_gradient_against_differences():
    rng = np.random.default_rng(0)
    z, dy = rng.standard_normal((5, 7)), rng.standard_normal((5, 7))
    for name in ref.ACTIVATIONS[1:]:
        dz, db = ref.activation_grad(dy, z, name)
        h = 1e-6
        for j in range(7):
            e = np.zeros(7)
            e[j] = h
            d = (dy * (ref.activation(z + e, name) - ref.activation(z - e, name))).sum() / (2 * h)
            assert abs(d - db[j]) < 1e-6
        assert np.allclose(dz.sum(0), db)


def test_adamw_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    p, kw = rng.standard_normal(50), dict(lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    leaf = torch.tensor(p, requires_grad=True)
    optimizer = torch.optim.AdamW([leaf], **kw)
    m, v = np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        norm = ref.grad_norm([g])
        leaf.grad = torch.tensor(g)
        assert abs(float(torch.nn.utils.clip_grad_norm_([leaf], 3.0)) - norm) < 1e-12
        optimizer.step()
        p, m, v = ref.adamw(p, g, m, v, step, limit=ref.clip(norm, 3.0), **kw)
        assert np.allclose(leaf.detach().numpy(), p, rtol=1e-12)


def test_codes():
    """Every code stands for itself; steps of an eighth of an octave from 1 down."""
    for most in (127, 255):
        codes = np.arange(256, dtype=np.uint8)
        values = ref.code_value(codes, np.ones(1, np.float32), most)
        size = np.abs(values[:most + 1])
        assert size[0] == 0 and size[most] == 1.0 and size[most - 8] == 0.5 and size[most - 1] == 0.9375
        assert np.all(np.diff(size) > 0) and size[1] == (1 + (1016 - most + 1) % 8 / 8) * 2.0 ** ((1016 - most + 1) // 8 - 127)
        if most == 127:
            assert np.array_equal(values[128:], -values[:128])
        back, scale = ref.code_of(size, most, np.full(most + 1, 8, np.uint64))
        assert np.array_equal(back, np.arange(most + 1)) and scale[0] == 1


def test_rounding_is_unbiased():
    n = 1 << 16
    x = np.full(n, 0.7, np.float32)
    x[::256] = 1
    for most in (127, 255):
        for bits in ref.random_bits(5, 7, 3, n):
            code, scale = ref.code_of(x, most, bits)
            got = ref.code_value(code, scale, most)[x < 1]
            assert set(np.unique(got)) == {np.float32(0.6875), np.float32(0.75)}
            # 65280 draws of a step of 1/16 with probability 0.2.
            assert abs(got.mean() - 0.7) < 5 * math.sqrt(0.16 / len(got)) / 16


def test_random_bits_differ():
    a, b = ref.random_bits(1, 2, 3, 1000)
    assert len(np.unique(a)) > 950 and len(np.unique(b)) > 950 and a.max() < 1 << 20 and b.min() >= 8
    for other in ((2, 2, 3), (1, 3, 3), (1, 2, 4)):
        assert not np.array_equal(ref.random_bits(*other, 1000)[0], a)


def test_8_bit_averages_follow_32_bit_ones():
    """Over 300 steps the second average stays within a few percent on the mean, and
    nearest rounding would not: a step changes it by 0.1%, a code by 6 to 12%."""
    rng = np.random.default_rng(2)
    n, kw = 1024, dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
    size = np.exp(rng.standard_normal(n)).astype(np.float32)
    p, m, v = np.zeros(n), np.zeros(n), np.zeros(n)
    state = [np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(4, np.float32), np.zeros(4, np.float32)]
    q = np.zeros(n)
    for step in range(1, 301):
        g = (rng.standard_normal(n) * size).astype(np.float32)
        p, m, v = ref.adamw(p, g, m, v, step, **kw)
        q, *state, _ = ref.adamw8(q, g, *state, step=step, seed=1, tensor=0, **kw)
    held = ref.code_value(state[1], state[3], 255)
    assert abs(np.mean(held / v) - 1) < 0.03
    assert np.corrcoef(p, q)[0, 1] > 0.99


@pytest.mark.parametrize("name", ref.ACTIVATIONS[1:])
def test_tolerances_see_planted_mistakes(name):
    """The tanh form of gelu for the exact one, a missing factor of the slope and the
    like lie far outside the tolerances."""
    z = np.linspace(-4, 4, 201)
    for other in ref.ACTIVATIONS:
        if other != name:
            far = np.abs(ref.activation(z, other) - ref.activation(z, name)) > 10 * tu.activation_error(z, name)
            steep = np.abs(ref.slope(z, other) - ref.slope(z, name)) > 10 * tu.slope_error(z, name)
            assert far.sum() > 20 and steep.sum() > 20
