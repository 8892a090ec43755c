"""The far tails of the smooth activations: every result from 2^-126 on is there,
though exp(-|x|) or its reciprocal left the float32 range.  Of their slopes those
from 2^-118 on are."""
import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import note, to_dev
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -126     # results below it may be zero
LEAST_SLOPE = 2.0 ** -118

# Around the places where exp(z), its reciprocal or the normal density cross 2^-126, and the steps of the code there.
TAILS = {"silu": (-93.5, -78.0), "gelu": (-13.6, -11.5), "gelu_tanh": (-10.4, -9.2)}


def values(name):
    lo, hi = TAILS[name]
    z = np.linspace(lo, hi, 1536).astype(np.float32)
    edge = np.array([-80, -12, -87.4, -88, -13.2], np.float32)
    return np.concatenate((z, edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(-200)), -z[:100]))


@pytest.mark.parametrize("name", TAILS)
@pytest.mark.parametrize("m", [1, 64, 400])
def test_activation(name, m):
    """Through every product kernel: the values come as the bias of a product of zeros."""
    bias = values(name)
    note(f"tail of {name}, {m} rows")
    y = pam.linear(to_dev(np.zeros((m, 8), np.float32)), to_dev(np.zeros((len(bias), 8), np.float32)), to_dev(bias), name)
    z = np.broadcast_to(bias.astype(np.float64), (m, len(bias)))
    want = ref.activation(z, name)
    check(y.cpu().numpy(), want, tu.activation_error(z, name) - tu.TINY + LEAST, "y")
    # Nothing that float32 holds as a normal number comes as zero.
    held = np.abs(want) >= LEAST * (1 + 1e-4)
    assert (np.abs(want[held]) < 2.0 ** -122).any() and (y.cpu().numpy()[held] != 0).all()


def slope_error(z, name):
    """training_util's; of gelu below 0 both terms are tails, without the 3 u of 1 - Q."""
    err = tu.slope_error(z, name) - tu.TINY
    if name != "gelu":
        return err
    q, bell = ref.normal_below(z), np.abs(z) * np.exp(-z * z / 2) * 0.4
    return np.where(z < 0, ((15 + z * z) * q + bell * (8 + z * z)) * tu.U, err)


@pytest.mark.parametrize("name", TAILS)
@pytest.mark.parametrize("shape", [(1, -1), (7, -1), (-1, 1)])
def test_slope(name, shape):
    z = values(name)
    z = np.tile(z, (shape[0], 1)) if shape[0] > 0 else z.reshape(-1, 1).copy()
    note(f"tail of {name}'s slope, {z.shape}")
    dz, _ = pam.activation_grad(to_dev(np.ones_like(z)), to_dev(z), name)
    z = z.astype(np.float64)
    want = ref.slope(z, name)
    check(dz.cpu().numpy(), want, slope_error(z, name) + tu.U * np.abs(want) + LEAST_SLOPE, "dz")
    held = np.abs(want) >= LEAST_SLOPE * (1 + 1e-4)
    assert (np.abs(want[held]) < 2.0 ** -114).any() and (dz.cpu().numpy()[held] != 0).all()
