"""The gradient of norm and rotation over so many rows that each workgroup works
through several: the loads ahead of the row at hand, positions among them, and
the sums of the weights' gradient over a workgroup's rows and over more than 256
workgroups.  A launch has about 1024 workgroups; every size here gives each
between two and five turns, the last of them not a full one, in all widths of a
lane's loads."""
import numpy as np
import pytest

import attention_util as au
from gpu_util import note, to_dev
from oracle import attention_ref as ref
from test_gpu_heads import EPS, Inputs, tensor

pytestmark = pytest.mark.gpu

SIZES = [
    # tokens, query heads, key heads, d, rot        values a load (float32, bfloat16)
    (9000, 8, 3, 64, 64),                         # 4, 8
    (9001, 6, 1, 128, 64),                        # 4, 8
    (12007, 2, 1, 256, 256),                      # 4, 8
    (9999, 4, 1, 96, 8),                          # 4, 4
    (11000, 3, 2, 72, 36),                        # 2, 2
    (2100, 5, 2, 250, 6),                         # 1, 1
]


def inputs(tokens, hq, hk, d, rot, bf16):
    """Every token at a position of its own."""
    s = Inputs(tokens, hq, hk, d, rot, bf16, seed=7, rows=tokens + 5)
    s.pos = s.rng.permutation(tokens + 5)[:tokens].astype(np.int32)
    return s


def check(got, dz, x, w, s, d, bf16, interleaved):
    """got: (dx, dweight); the tolerances of the gradient's other tests."""
    dx, dx_size, dw, dw_size = ref.norm_rope_grad(dz, x, w, s.pos, s.cos, s.sin, EPS, interleaved)
    tol = 2 * (d + 12) * au.U * dx_size + (2.0 ** -8 * np.abs(dx) if bf16 else 0) + 2.0 ** -126
    au.check(got[0].float().cpu().numpy(), dx, tol, "dx")
    n = x.shape[0] * x.shape[1]
    if w is None:
        assert got[1] is None
    else:
        au.check(got[1].cpu().numpy(), dw, (n + d / 2 + 12) * au.U * dw_size + 2.0 ** -126 * n, "dweight")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", SIZES)
def test_gradient_of_many_rows(tokens, hq, hk, d, rot, bf16, interleaved):
    import paper_2305_17190_amd as pam
    note(f"many rows {tokens} {hq} {hk} {d} {rot} {bf16} {interleaved}")
    s = inputs(tokens, hq, hk, d, rot, bf16)
    got = pam.norm_rope_grad(tensor(s.dq, bf16), tensor(s.dk, bf16, True), tensor(s.q, bf16, True), tensor(s.k, bf16),
                             **s.kw(interleaved))
    check(got[::2], s.dq, s.q, s.wq, s, d, bf16, interleaved)
    check(got[1::2], s.dk, s.k, s.wk, s, d, bf16, interleaved)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("weights", [False, True])
def test_one_side_of_many_rows(weights, bf16):
    """All workgroups on one operand; without weights the rotation alone."""
    import paper_2305_17190_amd as pam
    note(f"one side of many rows {weights} {bf16}")
    s = inputs(9001, 6, 1, 128, 128, bf16)
    got = pam.norm_rope_grad(tensor(s.dq, bf16), None, tensor(s.q, bf16), None, **s.kw(False, weights))
    assert got[1] is None and got[3] is None
    check(got[::2], s.dq, s.q, s.wq if weights else None, s, 128, bf16, False)


@pytest.mark.parametrize("bf16", [False, True])
def test_positions_of_many_rows(bf16):
    """A position without a table row: NaN in its own token's rows alone, and so
    in the weights' gradients."""
    import paper_2305_17190_amd as pam
    note(f"positions of many rows {bf16}")
    s = inputs(9000, 8, 3, 64, 32, bf16)
    bad = s.rng.choice(9000, 40, replace=False)
    s.pos[bad] = s.rng.choice([-1, 9005, 2 ** 31 - 1], 40)
    gq, gk, gqw, gkw = pam.norm_rope_grad(tensor(s.dq, bf16), tensor(s.dk, bf16), tensor(s.q, bf16), tensor(s.k, bf16),
                                          **s.kw(False))
    for g in (gq, gk):
        nan = np.isnan(g.float().cpu().numpy())
        assert nan[bad].all() and not np.delete(nan, bad, 0).any()
    for g in (gqw, gkw):
        assert np.array_equal(np.isnan(g.cpu().numpy()), np.arange(64) < 32)
