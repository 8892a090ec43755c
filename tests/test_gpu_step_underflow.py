"""AdamW steps whose averages come near the end of the float32 range: 8-bit codes
and scales bit for bit, 32-bit states by the definition with zeros below 2^-126."""
import numpy as np
import pytest

import paper_2305_17190_amd as pam
from attention_util import bf16, check
from gpu_util import note, to_dev
import training_util as tu
from oracle import training_ref as ref

pytestmark = pytest.mark.gpu

KW = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.05)


def gradients(n, seed):
    """Magnitudes from 1e-45 to 1e-15, a decade or so to a block, zeros among them."""
    rng = np.random.default_rng([n, seed])
    size = 10.0 ** (rng.uniform(-45, -15, -(-n // 256)).repeat(256)[:n] + rng.uniform(-1, 1, n))
    return (rng.choice([-1, 0, 1], n, p=[0.45, 0.1, 0.45]) * size).astype(np.float32)


@pytest.mark.parametrize("n", [1, 255, 256 * 40 + 9, 300000])
@pytest.mark.parametrize("grad_bf16", [False, True])
@pytest.mark.parametrize("limit", [False, True])
def test_codes(n, grad_bf16, limit):
    import torch
    note(f"adamw 8 bits near 2^-126, {n} values, bf16 {grad_bf16}, limit {limit}")
    p0 = np.ones(n, np.float32)
    blocks = -(-n // 256)
    rng = np.random.default_rng(n)
    # Held from before: codes of all kinds, scales from denormal to 1e-25.
    state = [rng.integers(0, 256, n).astype(np.uint8) for _ in "mv"]
    state += [(10.0 ** rng.uniform(-44, -25, blocks)).astype(np.float32) for _ in "mv"]
    p, *d = (to_dev(x) for x in (p0, *state))
    for step in (1, 2, 3):
        g = gradients(n, step)
        g = bf16(g) if grad_bf16 else g
        gd = to_dev(g).to(torch.bfloat16 if grad_bf16 else torch.float32)
        norm = torch.full((), 3.0, device=p.device) if limit else None
        pam.adamw_step([p], [gd], [d[0]], [d[1]], step, **KW, avg_scales=[d[2]], sq_scales=[d[3]], norm=norm,
                       max_norm=1.0 if limit else None)
        f = tu.norm_limit(3.0, 1.0)[0] if limit else None
        want = ref.adamw8(p0, g, *state, step=step, seed=0, tensor=0, limit=f, **KW)
        for got, w_, what in zip(d, want[1:5], ("avg", "sq", "avg_scale", "sq_scale")):
            assert np.array_equal(got.cpu().numpy(), w_), f"{what}, step {step}"
        tol = np.abs(want[5]) * 12 * tu.U + 3 * tu.U + tu.TINY
        check(p.cpu().numpy(), want[0], tol, f"p, step {step}")
        p0, state = p.cpu().numpy(), list(want[1:5])


@pytest.mark.parametrize("grad_bf16", [False, True])
def test_32_bits(grad_bf16):
    import torch
    n = 256 * 40 + 9
    note(f"adamw 32 bits near 2^-126, bf16 {grad_bf16}")
    g = gradients(n, 0)
    g = bf16(g) if grad_bf16 else g
    p, m, v = (to_dev(x) for x in (np.ones(n, np.float32), np.zeros(n, np.float32), np.zeros(n, np.float32)))
    pam.adamw_step([p], [to_dev(g).to(torch.bfloat16 if grad_bf16 else torch.float32)], [m], [v], 1, **KW)
    f, n_ = np.float32, ref.normal
    m1 = n_(n_(g) * f(1 - 0.9))
    v1 = n_(n_(n_(g) * f(1 - 0.999)) * n_(g))
    # Each is one fused operation on a zero and a product, itself rounded once: the same number.
    assert np.array_equal(m.cpu().numpy(), m1) and np.array_equal(v.cpu().numpy(), v1)
    want, by = ref.moved(np.ones(n), m1.astype(np.float64), v1.astype(np.float64), 1, *(KW[k] for k in (
        "lr", "betas", "eps", "weight_decay")))
    check(p.cpu().numpy(), want, np.abs(by) * 12 * tu.U + 3 * tu.U + tu.TINY, "p")
