"""The decoder of examples/: trained on whole sequences, answering from a paged
cache; and the differentiable norm and rotation it is trained with."""
import importlib.util
import os

import numpy as np
import pytest

import attention_util as au
from gpu_util import note, to_dev
from oracle import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def decoder():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder.py")
    spec = importlib.util.spec_from_file_location("pam_decoder_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_learns_and_the_cache_agrees(decoder):
    """Copying is learnt in a few steps from a loss of ln 64 = 4.2; logits are float32
    sums through two layers: 1e-4 of the largest is 1000 roundings."""
    note("decoder example")
    losses, apart = decoder.main(["--steps", "60", "--new", "6"])
    assert losses[0] > 3.5 and losses[-1] < losses[0] - 0.5
    assert apart < 1e-4


@pytest.mark.parametrize("chunk", [1, 5, 64])
def test_chunks_of_any_size_give_the_same_answer(decoder, chunk):
    import torch
    note(f"decoder chunk {chunk}")
    torch.manual_seed(1)
    model = decoder.Decoder(layers=1)
    rng = np.random.default_rng(2)
    prompts = [rng.integers(0, 64, n).tolist() for n in (3, 30, 17)]
    _, seen = decoder.answer(model, prompts, 4, chunk=chunk)
    _, other = decoder.answer(model, prompts, 4, chunk=9)
    assert float((seen - other).abs().max() / other.abs().max()) < 1e-4
    _, half = decoder.answer(model, prompts, 1, chunk=chunk, dtype=torch.bfloat16)
    # Keys and values rounded to 8 bits: relative errors of 2^-9 a value.
    assert float((half[:, 0] - other[:, 0]).abs().max() / other.abs().max()) < 0.05


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norm_rope_under_autograd(dtype):
    """Gradients through views of one projection, and through an output's sum
    (an expanded gradient)."""
    import torch
    from paper_2305_17190_amd.autograd import pam_norm_rope
    note(f"autograd {dtype}")
    bf16 = dtype == "bfloat16"
    rng = np.random.default_rng(3)
    tokens, hq, hk, d = 11, 4, 2, 64
    x = rng.standard_normal((tokens, (hq + hk) * d)).astype(np.float32)
    x = au.bf16(x) if bf16 else x
    wq, wk = ((1 + 0.2 * rng.standard_normal(d)).astype(np.float32) for _ in range(2))
    cos, sin = au.tables(20, d)
    pos = rng.integers(0, 20, tokens).astype(np.int32)
    leaf = to_dev(x).to(getattr(torch, dtype)).requires_grad_()
    weights = [to_dev(w).requires_grad_() for w in (wq, wk)]
    q, k = leaf.view(tokens, hq + hk, d).split((hq, hk), 1)
    zq, zk = pam_norm_rope(q, k, to_dev(pos), to_dev(cos), to_dev(sin), *weights, eps=1e-5)
    (zq.sum() + 2 * zk.sum()).backward()
    got = leaf.grad.float().cpu().numpy().reshape(tokens, hq + hk, d)
    for part, scale, w, grad in ((slice(0, hq), 1, wq, weights[0].grad), (slice(hq, None), 2, wk, weights[1].grad)):
        xs = x.reshape(tokens, hq + hk, d)[:, part]
        dx, dx_size, dw, dw_size = ref.norm_rope_grad(np.full(xs.shape, scale), xs, w, pos, cos, sin, 1e-5, False)
        au.check(got[:, part], dx, 2 * (d + 12) * au.U * dx_size + (2.0 ** -8 * np.abs(dx) if bf16 else 0), "dx")
        n = tokens * xs.shape[1]
        au.check(grad.cpu().numpy(), dw, (n + d / 2 + 12) * au.U * dw_size, "dw")
