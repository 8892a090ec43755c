"""Linear layers with sums in parts, by every form of the tiled kernel that takes
them, over several launches too."""
import numpy as np
import pytest

import paper_2305_17190_amd as pam
import training_util as tu
from attention_util import check
from gpu_util import device, note
from long_sum_cases import CASES
from oracle import pam_ref
from test_gpu_linear import same

pytestmark = pytest.mark.gpu


def places(size, tile):
    """Rows (or columns): the ends, the tiles' borders, and some between."""
    borders = [b + d for b in np.linspace(0, size // tile, 8).astype(int) * tile for d in (-1, 0)]
    some = np.concatenate((np.linspace(0, size - 1, 24).astype(int), borders))
    return np.unique(some[(some >= 0) & (some < size)])


@pytest.mark.parametrize("m,k,n,form", CASES)
@pytest.mark.parametrize("bf16", [False, True])
def test_long_sums(m, k, n, form, bf16):
    import torch
    note(f"linear {m}x{k}x{n} bf16 {bf16}, {form}")
    g = torch.Generator(device=device()).manual_seed(m + k + n)
    kind = torch.bfloat16 if bf16 else torch.float32
    x = torch.empty(m, k, device=device(), dtype=kind).normal_(generator=g)
    w = torch.empty(n, k, device=device(), dtype=kind).normal_(0, k ** -0.5, generator=g)
    bias = torch.empty(n, device=device()).normal_(generator=g)
    y = pam.linear(x, w, bias)
    rows, cols = places(m, form[0][0]), places(n, form[0][1])
    want, size = pam_ref.pam_gemm_ref(x[rows].float().cpu().numpy(), w[cols].float().cpu().numpy(), False, True)
    want = want + bias[cols].cpu().numpy().astype(np.float64)
    # Each sum has parts of at most 1024 terms, then as many more roundings as there are
    # parts, groups and slices (k / 1024 and 80 at most).
    tol = (1024 + k / 1024 + 80) * tu.U * size + tu.U * np.abs(want)
    check(y[rows][:, cols].cpu().numpy(), want, tol, "y")
    # Every output: a part left out or taken twice changes it by about sqrt(1024 / k) (the
    # sums are about 1), a chain of 2^16 roundings of partial sums near 1 by sqrt(2^16) / 3
    # units of 2^-24, 5e-6.
    off = (y - pam.gemm(x, w, trans_b=True) - bias).abs()
    assert float(off.max()) <= 0.02 * (1024 / k) ** 0.5
    assert same(pam.linear(x, w, bias), y)
