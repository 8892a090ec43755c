"""Expanded columns are refused, as other overlapping rows are, before a launch."""
import pytest

import paper_2305_17190_amd as pam
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def test_expanded_columns():
    import torch
    note("expanded columns, refused")
    one = torch.ones(1, 1, device=device()).expand(7, 1)
    col, row = torch.ones(7, 1, device=device()), torch.ones(1, 7, device=device())
    for bad in (lambda: pam.gemm(one, row), lambda: pam.gemm(col, one, trans_b=True), lambda: pam.gemm(col, torch.ones(1, 1, device=device()), out=one),
                lambda: pam.bmm(one.expand(2, 7, 1), row.expand(2, 1, 7)),
                lambda: pam.exact_grad(one, torch.ones(1, 3, device=device()), torch.ones(7, 3, device=device()))):
        with pytest.raises(pam.PamError, match="leading dimension"):
            bad()


def test_one_row_of_any_stride():
    """A single row's stride is never taken."""
    import torch
    note("one row of any stride")
    a, b = torch.randn(1, 40, device=device()), torch.randn(40, 30, device=device())
    want = pam.gemm(a, b)
    for strange in (a.as_strided((1, 40), (0, 1)), a.as_strided((1, 40), (1 << 40, 1)), a.as_strided((1, 40), (3, 1))):
        assert torch.equal(pam.gemm(strange, b), want)
