"""Leading dimensions the binding hands to the library (CPU), and what it refuses."""
import pytest
import torch

import dispatch_probe as probe
import paper_2305_17190_amd as pam


@pytest.mark.parametrize("t,ld", [
    (torch.ones(3, 4), 4), (torch.ones(3, 9)[:, 2:5], 9), (torch.ones(4), 4), (torch.ones(3, 0), 1), (torch.ones(0, 3), 3),
    (torch.ones(5, 3, 4), 4), (torch.ones(1, 9)[:, :4], 4)], ids=str)
def test_dense_rows(t, ld):
    assert pam._ld(t.reshape(1, -1) if t.dim() == 1 else t) == ld


@pytest.mark.parametrize("t", [torch.ones(1, 1).expand(7, 1), torch.ones(2, 1, 1).expand(2, 7, 1)], ids=["matrix", "batch"])
def test_an_expanded_column_is_no_dense_one(t):
    """Its elements are one and the same: a leading dimension of 1 would read, or
    write, behind it."""
    assert t.stride(-1) == 1 and pam._ld(t) == 0


@pytest.mark.parametrize("operand", [6, 9, 12])
def test_the_library_refuses_it(operand):
    lib = probe.library()
    args = [0, 1, 7, 7, 1, 1 << 20, 1, 1 << 20, 1, 1 << 20, 7, None]
    assert lib.pam_gemm(*args) == 0
    at = {6: 6, 9: 8, 12: 10}[operand]
    args[at] = 0
    assert lib.pam_gemm(*args) == 1 and b"leading dimension" in lib.pam_last_error()
    probe._launches()
