"""Which product kernels a linear layer launches (CPU: the launches are recorded,
not run)."""
import pytest

import linear_probe as probe


@pytest.mark.parametrize("m", [2, 33, 500, 4096, 65536])
@pytest.mark.parametrize("k", [1, 16, 100, 512, 4096])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("ldy", [1, 7])
def test_one_output_is_one_row_of_weights(m, k, bf16, ldy):
    """The few rows are the weights', also where y's rows are one value apart: as
    columns of few rows of x, the bias would be read past its one value."""
    launches, count = probe.linear(m, k, 1, bf16, ldy)
    assert count == 1
    assert launches[0].name != "few rows" or not launches[0].few_rows_of_a
    if k in (512, 4096) and m <= 4096:
        assert launches[0].name == "few rows"


@pytest.mark.parametrize("m,k,n,of_x", [(1, 512, 1, True), (1, 512, 2, True), (2, 512, 2, True), (3, 512, 2, False),
                                        (8, 4096, 512, True), (512, 4096, 8, False)])
def test_the_shorter_side_is_few(m, k, n, of_x):
    launches, count = probe.linear(m, k, n)
    assert count == 1 and launches[0].name == "few rows" and bool(launches[0].few_rows_of_a) == of_x
