"""Which product kernels a linear layer launches (CPU: the launches are recorded,
not run)."""
import pytest

import linear_probe as probe
import paper_2305_17190_amd as pam
from long_sum_cases import CASES


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


@pytest.mark.parametrize("m,k,n,form", CASES)
@pytest.mark.parametrize("bf16", [False, True])
def test_long_sums_take_the_form_meant(m, k, n, form, bf16):
    """Running sums in the workspace (at most 512 MiB of them, more tiles in several
    launches), under the plan of the product."""
    tile, kgroups, split, whole, launches = form
    plan = pam.plan(m, n, k)
    assert (plan[:2], plan[3], plan[2] > 1, plan[2] == 1 or plan[4] > 0) == form[:4]
    tiles = -(-m // tile[0]) * -(-n // tile[1])
    items = tiles if not split else plan[4] + (tiles - plan[4]) * plan[2]
    sums = items * kgroups * tile[0] * tile[1] * 4
    layer, product = probe.workspace(m, n, k)
    assert layer == -(-product // 256) * 256 + min(sums, 512 << 20)
    got, count = probe.linear(m, k, n, bf16)
    assert [x.name for x in got] == ["tiled"] * launches + ["reduce"] * split
    assert -(-sums // (512 << 20)) == launches and count == launches + split


@pytest.mark.parametrize("m,k,n", [(4096, 1024, 1024), (8192, 512, 2048), (8, 4096, 512), (1773, 197, 770)])
def test_short_sums_take_no_memory(m, k, n):
    layer, product = probe.workspace(m, n, k)
    assert layer == -(-product // 256) * 256
