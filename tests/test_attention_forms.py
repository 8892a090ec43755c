"""The cases of attention with few rows take the forms they are named by (CPU:
the launches are recorded, not run)."""
import random

import pytest

import attention_probe as probe
import few_rows_cases as cases


def rows_of(rows):
    return rows if rows <= 4 else 6 if rows <= 6 else 8


def lanes_of(d, bf16):
    lanes = 4
    while lanes * (8 if bf16 else 4) < d:
        lanes *= 2
    return lanes


@pytest.mark.parametrize("case", cases.OUTSIDE + cases.ROUNDS + cases.FINE + cases.WIDE, ids=repr)
def test_cases_take_their_form(case):
    new = max(case.counts)
    assert probe.form(case.d, case.heads, case.group, case.bf16, len(case.seqs), new, case.width * case.page) == (
        case.form, case.fine, rows_of(new * case.group), lanes_of(case.d, case.bf16))


@pytest.mark.parametrize("some", [cases.FINE, cases.WIDE], ids=["fine", "wide"])
def test_cases_reach_every_kernel(some):
    """Rows a unit times lanes a key, in both types and forms."""
    reached = {(case.form, case.bf16, rows_of(max(case.counts) * case.group), lanes_of(case.d, case.bf16))
               for case in some}
    assert reached == {(form, bf16, rows, lanes) for form in ("whole", "split") for bf16 in (False, True)
                       for rows in (1, 2, 3, 4, 6, 8) for lanes in (4, 8, 16, 32) + (() if bf16 else (64,))}


ROUND = 512 << 20


def bounds(case):
    return (case.d, case.heads, case.group, case.bf16, len(case.seqs), max(case.counts), case.width * case.page)


@pytest.mark.parametrize("case", cases.ROUNDS, ids=repr)
def test_rounds_take_every_unit_once(case):
    status, launches = probe.attention(*bounds(case))
    assert status == 0 and len(launches) > 3
    for i, x in enumerate(launches):
        assert x.name == ("scores", "values", "join")[i % 3]
        assert x.units == launches[i - i % 3].units and x.first_unit == sum(y.units for y in launches[:i:3][:i // 3])
    assert sum(x.units for x in launches[::3]) == len(case.seqs) * case.heads


def test_split_workspace_is_bounded_by_a_round_or_a_unit():
    """However far the table reaches: 128 sequences of 8 key heads, 4 rows each,
    over 131072 keys would take 2.3 GiB at once."""
    assert probe.workspace(128, 8, 4, True, 128, 1, 131072) <= ROUND
    rng = random.Random(1)
    seen = 0
    while seen < 500:
        d, heads, group, bf16 = 8 * rng.randint(1, 32), rng.randint(1, 32), rng.randint(1, 16), rng.random() < 0.5
        batch, new, keys = (int(2 ** rng.uniform(0, top)) for top in (12, 4, 24))
        status, launches = probe.attention(d, heads, group, bf16, batch, new, keys)
        assert status == 0
        if launches[0].name != "scores":
            continue
        seen += 1
        x = launches[0]
        one = x.splits * x.rows * (x.split_keys + d + 4) * 4
        assert probe.workspace(d, heads, group, bf16, batch, new, keys) <= max(ROUND * (1 + 4 / (x.split_keys + d)), one) + 16


@pytest.mark.parametrize("keys", [200, 1000, 4000])
def test_launches_stay_below_the_grid_limit(keys):
    """Less than 2^32 threads a launch; the one launch of short contexts has up to
    1024 a workgroup, and with more units is refused."""
    for batch in (1 << 20, (1 << 22) - 1, 1 << 22, (1 << 24) - 1, 1 << 24, 1 << 26):
        status, launches = probe.attention(64, 1, 1, False, batch, 1, keys)
        assert (status == 0) == bool(launches) and status in (0, 1)
        for x in launches:
            groups = x.units * (x.splits if x.name in ("scores", "values") else 1)
            assert groups * x.threads < 1 << 32, (batch, x.name)
            if x.name == "whole":
                assert x.units == batch
    assert probe.attention(64, 1, 1, False, 1 << 26, 1, 1000)[0] == 1      # 16 waves a unit
