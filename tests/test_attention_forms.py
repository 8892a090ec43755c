"""The cases of attention with few rows take the forms they are named by (CPU:
the launches are recorded, not run)."""
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


@pytest.mark.parametrize("case", cases.OUTSIDE, ids=repr)
def test_cases_take_their_form(case):
    new = max(case.counts)
    assert probe.form(case.d, case.heads, case.group, case.bf16, len(case.seqs), new, case.width * case.page) == (
        case.form, case.fine, rows_of(new * case.group), lanes_of(case.d, case.bf16))
