"""PAM attention with few rows a key head in each of its forms (the cases say
which; ``test_attention_forms.py`` holds them to it)."""
import numpy as np
import pytest

import few_rows_cases as cases
from gpu_util import note
from test_gpu_paged_attention import compare, run

pytestmark = pytest.mark.gpu


def result(case, cache, q):
    return run(cache, q, None if max(case.counts) == 1 else case.counts, bf16_cache=case.bf16, **case.kw())


@pytest.mark.parametrize("case", cases.OUTSIDE, ids=repr)
def test_values_of_no_key_have_no_influence(case):
    """Page 0 belongs to no sequence; whatever it holds, the outputs have the same
    bits.  Some pages are none, in the longest sequence more than a wave's keys of
    them in a row."""
    note(f"outside {case}")
    rng = np.random.default_rng(41)
    cache = case.cache(rng)
    cache.table = np.where(cache.table >= 0, cache.table + 1, cache.table).astype(np.int32)
    cache.k, cache.v = (np.concatenate([np.ones_like(c[:1]), c]) for c in (cache.k, cache.v))
    cache.table[0, 4:13] = -1
    cache.table[-1, 0] = -1
    q = case.queries(rng)
    clean = result(case, cache, q)
    compare(cache, q, case.counts, clean, "page 0 of ones", causal=case.causal, window=case.window)
    clean = clean.cpu().numpy().view(np.uint32)
    for value in (np.inf, -np.inf, np.nan):
        cache.k[0], cache.v[0] = value, value
        assert np.array_equal(result(case, cache, q).cpu().numpy().view(np.uint32), clean), value


@pytest.mark.parametrize("case", cases.ROUNDS, ids=repr)
def test_several_rounds(case):
    """Workspaces of more than a round: the units take turns in it."""
    note(f"rounds {case}")
    rng = np.random.default_rng(42)
    cache = case.cache(rng)
    q = case.queries(rng)
    out = result(case, cache, q)
    compare(cache, q, case.counts, out, "rounds", causal=case.causal, window=case.window)
    assert np.array_equal(result(case, cache, q).cpu().numpy(), out.cpu().numpy())
