"""PAM attention with few rows a key head in each of its forms (the cases say
which; ``test_attention_forms.py`` holds them to it)."""
import numpy as np
import pytest

import attention_util as au
import few_rows_cases as cases
from gpu_util import note, to_dev
from test_gpu_paged_attention import compare, run, starts_of

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


@pytest.mark.parametrize("case", cases.FINE + cases.WIDE, ids=repr)
def test_every_kernel(case):
    note(f"{case}")
    rng = np.random.default_rng(43)
    cache = case.cache(rng)
    q = case.queries(rng)
    out = result(case, cache, q)
    compare(cache, q, case.counts, out, "few rows", causal=case.causal, window=case.window)


def last_token(case, b):
    return sum(case.counts[:b + 1]) - 1


@pytest.mark.parametrize("case", cases.CORNERS, ids=repr)
def test_masked_places_of_wide_waves(case):
    """Pages that are none, inf and NaN before every window (unused slots hold NaN
    in every test), and in the last key of every second sequence, which its last
    token alone sees."""
    note(f"masked {case}")
    rng = np.random.default_rng(44)
    cache = case.cache(rng)
    q = case.queries(rng)
    for b, (n, kv) in enumerate(zip(case.counts, case.kv_lens)):
        if b % 4 == 3 and kv > 3 * case.page:
            cache.table[b, [1, 2]] = (-1, cache.k.shape[0])
    clean = result(case, cache, q).cpu().numpy()
    compare(cache, q, case.counts, to_dev(clean), "pages", causal=case.causal, window=case.window)
    if case.window:
        for b, (n, kv) in enumerate(zip(case.counts, case.kv_lens)):
            for j in range(0, max(kv - n - case.window + 1, 0)):
                page = cache.table[b, j // case.page]
                if 0 <= page < cache.k.shape[0]:
                    cache.k[page, j % case.page] = np.nan if j % 3 else np.inf
                    cache.v[page, j % case.page] = np.inf if j % 2 else np.nan
        assert np.array_equal(result(case, cache, q).cpu().numpy(), clean)
    if case.causal:
        for b in range(0, len(case.seqs), 2):
            kv = case.kv_lens[b]
            if kv > case.counts[b]:
                page = cache.table[b, (kv - 1) // case.page]
                if 0 <= page < cache.k.shape[0]:
                    cache.k[page, (kv - 1) % case.page, :, 3] = np.nan
                    cache.v[page, (kv - 1) % case.page, :, 1] = np.inf
        out = result(case, cache, q)
        compare(cache, q, case.counts, out, "last key", causal=case.causal, window=case.window)
        got = out.cpu().numpy()
        seen = np.zeros(len(got), bool)
        for b in range(0, len(case.seqs), 2):
            if case.kv_lens[b] > case.counts[b]:
                seen[last_token(case, b)] = True
        assert np.isnan(got[seen]).all() and np.isfinite(got[~seen]).all()


@pytest.mark.parametrize("case", cases.CORNERS, ids=repr)
def test_special_values_of_wide_waves(case):
    """Zeros, denormals, both ends of the range, inf and NaN in what is seen."""
    note(f"special {case}")
    rng = np.random.default_rng(45)
    cache = case.cache(rng)
    q = case.queries(rng)
    special = np.array([0.0, -0.0, 1e-40, -1e-39, 1.2e-38, 2.0 ** -126, 1e-30, 3e38, -2.0 ** 127, 1e20], np.float32)
    special = au.bf16(special) if case.bf16 else special

    def plant(c, b, j, values):
        c[cache.table[b, j // case.page], j % case.page, 0, :len(values)] = values

    for j in range(0, case.kv_lens[0], 3):
        plant(cache.k, 0, j, special[:7])
        plant(cache.v, 0, j, special)
    plant(cache.v, 3, 60, [np.inf, -np.inf, np.nan])
    plant(cache.k, 3, case.kv_lens[3] - 1, [-np.inf])
    q[0, 0, :5] = special[:5]
    q[last_token(case, 3), -1, 7] = np.nan
    out = result(case, cache, q)
    compare(cache, q, case.counts, out, "special", causal=case.causal, window=case.window)


@pytest.mark.parametrize("case", cases.CORNERS[::3], ids=repr)
@pytest.mark.parametrize("layout", ["head", "padded"])
def test_strides_of_wide_waves(case, layout):
    note(f"strides {layout} {case}")
    rng = np.random.default_rng(46)
    cache = case.cache(rng)
    q = case.queries(rng)
    q = au.bf16(q) if case.bf16 else q
    out = run(cache, q, None if max(case.counts) == 1 else case.counts, bf16_cache=case.bf16, bf16_q=case.bf16,
              layout=layout, **case.kw())
    compare(cache, q, case.counts, out, layout, causal=case.causal, window=case.window)


@pytest.mark.parametrize("case", cases.CORNERS[::3], ids=repr)
def test_wide_waves_in_a_graph_and_on_another_stream(case):
    import torch
    import paper_2305_17190_amd as pam
    note(f"graph {case}")
    rng = np.random.default_rng(47)
    cache = case.cache(rng)
    q = to_dev(case.queries(rng))
    kw = case.kw()
    if max(case.counts) > 1:
        kw.update(q_starts=to_dev(starts_of(case.counts)), max_q=max(case.counts))
    args = [to_dev(x).bfloat16() if case.bf16 else to_dev(x) for x in (cache.k, cache.v)]
    args += [to_dev(cache.table), to_dev(cache.kv_lens)]
    first = pam.paged_attention(q, *args, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = pam.paged_attention(q, *args, **kw)
    side.synchronize()
    assert torch.equal(first, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pam.paged_attention(q, *args, **kw)
    for i in range(4):
        q.copy_(to_dev(case.queries(rng)))
        args[3].copy_(to_dev(np.maximum(cache.kv_lens - i, 0)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pam.paged_attention(q, *args, **kw)), i
