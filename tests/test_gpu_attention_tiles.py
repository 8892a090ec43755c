"""PAM attention in its form of tiles, which the library takes for large calls.
It decides by the bounds ``max_q`` and ``max_kv`` alone, so a table that could
reach far takes short sequences there; each test asks the workspace's size
whether its call did."""

import ctypes

import numpy as np
import pytest

import attention_util as au
from gpu_util import device, note, to_dev
from oracle import attention_ref as ref
from test_gpu_paged_attention import compare, run, starts_of

pytestmark = pytest.mark.gpu


def reach_far(cache, keys, page):
    """Widens the table, by pages that are none, to ``keys`` keys."""
    wide = np.full((cache.table.shape[0], -(-keys // page)), -1, np.int32)
    wide[:, :cache.table.shape[1]] = cache.table
    cache.table = wide


def tile_rows(d, heads, group, bf16, batch, max_q, max_kv):
    """Rows of the call's tiles, 0: it takes none.  Told by the workspace: the
    scores of a round of whole tiles, the values' sums over splits of 128 or 256
    keys, and two numbers a row for 128 keys.  Units of up to 8 rows have splits of 1024
    keys at these sizes."""
    import paper_2305_17190_amd as pam
    device()                                             # torch's HIP runtime, before the library's is looked for
    need = ctypes.c_size_t()
    assert pam.attention._library().pam_paged_attention_workspace_size(
        d, heads * group, heads, 1 if bf16 else 0, batch, max_q, max_kv, ctypes.byref(need)) == 0
    for rows in (128, 64):
        units = batch * heads * -(-max_q * group // rows)
        each = max_kv * rows * 4
        for split in (128, 256):
            size = min(units, max((512 << 20) // each, 1)) * each * (1 + d / split + 1 / 64)
            if 0.99 * size < need.value < 1.01 * size:
                return rows
    return 0


def far_cache(rng, kv_lens, page, heads, d, bf16, keys, max_q, group):
    """A cache whose table reaches far enough that its call takes tiles."""
    cache = au.Paged(rng, kv_lens, page, heads, d, bf16)
    reach_far(cache, keys, page)
    assert tile_rows(d, heads, group, bf16, len(kv_lens), max_q, cache.table.shape[1] * page)
    return cache


CALLS = [
    # (new tokens, keys) of each sequence, page, kv heads, group, d, causal, window, reach of the table
    ([(62, 62), (33, 300), (0, 9), (1, 1)], 16, 1, 1, 64, True, 0, 100000),
    ([(50, 331), (9, 4)], 48, 2, 1, 80, True, 0, 100000),
    ([(20, 290), (17, 129)], 16, 1, 3, 128, False, 0, 100000),
    ([(60, 700)], 128, 1, 2, 32, True, 100, 400000),
    ([(31, 150), (11, 200)], 1, 2, 2, 256, False, 20, 60000),
    ([(64, 513)], 64, 1, 1, 192, True, 1, 200000),
    ([(140, 400), (65, 128)], 32, 2, 1, 64, True, 0, 140000),
    ([(30, 270), (3, 900)], 5, 1, 5, 128, True, 0, 140000),
    ([(33, 200)], 16, 3, 4, 8, True, 50, 600000),
    ([(19, 140), (40, 40)], 7, 1, 7, 136, False, 0, 150000),
]


@pytest.mark.parametrize("bf16_cache,bf16_q", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("seqs,page,heads,group,d,causal,window,reach", CALLS)
def test_chunks(seqs, page, heads, group, d, causal, window, reach, bf16_cache, bf16_q):
    note(f"tiles {seqs} page {page} heads {heads}x{group} d {d} {causal} {window} bf16 {bf16_cache} {bf16_q}")
    rng = np.random.default_rng(d + page)
    counts = [n for n, _ in seqs]
    cache = far_cache(rng, [kv for _, kv in seqs], page, heads, d, bf16_cache, reach, max(counts), group)
    q = rng.standard_normal((sum(counts), heads * group, d)).astype(np.float32) * 2
    q = au.bf16(q) if bf16_q else q
    out = run(cache, q, counts, bf16_cache=bf16_cache, bf16_q=bf16_q, causal=causal, window=window)
    compare(cache, q, counts, out, "tiles", causal=causal, window=window)


def test_both_heights_are_reached():
    rows = {tile_rows(d, heads, group, False, len(seqs), max(n for n, _ in seqs), -(-reach // page) * page)
            for seqs, page, heads, group, d, _, _, reach in CALLS}
    assert rows == {64, 128}


@pytest.mark.parametrize("layout", ["head", "padded"])
@pytest.mark.parametrize("bf16", [False, True])
def test_strides(layout, bf16):
    note(f"tile strides {layout} bf16 {bf16}")
    rng = np.random.default_rng(31)
    counts = [30, 20]
    cache = far_cache(rng, [50, 141], 16, 2, 64, bf16, 100000, max(counts), 2)
    q = rng.standard_normal((sum(counts), 4, 64)).astype(np.float32)
    q = au.bf16(q) if bf16 else q
    out = run(cache, q, counts, bf16_cache=bf16, bf16_q=bf16, layout=layout)
    compare(cache, q, counts, out, layout)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts", [[24, 30], [100, 80]])
def test_masked_places_have_no_influence(counts, d):
    """NaN and inf before the windows, after the rows' positions and in unused
    slots (NaN in every test)."""
    note(f"tile masked places {counts} {d}")
    rng = np.random.default_rng(32)
    cache = far_cache(rng, [300, 190], 16, 1, d, False, 100000, max(counts), 2)
    q = rng.standard_normal((sum(counts), 2, d)).astype(np.float32)
    clean = run(cache, q, counts, window=60).cpu().numpy()
    for b, n in enumerate(counts):
        for j in range(0, max(int(cache.kv_lens[b]) - n - 59, 0)):
            where = cache.table[b, j // 16], j % 16
            cache.k[where], cache.v[where] = np.nan, (np.inf if j % 2 else np.nan)
    assert np.array_equal(run(cache, q, counts, window=60).cpu().numpy(), clean)
    # The last key is seen by the last token alone.
    j = int(cache.kv_lens[0]) - 1
    cache.v[cache.table[0, j // 16], j % 16] = np.inf
    cache.k[cache.table[0, j // 16], j % 16, 0, 3] = np.nan
    out = run(cache, q, counts, window=60)
    compare(cache, q, counts, out, "last key", window=60)
    got = out.cpu().numpy()
    assert np.isnan(got[counts[0] - 1]).all() and np.isfinite(np.delete(got, counts[0] - 1, 0)).all()


@pytest.mark.parametrize("bf16", [False, True])
def test_pages_that_are_none(bf16):
    note(f"tile pages {bf16}")
    rng = np.random.default_rng(33)
    counts = [60, 30]
    cache = far_cache(rng, [290, 60], 16, 2, 64, bf16, 100000, max(counts), 2)
    cache.table[0, [2, 9]] = -1
    cache.table[0, 4] = cache.k.shape[0]
    cache.table[0, 5] = 2 ** 31 - 1
    cache.table[1, :] = -2 ** 31
    q = rng.standard_normal((sum(counts), 4, 64)).astype(np.float32)
    out = run(cache, q, counts, bf16_cache=bf16)
    compare(cache, q, counts, out, "pages")
    assert np.all(out.cpu().numpy()[counts[0]:] == 0)


@pytest.mark.parametrize("counts", [[6, 25, 70], [40, 64, 50]])
@pytest.mark.parametrize("bf16", [False, True])
def test_special_values(counts, bf16):
    """Zeros, denormals, both ends of the range, inf and NaN in what is seen."""
    note(f"tile special values {counts} {bf16}")
    rng = np.random.default_rng(34)
    cache = far_cache(rng, [40, 64, 90], 16, 1, 32, bf16, 300000, max(counts), 2)
    special = np.array([0.0, -0.0, 1e-40, -1e-39, 1.2e-38, 2.0 ** -126, 1e-30, 3e38, -2.0 ** 127, 1e20],
                       np.float32)
    special = au.bf16(special) if bf16 else special

    def plant(c, b, j, values):
        c[cache.table[b, j // 16], j % 16, 0, :len(values)] = values

    for j in range(0, 40, 3):
        plant(cache.k, 0, j, special[:7])
        plant(cache.v, 0, j, special)
    plant(cache.v, 1, 5, [np.inf, -np.inf, np.nan])
    plant(cache.k, 2, 50, [-np.inf])
    q = rng.standard_normal((sum(counts), 2, 32)).astype(np.float32)
    q[0, 0, :5] = special[:5]
    q[0, 1, 3] = np.inf
    q[-1, 0, 7] = np.nan
    out = run(cache, q, counts, bf16_cache=bf16)
    compare(cache, q, counts, out, "special")


def test_steep_rows():
    """Probabilities that span the whole range, down to zero."""
    note("tile steep rows")
    rng = np.random.default_rng(35)
    counts = [50, 20]
    cache = far_cache(rng, [200, 260], 16, 1, 64, False, 100000, max(counts), 2)
    q = rng.standard_normal((sum(counts), 2, 64)).astype(np.float32) * 20
    out = run(cache, q, counts)
    compare(cache, q, counts, out, "steep")


def test_several_rounds():
    """Scores of more than a round's workspace: the units take turns in it."""
    import torch
    note("tile rounds")
    rng = np.random.default_rng(36)
    counts = [40, 0, 64, 21, 9]
    cache = far_cache(rng, [300, 50, 64, 700, 9], 1024, 1, 64, True, 1200000, max(counts), 1)
    max_kv = cache.table.shape[1] * 1024
    assert 5 * max_kv * 64 * 4 > 2 * (512 << 20)
    q = rng.standard_normal((sum(counts), 1, 64)).astype(np.float32)
    out = run(cache, q, counts, bf16_cache=True)
    compare(cache, q, counts, out, "rounds")
    assert torch.equal(out, run(cache, q, counts, bf16_cache=True))


def test_tokens_past_max_q_and_starts_out_of_range():
    """Tokens of no sequence keep what they had; offsets that leave q touch
    nothing else."""
    import torch
    note("tile max_q")
    rng = np.random.default_rng(37)
    cache = far_cache(rng, [130, 225], 16, 1, 64, False, 200000, 58, 1)
    q = rng.standard_normal((96, 1, 64)).astype(np.float32)
    out = torch.full((96, 1, 64), 7.0, device=device())
    run(cache, q, [60, 40], max_q=58, out=out)           # the second ends past the 96 tokens there are
    got = out.cpu().numpy()
    whole = np.concatenate([q, np.zeros((4, 1, 64), np.float32)])
    want, size, score = ref.attention(whole, cache.k, cache.v, cache.table, cache.kv_lens, [0, 60, 100], 64 ** -0.5)
    tol = au.attention_tolerance(size, score, 64, 225)
    seen = np.r_[0:58, 60:96]
    au.check(got[seen], want[seen], tol[seen], "max_q")
    assert np.all(got[58:60] == 7.0)


@pytest.mark.parametrize("counts", [[30, 25], [130, 90]])
def test_another_stream_and_graph_replays(counts):
    import torch
    import paper_2305_17190_amd as pam
    note(f"tile streams and graphs {counts}")
    rng = np.random.default_rng(38)
    cache = far_cache(rng, [500, 450], 16, 2, 64, True, 100000, max(counts), 2)
    q = to_dev(rng.standard_normal((sum(counts), 4, 64)).astype(np.float32))
    kw = dict(q_starts=to_dev(starts_of(counts)), max_q=max(counts))
    args = [to_dev(x).bfloat16() for x in (cache.k, cache.v)] + [to_dev(cache.table), to_dev(cache.kv_lens)]
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
        q.copy_(to_dev(rng.standard_normal(tuple(q.shape)).astype(np.float32)))
        args[3].copy_(to_dev(np.maximum(cache.kv_lens - i, 0)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pam.paged_attention(q, *args, **kw)), i
