"""PAM attention over a paged cache on the GPU against the float64 definition."""

import numpy as np
import pytest

import attention_util as au
from gpu_util import device, note, to_dev
from oracle import attention_ref as ref
from oracle import pam_ref

pytestmark = pytest.mark.gpu


def starts_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def run(cache, q, counts=None, bf16_cache=False, bf16_q=False, layout="page", **kw):
    """The call on device copies; layout "head": the pages hold head after head."""
    import torch
    import paper_2305_17190_amd as pam
    caches = []
    for c in (cache.k, cache.v):
        t = to_dev(c)
        t = t.bfloat16() if bf16_cache else t
        if layout == "head":
            t = t.transpose(1, 2).contiguous().transpose(1, 2)
        elif layout == "padded":
            wide = torch.full((t.shape[0], t.shape[1] + 1, t.shape[2], t.shape[3] + 5), float("nan"), dtype=t.dtype,
                              device=t.device)
            wide[:, 1:, :, 3:3 + t.shape[3]] = t
            t = wide[:, 1:, :, 3:3 + t.shape[3]]
        caches.append(t)
    qd = to_dev(q)
    qd = qd.bfloat16() if bf16_q else qd
    if layout == "padded":
        wide = torch.full((q.shape[0], q.shape[1] + 2, q.shape[2] + 1), float("nan"), dtype=qd.dtype, device=qd.device)
        wide[:, 1:-1, 1:] = qd
        qd = wide[:, 1:-1, 1:]
    if counts is not None:
        kw.update(q_starts=to_dev(starts_of(counts)), max_q=kw.get("max_q", max(counts)))
    out = pam.paged_attention(qd, *caches, to_dev(cache.table), to_dev(cache.kv_lens), **kw)
    return out


def compare(cache, q, counts, out, what, scale=None, causal=True, window=0):
    d = q.shape[2]
    want, size, score = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens,
                                      starts_of(counts if counts is not None else [1] * len(cache.kv_lens)),
                                      d ** -0.5 if scale is None else scale, causal, window)
    keys = max([int(n) for n in cache.kv_lens] + [1])
    au.check(out.cpu().numpy(), want, au.attention_tolerance(size, score, d, keys), what)


DECODE = [
    # kv_lens, page, kv heads, group, d
    ([1], 16, 1, 1, 64),
    ([0, 1, 2, 3], 4, 2, 2, 32),
    ([17, 64, 65, 0, 130], 16, 2, 4, 128),
    ([300, 5], 48, 1, 8, 64),
    ([77, 200], 7, 3, 3, 80),
    ([513], 32, 1, 1, 256),
    ([100, 33], 1, 2, 5, 8),
    ([255, 256, 257], 64, 2, 12, 96),
    ([1500, 700], 128, 1, 2, 192),
]


@pytest.mark.parametrize("bf16_cache,bf16_q", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("kv,page,heads,group,d", DECODE)
def test_single_tokens(kv, page, heads, group, d, bf16_cache, bf16_q):
    note(f"decode {kv} page {page} heads {heads}x{group} d {d} bf16 {bf16_cache} {bf16_q}")
    rng = np.random.default_rng(len(kv) * 1000 + d)
    cache = au.Paged(rng, kv, page, heads, d, bf16_cache)
    q = rng.standard_normal((len(kv), heads * group, d)).astype(np.float32) * 2
    q = au.bf16(q) if bf16_q else q
    out = run(cache, q, bf16_cache=bf16_cache, bf16_q=bf16_q)
    compare(cache, q, None, out, "decode")


CHUNKS = [
    # (new tokens, keys) of each sequence, page, kv heads, group, d, causal, window
    ([(1, 1), (3, 9), (7, 7)], 4, 1, 2, 32, True, 0),
    ([(20, 70), (0, 5), (33, 33)], 16, 2, 1, 64, True, 0),
    ([(20, 70), (5, 64)], 16, 1, 4, 64, False, 0),
    ([(40, 150)], 48, 1, 3, 128, True, 33),
    ([(40, 150), (11, 200)], 48, 2, 1, 64, False, 20),
    ([(9, 4), (5, 2)], 4, 1, 2, 64, True, 0),           # more new tokens than keys: the first see none
    ([(30, 290)], 32, 1, 1, 96, True, 1),
    ([(65, 65), (130, 131)], 64, 1, 2, 80, True, 0),
    ([(17, 700)], 128, 1, 8, 256, True, 300),
]


@pytest.mark.parametrize("bf16_cache", [False, True])
@pytest.mark.parametrize("seqs,page,heads,group,d,causal,window", CHUNKS)
def test_chunks(seqs, page, heads, group, d, causal, window, bf16_cache):
    note(f"chunk {seqs} page {page} heads {heads}x{group} d {d} causal {causal} window {window} bf16 {bf16_cache}")
    rng = np.random.default_rng(d + page)
    counts = [n for n, _ in seqs]
    cache = au.Paged(rng, [kv for _, kv in seqs], page, heads, d, bf16_cache)
    q = rng.standard_normal((sum(counts), heads * group, d)).astype(np.float32) * 2
    out = run(cache, q, counts, bf16_cache=bf16_cache, causal=causal, window=window)
    compare(cache, q, counts, out, "chunk", causal=causal, window=window)


@pytest.mark.parametrize("counts", [[1, 1, 1], [5, 3, 40]])
@pytest.mark.parametrize("layout", ["head", "padded"])
@pytest.mark.parametrize("bf16", [False, True])
def test_strides(counts, layout, bf16):
    """Caches stored head by head, and views at odd offsets of wider tensors."""
    note(f"strides {layout} {counts} bf16 {bf16}")
    rng = np.random.default_rng(7)
    cache = au.Paged(rng, [50, 41, 90], 16, 2, 64, bf16)
    q = rng.standard_normal((sum(counts), 4, 64)).astype(np.float32)
    q = au.bf16(q) if bf16 else q
    out = run(cache, q, counts, bf16_cache=bf16, bf16_q=bf16, layout=layout)
    compare(cache, q, counts, out, layout)


@pytest.mark.parametrize("counts", [[1, 1], [24, 40]])
def test_masked_places_have_no_influence(counts):
    """NaN and inf in keys and values that a token does not see: unused slots
    (NaN in every test), keys after its position, before its window, on pages
    that are none."""
    note(f"masked places {counts}")
    rng = np.random.default_rng(8)
    cache = au.Paged(rng, [100, 90], 16, 1, 64, False)
    q = rng.standard_normal((sum(counts), 2, 64)).astype(np.float32)
    clean = run(cache, q, counts, window=60).cpu().numpy()
    # Visible to no token with this window.
    for b, n in enumerate(counts):
        last = int(cache.kv_lens[b]) - n - 60
        for j in range(0, max(last + 1, 0)):
            where = cache.table[b, j // 16], j % 16
            cache.k[where], cache.v[where] = np.nan, (np.inf if j % 2 else np.nan)
    assert np.array_equal(run(cache, q, counts, window=60).cpu().numpy(), clean)
    # The last key is seen by the last token alone: all others stay finite and right.
    j = int(cache.kv_lens[0]) - 1
    cache.v[cache.table[0, j // 16], j % 16] = np.inf
    cache.k[cache.table[0, j // 16], j % 16, 0, 3] = np.nan
    out = run(cache, q, counts, window=60)
    compare(cache, q, counts, out, "last key", window=60)
    got = out.cpu().numpy()
    assert np.isnan(got[counts[0] - 1]).all() and np.isfinite(np.delete(got, counts[0] - 1, 0)).all()


@pytest.mark.parametrize("counts", [[1, 1], [20, 30]])
@pytest.mark.parametrize("bf16", [False, True])
def test_pages_that_are_none(counts, bf16):
    """Table entries outside the cache: their keys are not seen; a token of
    only such keys gets zeros."""
    note(f"no pages {counts} {bf16}")
    rng = np.random.default_rng(9)
    cache = au.Paged(rng, [100, 60], 16, 2, 64, bf16)
    cache.table[0, 2] = -1
    cache.table[0, 4] = cache.k.shape[0]
    cache.table[0, 5] = 2 ** 31 - 1
    cache.table[1, :] = -2 ** 31
    q = rng.standard_normal((sum(counts), 4, 64)).astype(np.float32)
    out = run(cache, q, counts, bf16_cache=bf16)
    compare(cache, q, counts, out, "pages")
    assert np.all(out.cpu().numpy()[counts[0]:] == 0)


@pytest.mark.parametrize("counts", [[1, 1, 1], [6, 25, 70]])
@pytest.mark.parametrize("bf16", [False, True])
def test_special_values(counts, bf16):
    """Zeros, denormals, values near both ends of the range, inf and NaN in
    what the tokens see."""
    note(f"special values {counts} {bf16}")
    rng = np.random.default_rng(10)
    cache = au.Paged(rng, [40, 64, 90], 16, 1, 32, bf16)
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
    q[0, 1, 3] = np.inf if counts[0] > 1 else q[0, 1, 3]
    q[-1, 0, 7] = np.nan
    out = run(cache, q, counts, bf16_cache=bf16)
    compare(cache, q, counts, out, "special")


def test_scores_past_the_range():
    """Scores that overflow give inf (and NaN weights), huge finite ones a
    one-hot row whose output is the value itself, bit for bit."""
    note("huge scores")
    rng = np.random.default_rng(11)
    cache = au.Paged(rng, [30, 30], 16, 1, 16, False)
    q = rng.standard_normal((2, 1, 16)).astype(np.float32)
    q[0] *= 1e6
    q[1] = 2.0 ** 127
    cache.k[cache.table[1, 0]] = np.abs(cache.k[cache.table[1, 0]]) + 4
    cache.k[cache.table[1, 1], :14] = np.abs(cache.k[cache.table[1, 1], :14]) + 4
    out = run(cache, q).cpu().numpy()
    k = np.stack([cache.k[cache.table[0, j // 16], j % 16, 0] for j in range(30)])
    s = pam_ref.pam_mul_ref(np.broadcast_to(q[0, 0], k.shape), k).astype(np.float64).sum(-1)
    j = int(np.argmax(s))
    assert np.sort(s)[-1] - np.sort(s)[-2] > 1e4        # its weight is 1 and all others' 0 in float32
    assert np.array_equal(out[0, 0], cache.v[cache.table[0, j // 16], j % 16, 0])
    assert np.isnan(out[1]).all()


def test_long_contexts_are_split():
    """Splits along the keys, against the definition and against one another."""
    note("long contexts")
    rng = np.random.default_rng(12)
    cache = au.Paged(rng, [5000, 1, 0, 2049], 64, 1, 64, True)
    q = rng.standard_normal((4, 2, 64)).astype(np.float32)
    near = run(cache, q, bf16_cache=True)
    compare(cache, q, None, near, "long")
    wide = np.full((4, 3 * cache.table.shape[1]), -1, np.int32)
    wide[:, :cache.table.shape[1]] = cache.table
    cache.table = wide
    far = run(cache, q, bf16_cache=True)                 # a far bound on the lengths cuts the keys otherwise
    compare(cache, q, None, far, "far bound")


def test_keys_past_max_kv_are_not_seen():
    note("max_kv")
    rng = np.random.default_rng(13)
    cache = au.Paged(rng, [100], 16, 1, 64, False)
    q = rng.standard_normal((1, 1, 64)).astype(np.float32)
    out = run(cache, q, max_kv=40).cpu().numpy()
    cache.kv_lens[:] = 40
    compare(cache, q, None, to_dev(out), "max_kv")


def test_offsets_past_32_bits():
    """Pages more than 2^31 elements (and 2^32 bytes) into the cache."""
    import torch
    import paper_2305_17190_amd as pam
    note("long cache")
    pages, page, heads, d = 2 ** 31 // (64 * 8 * 128) + 40, 64, 8, 128
    dev = device()
    k = torch.zeros(pages, page, heads, d, dtype=torch.bfloat16, device=dev)
    v = torch.zeros_like(k)
    rng = np.random.default_rng(14)
    small = au.Paged(rng, [150, 64], page, heads, d, True, spare=0)
    q = rng.standard_normal((2, 16, d)).astype(np.float32)
    moved = small.table + (pages - small.k.shape[0])
    k[pages - small.k.shape[0]:] = to_dev(small.k).bfloat16()
    v[pages - small.k.shape[0]:] = to_dev(small.v).bfloat16()
    table = np.where(small.table >= 0, moved, -1).astype(np.int32)
    out = pam.paged_attention(to_dev(q), k, v, to_dev(table), to_dev(small.kv_lens))
    compare(small, q, None, out, "long cache")


def test_scale_and_out():
    import torch
    note("scale, out")
    rng = np.random.default_rng(15)
    cache = au.Paged(rng, [70, 12], 16, 2, 64, False)
    q = rng.standard_normal((2, 2, 64)).astype(np.float32)
    for scale in (0.0, -0.7, 3.0):
        wide = torch.full((2, 5, 70), 7.0, device=device())
        out = wide[:, 1:3, 2:66]
        assert run(cache, q, scale=scale, out=out) is out
        compare(cache, q, None, out, f"scale {scale}", scale=scale)
        rest = wide.clone()
        rest[:, 1:3, 2:66] = 7.0
        assert bool((rest == 7.0).all())


def test_tokens_past_max_q_and_of_no_sequence_are_left_alone():
    import torch
    note("max_q")
    rng = np.random.default_rng(16)
    cache = au.Paged(rng, [30, 25], 16, 1, 64, False)
    q = rng.standard_normal((12, 1, 64)).astype(np.float32)
    out = torch.full((12, 1, 64), 7.0, device=device())
    run(cache, q, [4, 6], max_q=4, out=out)              # 10 of 12 tokens; the second sequence's last two past max_q
    got = out.cpu().numpy()
    assert np.all(got[8:] == 7.0) and np.all(got[:8] != 7.0)
    want, size, score = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens, [0, 4, 10], 64 ** -0.5)
    au.check(got[:8], want[:8], au.attention_tolerance(size, score, 64, 30)[:8], "max_q")


def test_starts_out_of_range_stay_in_bounds():
    """Offsets that leave q: the tokens that are there are right, nothing else
    is read or written."""
    import torch
    import paper_2305_17190_amd as pam
    note("starts out of range")
    rng = np.random.default_rng(17)
    cache = au.Paged(rng, [30, 25, 9], 16, 1, 64, False)
    q = to_dev(rng.standard_normal((4, 1, 64)).astype(np.float32))
    out = torch.full((4, 1, 64), 7.0, device=device())
    pam.paged_attention(q, to_dev(cache.k), to_dev(cache.v), to_dev(cache.table), to_dev(cache.kv_lens),
                        q_starts=to_dev(np.array([-3, 2, 1, 900], np.int32)), max_q=8, out=out)
    got = out.cpu().numpy()
    assert np.all(got[0] == 7.0)


@pytest.mark.parametrize("kv,counts", [([3000, 400], None), ([300, 200], [60, 9]), ([700, 650], [300, 250])])
def test_same_bits_every_time_and_on_another_stream(kv, counts):
    import torch
    note(f"streams {kv}")
    rng = np.random.default_rng(18)
    cache = au.Paged(rng, kv, 16, 1, 64, True)
    q = rng.standard_normal((2 if counts is None else sum(counts), 4, 64)).astype(np.float32)
    first = run(cache, q, counts, bf16_cache=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = run(cache, q, counts, bf16_cache=True)
    side.synchronize()
    assert torch.equal(first, other)


@pytest.mark.parametrize("kv,counts", [([5000, 300], None), ([40, 300], None), ([500, 450], [200, 150])])
def test_graph_replays(kv, counts):
    """A captured call, replayed on new inputs with eager work in between."""
    import torch
    import paper_2305_17190_amd as pam
    note(f"graph {kv} {counts}")
    rng = np.random.default_rng(19)
    cache = au.Paged(rng, kv, 16, 2, 64, True)
    tokens = 2 if counts is None else sum(counts)
    kw = {} if counts is None else dict(q_starts=to_dev(starts_of(counts)), max_q=max(counts))
    q = to_dev(rng.standard_normal((tokens, 4, 64)).astype(np.float32))
    args = [to_dev(x).bfloat16() for x in (cache.k, cache.v)] + [to_dev(cache.table), to_dev(cache.kv_lens)]
    pam.paged_attention(q, *args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pam.paged_attention(q, *args, **kw)
    for i in range(4):
        q.copy_(to_dev(rng.standard_normal((tokens, 4, 64)).astype(np.float32)))
        args[3].copy_(to_dev(np.maximum(cache.kv_lens - i, 0)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pam.paged_attention(q, *args, **kw)), i


def test_empty_calls():
    import torch
    import paper_2305_17190_amd as pam
    note("empty")
    dev = device()
    cache = torch.zeros(3, 16, 1, 64, device=dev)
    ints = dict(dtype=torch.int32, device=dev)
    out = pam.paged_attention(torch.zeros(0, 2, 64, device=dev), cache, cache, torch.zeros(0, 2, **ints),
                              torch.zeros(0, **ints))
    assert out.shape == (0, 2, 64)
    # No pages at all, and a table of no width: nothing is seen.
    none = torch.zeros(0, 16, 1, 64, device=dev)
    q = torch.ones(2, 2, 64, device=dev)
    for table in (torch.zeros(2, 3, **ints), torch.zeros(2, 0, **ints)):
        out = pam.paged_attention(q, none, none, table, torch.tensor([0, 5], **ints))
        assert bool((out == 0).all())


def test_random_calls():
    """Sizes drawn at random, across the kernels' ranges of rows and keys."""
    rng = np.random.default_rng(20)
    for i in range(24):
        d = int(rng.choice([8, 24, 64, 72, 96, 128, 160, 256]))
        heads, group = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 7, 8]))
        page = int(rng.choice([1, 5, 16, 32, 60]))
        seqs = []
        for _ in range(int(rng.integers(1, 4))):
            n = int(rng.choice([1, 1, 2, int(rng.integers(3, 40))]))
            seqs.append((n, int(rng.integers(0, 400 if n < 8 else 150))))
        bf16, causal = bool(rng.integers(2)), bool(rng.integers(4))
        window = int(rng.choice([0, 0, int(rng.integers(1, 200))]))
        note(f"random {i}: {seqs} page {page} heads {heads}x{group} d {d} {bf16} {causal} {window}")
        counts = [n for n, _ in seqs]
        cache = au.Paged(rng, [kv for _, kv in seqs], page, heads, d, bf16)
        q = rng.standard_normal((sum(counts), heads * group, d)).astype(np.float32) * 2
        out = run(cache, q, counts, bf16_cache=bf16, causal=causal, window=window)
        compare(cache, q, counts, out, f"random {i}", causal=causal, window=window)


def test_matches_products_with_a_softmax_between():
    """What a layer trained with the batched products computes: the chunk of
    all tokens of a sequence against pam_matmul, softmax, pam_matmul."""
    import torch
    from paper_2305_17190_amd.autograd import pam_matmul
    note("batched products")
    rng = np.random.default_rng(21)
    n, heads, d = 150, 3, 64
    cache = au.Paged(rng, [n], 16, heads, d, False)
    q = rng.standard_normal((n, heads, d)).astype(np.float32)
    out = run(cache, q, [n])
    k, v = (to_dev(c[cache.table[0, np.arange(n) // 16], np.arange(n) % 16]).transpose(0, 1).contiguous()
            for c in (cache.k, cache.v))
    s = pam_matmul(to_dev(q).transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * d ** -0.5
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
    want = pam_matmul(torch.softmax(s, -1), v).transpose(0, 1)
    _, size, score = ref.attention(q, cache.k, cache.v, cache.table, cache.kv_lens, [0, n], d ** -0.5)
    tol = 2 * au.attention_tolerance(size, score, d, n)
    au.check(out.cpu().numpy(), want.cpu().numpy().astype(np.float64), tol, "batched products")
