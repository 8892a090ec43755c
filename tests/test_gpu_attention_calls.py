"""PAM attention over a paged cache: arguments left out and unusual ones."""
import numpy as np
import pytest

import attention_util as au
from gpu_util import note, to_dev
from test_gpu_paged_attention import compare, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,kv", [([3, 9, 1], [9, 60, 30]), ([40, 0, 70], [40, 5, 300]), ([1, 1], [50, 7])])
def test_chunks_without_max_q(counts, kv):
    """No bound on the new tokens: every one of them gets its output."""
    import paper_2305_17190_amd as pam
    note(f"no max_q {counts} {kv}")
    rng = np.random.default_rng(51)
    cache = au.Paged(rng, kv, 16, 2, 64, False)
    q = rng.standard_normal((sum(counts), 4, 64)).astype(np.float32)
    out = pam.paged_attention(to_dev(q), to_dev(cache.k), to_dev(cache.v), to_dev(cache.table), to_dev(cache.kv_lens),
                              to_dev(starts_of(counts)))
    compare(cache, q, counts, out, "no max_q")
