"""Refusals of the attention-side entry points that depend on where an operand's
rows lie, and what stays accepted (CPU: launches are recorded, not run)."""
import itertools
import random

import pytest

import attention_probe as probe
import test_attention_abi as abi
from test_attention_abi import INVALID, NONE, cache, heads

DENSE = dict(page=8192, slot=512, head=64)


def accepted(status):
    launches = probe.take()
    assert (status == 0) == bool(launches)
    return status == 0


@pytest.mark.parametrize("which", ["k_cache_layout", "v_cache_layout"])
@pytest.mark.parametrize("kw", [dict(head=0), dict(slot=0), dict(page=0), dict(head=32), dict(slot=64), dict(page=512),
                                dict(page=8191), dict(slot=64, head=64), dict(slot=511), dict(head=512, slot=512)])
def test_append_refuses_caches_whose_slots_overlap(which, kw):
    lib = probe.library()
    assert abi.append(lib, **{which: cache(**dict(DENSE, **kw))}) == INVALID
    assert b"overlap" in lib.probe_error() and not probe.take()


@pytest.mark.parametrize("kw", [DENSE, dict(page=8192, slot=64, head=1024), dict(page=64, slot=5120, head=640),
                                dict(page=16384, slot=1024, head=128), dict(page=8197, slot=512, head=64),
                                dict(page=0, slot=512, head=64, pages=1), dict(page=64, slot=0, head=1024, size=1, pages=16),
                                dict(page=16, slot=1, head=64, pages=0)])
def test_append_takes_caches_in_any_order_of_dimensions(kw):
    kw = dict(k_cache_layout=cache(**kw), v_cache_layout=cache(**kw))
    if kw["k_cache_layout"].pages == 0:
        kw = dict(k_cache_layout=cache(pages=0), v_cache_layout=cache(pages=0))
    assert accepted(abi.append(probe.library(), **kw))


@pytest.mark.parametrize("call,name", [(abi.norm_rope, "q_out_heads"), (abi.norm_rope, "k_out_heads"),
                                       (abi.grad, "dq_in_heads"), (abi.append, "q_out_heads"), (abi.attention, "out_heads")])
def test_written_heads_of_equal_strides_are_refused(call, name):
    """Token and head strides of one row each: rows (1, 0) and (0, 1) are one."""
    lib = probe.library()
    for bad in (heads(token=64, head=64), heads(token=500, head=64), heads(token=64, head=200), heads(token=128, head=64)):
        assert call(lib, **{name: bad}) == INVALID
        assert b"overlap" in lib.probe_error() and not probe.take()
    for good in (heads(), heads(token=64, head=64 * 40), heads(token=513, head=64), heads(token=2000, head=80)):
        assert accepted(call(lib, **{name: good}))


def test_many_tokens_do_not_pass_the_check_by_overflow():
    lib = probe.library()
    assert abi.attention(lib, tokens=1 << 62, out_heads=heads(token=1 << 31, head=64)) in (0, INVALID)
    probe.take()
    assert abi.attention(lib, tokens=1 << 62, out_heads=heads(token=64, head=1 << 31)) == INVALID


def test_no_accepted_layout_overlaps():
    """Small strides at random against the offsets written."""
    rng = random.Random(2)
    lib, d, seen = probe.library(), 2, [0, 0]
    for _ in range(4000):
        pages, size, count = (rng.randint(1, 4) for _ in range(3))
        strides = [rng.choice((0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48)) for _ in range(3)]
        layout = cache(*strides, pages, size, count)
        ok = accepted(abi.append(lib, d=d, rotation=abi.rotation(rot=0), k_cache_layout=layout, v_cache_layout=layout,
                                 k_heads=heads(64, 2, count), v_heads=heads(64, 2, count), q_in_heads=NONE,
                                 q_out_heads=NONE))
        at = [sum(i * s for i, s in zip(index, strides)) + e
              for index in itertools.product(range(pages), range(size), range(count)) for e in range(d)]
        overlap = len(set(at)) < len(at)
        assert not (ok and overlap), (strides, pages, size, count)
        seen[ok] += 1
    assert min(seen) > 200
