"""The Python binding of the attention-side operators around its calls of the
library (CPU: the checks' results and the library are stand-ins)."""
import struct
import sys
import threading
import time

import pytest

torch = pytest.importorskip("torch")

from paper_2305_17190_amd import attention as att  # noqa: E402


@pytest.fixture
def launched(monkeypatch):
    """paged_attention on CPU tensors up to its call of the library: the (max_q,
    max_kv) it hands over and those it sizes the workspace by."""
    seen = []

    def plan(q, k_cache, v_cache, table, kv_lens, q_starts, scale, causal, window, out):
        return b"", (q.shape[2], q.shape[1], k_cache.shape[2], 0, kv_lens.shape[0]), table.shape[1] * k_cache.shape[1]

    def workspace(sizes):
        seen.append(sizes[-2:])
        return 0

    monkeypatch.setattr(att, "_attention_plan", plan)
    monkeypatch.setattr(att, "_calls", {})
    monkeypatch.setattr(att, "_attention_workspace", workspace)
    monkeypatch.setattr(att, "_library", lambda: type("library", (), {"pam_paged_attention": None}))
    monkeypatch.setattr(att, "_bound", None)
    monkeypatch.setattr(att, "_launch", lambda t, fn, args: seen.append(struct.unpack("=iiq", args[-16:])[:2]))
    return seen


def call(tokens, batch, width=3, page=16, **kw):
    cache = torch.zeros(4, page, 1, 8)
    return att.paged_attention(torch.zeros(tokens, 2, 8), cache, cache, torch.zeros(batch, width, dtype=torch.int32),
                               torch.ones(batch, dtype=torch.int32), **kw)


def test_bounds_left_out_hold_for_every_call(launched):
    """Without max_q a sequence may have all of q's tokens, without max_kv all the
    table reaches."""
    starts = torch.tensor([0, 1, 6], dtype=torch.int32)
    call(6, 2, q_starts=starts)
    assert launched == [(6, 48), (6, 48)]
    del launched[:]
    call(6, 2, q_starts=starts, max_q=5, max_kv=20)
    call(2, 2)
    call(2, 2, max_q=7)
    assert launched == [(5, 20), (5, 20), (1, 48), (1, 48), (1, 48), (1, 48)]


def test_a_first_call_is_whole_at_every_step(monkeypatch):
    """Another thread may see the binding between any two steps of a first call:
    what pack goes through must find make."""
    monkeypatch.setattr(att, "_pack_tensors", None)
    monkeypatch.setattr(att, "_make", None)
    steps = []

    def trace(frame, event, arg):
        if frame.f_code is not att._pack.__code__:
            return None
        frame.f_trace_opcodes = True
        if event == "opcode":
            steps.append((att._pack_tensors is not None, att._make is not None))
        return trace

    before = sys.gettrace()
    sys.settrace(trace)
    try:
        assert att._pack(torch.zeros(2)) is not None
    finally:
        sys.settrace(before)
    assert steps[0] == (False, False) and steps[-1] == (True, True)
    assert (True, False) not in steps


def test_other_threads_run_during_the_allocations():
    """With a switch interval past the test's length another thread runs only where
    this one lets go of the interpreter."""
    att._pack(torch.zeros(2))
    like = torch.zeros(4, 3, 8)
    ran, stop = [0], threading.Event()

    def count():
        while not stop.is_set():
            ran[0] += 1
            time.sleep(0)                             # lets go, in turn

    interval = sys.getswitchinterval()
    thread = threading.Thread(target=count, daemon=True)
    sys.setswitchinterval(100)                        # before the thread first waits its turn
    thread.start()
    try:
        kept, before = [], ran[0]                     # kept: a tensor's end lets go as well
        while ran[0] == before and len(kept) < 20000:
            kept.append(att._make(-1, 16, like, None, like))
        assert ran[0] > before
    finally:
        sys.setswitchinterval(interval)
        stop.set()
        thread.join()


def test_what_is_made():
    att._pack(torch.zeros(2))
    like = torch.zeros(4, 3, 8).transpose(0, 1)
    a, none, b, room, addresses = att._make(-1, 48, like, None, like.bfloat16())
    assert none is None and a.shape == b.shape == like.shape and a.is_contiguous() and b.is_contiguous()
    assert (a.dtype, b.dtype, room.dtype, room.numel()) == (torch.float32, torch.bfloat16, torch.uint8, 48)
    assert struct.unpack("=4q", addresses) == (a.data_ptr(), 0, b.data_ptr(), room.data_ptr())
    a, room, addresses = att._make(1, 0, like)
    assert a.dtype == torch.bfloat16 and room is None and struct.unpack("=2q", addresses) == (a.data_ptr(), 0)
    assert att._make(0, 0, like)[0].dtype == torch.float32
    none, room, _ = att._make(0, 16, None)                # no tensor whose device would do
    assert none is None and room is None
    with pytest.raises(TypeError):
        att._make(0, 0, 3)
    with pytest.raises(TypeError):
        att._make(0, 0)
    with pytest.raises(TypeError):
        att._make("float", 0, like)


def test_bounds_past_32_bits(launched, monkeypatch):
    """A reach of 2^31 keys and more bounds lengths that are int32 all the same, a
    window of as many hides nothing; other bounds past the range are refused."""
    windows = []
    plan = att._attention_plan
    monkeypatch.setattr(att, "_attention_plan", lambda *args: windows.append(args[8]) or plan(*args))
    cache = torch.zeros(1, 1, 1, 8).expand(1, 2 ** 30, 1, 8)
    table, lens = torch.zeros(1, 3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    att.paged_attention(torch.zeros(1, 2, 8), cache, cache, table, lens, window=2 ** 40)
    assert launched == [(1, 2 ** 31 - 1)] * 2 and windows == [2 ** 31 - 1]
    for bounds in (dict(max_kv=2 ** 31), dict(max_q=2 ** 32 + 1), dict(max_q=-1), dict(max_kv=-2 ** 40)):
        with pytest.raises(ValueError, match="must be in"):
            call(2, 2, q_starts=torch.tensor([0, 1, 2], dtype=torch.int32), **bounds)
