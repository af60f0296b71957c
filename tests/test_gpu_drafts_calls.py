"""The Python calls on drafted tokens as a program's other threads and its mistakes meet them."""
import ctypes
import threading
import time

import pytest
import torch

from paged_util import ok, pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    from paper_2609_21264_b200 import binding
    h = binding.fa_create()
    yield h
    binding.fa_destroy(h)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_compaction_asks_how_many_drafts_there_are(handle):
    """Without offsets and without a total nothing says how many drafts there were: refused, not taken for none."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([30, 18], 16, 2, 128, 128, False, False, 9, poison=False)
    cache, k0 = b.PagedCache(k, v), k.clone()
    before = b.fa_launch_count(handle)
    with pytest.raises(ValueError, match="total"):
        b.compact_paged(handle, cache, table, lens_t, ints([[1, 4], [0, 2]]), ints([2, 1]))
    assert b.fa_launch_count(handle) == before and torch.equal(k, k0)
    # a step without drafts says so, an empty batch has nothing to say
    assert b.compact_paged(handle, cache, table, lens_t, ints([[1, 4], [0, 2]]), ints([0, 0]), total=0).tolist() == [30, 18]
    assert b.compact_paged(handle, cache, table[:0], lens_t[:0], ints([[1, 4]])[:0], ints([1])[:0]).shape == (0,)
    ok(handle)
    assert torch.equal(k, k0)


def test_other_threads_run_while_a_call_waits():
    """A launch can wait for a full queue: the calls give the interpreter's lock back meanwhile, as those through ctypes do.  (In the entries'
    place stands a function that sleeps for as many microseconds as the handle says; nothing is launched.)"""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([30, 18], 16, 2, 64, 64, False, False, 10, poison=False)
    cache, rope = b.PagedCache(k, v), b.Rope(torch.zeros(64, 64, device="cuda"))
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    x, keep = ints([0, 1, 2, 3]), ints([[0, 1], [0, 1]])
    torch.cuda.synchronize()
    naps = 400000
    calls = {"tree_layout": lambda: b.tree_layout(naps, x, lens_t), "forward_paged_tree": lambda: b.forward_paged_tree(naps, q, cache, table, lens_t, None),
             "append_paged": lambda: b.append_paged(naps, q, q, cache, table, lens_t, q=q, rope=rope, positions=x),
             "compact_paged": lambda: b.compact_paged(naps, cache, table, lens_t, keep, ints([0, 0]), total=4),
             "copy_pages": lambda: b.copy_pages(naps, cache, x, x)}
    usleep = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value
    device_of = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p)(lambda h: 0)
    stamps, stop = [], threading.Event()

    def other():
        while not stop.is_set():
            time.sleep(0.005)
            stamps.append(time.monotonic())

    thread = threading.Thread(target=other, daemon=True)
    native = b._native()
    try:
        native.bind(ctypes.cast(device_of, ctypes.c_void_p).value, *[usleep] * 5)
        thread.start()
        for name, call in calls.items():
            t0 = time.monotonic()
            call()
            t1 = time.monotonic()
            assert t1 - t0 >= 0.39, name
            ran = sum(1 for s in list(stamps) if t0 + 0.1 < s < t0 + 0.35)
            assert ran >= 5, "%s: the other thread ran %d times" % (name, ran)
    finally:
        stop.set()
        b._native()
        if thread.is_alive():
            thread.join()
