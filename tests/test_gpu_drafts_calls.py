"""The Python calls on drafted tokens as a program's other threads and its mistakes meet them."""
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
