"""The Python calls on drafted tokens without a GPU."""
import types

import pytest
import torch

from paper_2609_21264_b200 import binding as b


def test_compaction_asks_how_many_drafts_there_are():
    """No offsets and no total: nothing says how many drafts the sequences have.  (Looked at before the tensors' devices.)"""
    x = torch.zeros(2, dtype=torch.int32)
    cache = types.SimpleNamespace(address=0, index=0, count=1)
    call = lambda **kw: b.compact_paged(0, cache, x.view(2, 1), x, x.view(2, 1), x, **kw)  # noqa: E731
    with pytest.raises(ValueError, match="total"):
        call()
    with pytest.raises(ValueError, match="total"):
        call(total=None)
    for kw in ({"total": 2}, {"total": 0}, {"cu_seqlens": torch.zeros(3, dtype=torch.int32)}):
        with pytest.raises(ValueError, match="block_table"):         # (the next thing that is wrong here)
            call(**kw)
