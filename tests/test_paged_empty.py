"""An empty batch through the argument checks of the paged calls, without a GPU."""
import types

import pytest
import torch

from paper_2609_21264_b200 import binding

bf16 = torch.bfloat16


def cache():
    return types.SimpleNamespace(device=torch.device("cpu"), dqk=128, dv=64)


def seqs(B):
    return binding.fa_paged_seqs(0, B, None, 1, None, 1, 0)


def test_no_sequences_and_no_tokens_is_a_call_of_nothing():
    Hq, T, Sq, strides, out = binding._paged_out(torch.empty(0, 8, 128, dtype=bf16), cache(), seqs(0), None)
    assert (Hq, T, Sq) == (8, 0, 1) and out.shape == (0, 8, 64) and out.dtype == bf16
    assert all(x > 0 and x % 8 == 0 for x in strides)
    given = torch.empty(0, 8, 64, dtype=bf16)
    assert binding._paged_out(torch.empty(5, 8, 128, dtype=bf16)[:0], cache(), seqs(0), given)[4] is given


@pytest.mark.parametrize("T,B", [(3, 0), (0, 2), (3, 2)])
def test_tokens_that_do_not_go_round_the_sequences_are_refused(T, B):
    with pytest.raises(ValueError, match="every sequence"):
        binding._paged_out(torch.empty(T, 8, 128, dtype=bf16), cache(), seqs(B), None)
