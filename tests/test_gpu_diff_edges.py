"""Differential attention over prompts at the edges of its types: masked values of the largest size."""

import pytest
import torch

from paged_util import ok

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["serial", "default"])
def handle(request):
    from paper_2609_21264_b200 import binding
    h = binding.fa_create(flags=binding.FA_FLAG_SERIAL_KERNEL if request.param == "serial" else 0)
    yield h
    binding.fa_destroy(h)


def inputs(H, S, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(1, H, S, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(3)]


@pytest.mark.parametrize("S", [101, 140, 300])
def test_masked_values_of_the_largest_size_weigh_nothing(handle, S):
    """The last 20 values are bf16's lowest number.  The rows that do not see them are what they are without them."""
    from paper_2609_21264_b200 import binding as b
    q, k, v = inputs(2, S, 22)
    lam = torch.full((2,), 0.3, device="cuda")
    want = b.forward_diff(handle, q, k, v, lam, causal=True)
    v[:, :, S - 20:] = torch.finfo(torch.bfloat16).min
    o = b.forward_diff(handle, q, k, v, lam, causal=True)
    ok(handle)
    assert torch.equal(o[:, :, :S - 20], want[:, :, :S - 20])


def test_rows_that_see_no_key_are_zero_over_values_of_the_largest_size(handle):
    from paper_2609_21264_b200 import binding as b
    q, k, v = inputs(2, 200, 23)
    v[:] = torch.finfo(torch.bfloat16).min
    o = b.forward_diff(handle, q, k[:, :, :60], v[:, :, :60], torch.full((2,), 0.3, device="cuda"), causal=True)
    ok(handle)
    assert (o[:, :, :140] == 0).all()
