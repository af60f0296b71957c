"""Paged entry points at the edges: queries of any size over 8-bit caches."""
import pytest
import torch

from paged_util import assert_attention, ok, paged_reference, pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["serial", "default"])
def handle(request):
    from paper_2609_21264_b200 import binding
    h = binding.fa_create(flags=binding.FA_FLAG_SERIAL_KERNEL if request.param == "serial" else 0)
    yield h
    binding.fa_destroy(h)


@pytest.mark.parametrize("shift", [-118, -90, 90, 118])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_queries_of_any_size_over_an_8_bit_cache(handle, shift, dqk, dv):
    """Queries of 2^shift against keys whose scale is 2^-shift: ordinary scores from numbers near either end of the range."""
    from paper_2609_21264_b200 import binding as b
    lens = [150, 40]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, True, False, 30)
    q = (torch.randn(2, 8, dqk, generator=torch.Generator().manual_seed(31)) * 2.0 ** shift).to(torch.bfloat16).cuda()
    ks = ks * 2.0 ** -shift
    o, lse = b.forward_paged(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert_attention(o, lse, *paged_reference(q, k, v, ks, vs, table, lens, 1, dqk ** -0.5))
