"""fa_forward_paged_tree with more than 32 rows, where the calls of other tests are few rows or say nothing about the kernel: every test looks
at the name of the kernel that ran."""
import pytest
import torch

from draft_util import tree_reference
from paged_util import assert_attention, ok, pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    from paper_2609_21264_b200 import binding
    h = binding.fa_create()
    yield h
    binding.fa_destroy(h)


def kernel_was(handle, rows, e4m3):
    from paper_2609_21264_b200 import binding
    assert binding.fa_last_kernel_name(handle) == ("fa_tree_few" if rows <= 32 else "fa_tree") + ("_e4m3" if e4m3 else "")


@pytest.mark.parametrize("n", [5, 11], ids=["20rows", "44rows"])
@pytest.mark.parametrize("q_exp,k_exp", [(-120, -24), (-126, -60), (-120, -100)])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_a_score_factor_below_the_normal_numbers(handle, n, q_exp, k_exp, dqk, dv):
    """Queries and scales so small that their product is 0 in 32 bits: all scores are equal, and what a row does not see stays hidden."""
    from paper_2609_21264_b200 import binding as b
    lens = [150, 40]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, True, False, 40)
    q = (torch.randn(2 * n, 8, dqk, generator=torch.Generator().manual_seed(41)) * 2.0 ** q_exp).to(torch.bfloat16).cuda()
    ks = ks * 2.0 ** k_exp
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    kernel_was(handle, 4 * n, True)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, lens, [0, n, 2 * n], [torch.ones(n, n).tril() > 0] * 2, dqk ** -0.5))
