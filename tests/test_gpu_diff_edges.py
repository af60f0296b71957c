"""Differential attention over prompts at the edges of its types: masked values of the largest size, keys that
are no numbers, scores past the largest one, the smallest scales."""

import math

import pytest
import torch

from paged_util import assert_close, diff_norm, diff_rows, ok

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


@pytest.mark.parametrize("column", [5, 90], ids=["map0", "map1"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_a_key_that_is_no_number_shows_wherever_it_stands(handle, column, causal):
    """32 heads, each with its key at another place of a chunk of 32 keys, in other chunks and tiles: every row that sees the key is
    NaN, every other row what it is without it."""
    from paper_2609_21264_b200 import binding as b
    H, S = 32, 300
    q, k, v = inputs(H, S, 20)
    lam = torch.full((H,), 0.5, device="cuda")
    want = b.forward_diff(handle, q, k, v, lam, causal=causal)
    place = [(h * 7 % 9) * 32 + h for h in range(H)]
    assert sorted(j % 32 for j in place) == list(range(32)) and max(place) < S
    for h, j in enumerate(place):
        k[0, h, j, column] = math.nan
    o = b.forward_diff(handle, q, k, v, lam, causal=causal)
    ok(handle)
    for h, j in enumerate(place):
        first = j if causal else 0
        assert o[0, h, first:].isnan().all(), "key %d" % j
        assert torch.equal(o[0, h, :first], want[0, h, :first]), "key %d" % j


@pytest.mark.parametrize("half", [0, 64], ids=["map0", "map1"])
def test_a_score_past_the_largest_number_shows(handle, half):
    """A score of +inf has no softmax in 32 bits: its rows are NaN.  One of -inf weighs nothing."""
    from paper_2609_21264_b200 import binding as b
    H, S = 32, 200
    q, k, v = inputs(H, S, 21)
    lam = torch.full((H,), 0.5, device="cuda")
    q[..., half] = 0.0
    k[..., half] = 0.0
    place = [(h * 5 % 6) * 32 + h for h in range(H)]
    q[0, :, 196, half] = 1e30
    q[0, :, 198, half] = -1e30
    gone = v.clone()
    for h, j in enumerate(place):
        k[0, h, j, half] = 1e30
        gone[0, h, j] = 0
    o = b.forward_diff(handle, q, k, v, lam, causal=True)
    ok(handle)
    assert o[0, :, 196].isnan().all()
    o[0, :, 196] = 0
    assert o.isfinite().all()
    for h, j in enumerate(place):
        Y, A = torch.zeros(1, 128, dtype=torch.float64, device="cuda"), torch.zeros(1, 128, dtype=torch.float64, device="cuda")
        for part, sign in ((slice(0, 64), 1.0), (slice(64, 128), -0.5)):
            z = (q[0, h, 198:199, part].double() @ k[0, h, :199, part].double().T) * 0.125
            p = torch.softmax(z, 1)
            Y += sign * p @ v[0, h, :199].double()
            A += abs(sign) * p @ v[0, h, :199].double().abs()
        assert_close(o[0, h, 198:199], *diff_norm(Y.cpu(), A.cpu(), None, 1e-5, 1.0), "key %d" % j)


@pytest.mark.parametrize("scale", [1e-38, 2e-38, 1e-40, 1e-30])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_the_smallest_scales_weigh_all_keys_alike(handle, scale, causal):
    from paper_2609_21264_b200 import binding as b
    q, k, v = inputs(2, 200, 24)
    lam = torch.tensor([0.3, -0.2], device="cuda")
    o = b.forward_diff(handle, q, k, v, lam, causal=causal, scale=scale)
    ok(handle)
    last = torch.arange(200) if causal else torch.full((200,), 200)
    for h in range(2):
        Y, A = diff_rows(q[0, h].cpu().double(), k[0, h].cpu().double(), v[0, h].cpu().double(), lam[h].item(), scale, last)
        assert_close(o[0, h], *diff_norm(Y, A, None, 1e-5, 1.0), "h%d" % h)
