"""Paged entry points at the edges: queries of any size over 8-bit caches, statuses of several kinds, empty
batches, precision of the difference of two maps."""
import pytest
import torch

from paged_util import assert_attention, assert_close, ok, paged_reference, pool

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


def bad_append(h):
    """An append into a page that the pool does not have."""
    from paper_2609_21264_b200 import binding as b
    k, v = (torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    b.append_paged(h, x, x, b.PagedCache(k, v), torch.full((1, 1), 7, dtype=torch.int32, device="cuda"),
                   torch.ones(1, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


@pytest.mark.parametrize("order", ["timeout first", "timeout last"])
def test_a_wait_that_ran_out_is_not_hidden_by_bad_contents(order):
    """A launch that gave up (its first V tiles are left out) and one that met a page outside the pool, before the status is read: the
    status is the one that makes every result doubtful."""
    from paper_2609_21264_b200 import binding as b
    lens = [700, 40]
    k, v, table, lens_t, _, _ = pool(lens, 16, 2, 128, 128, False, False, 32)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    cache = b.PagedCache(k, v)
    h = b.fa_create(flags=b.FA_FLAG_DEBUG_DROP_V_LOAD, wait_limit_ms=20)
    try:
        if order == "timeout last":
            bad_append(h)
        b.forward_paged(h, q, cache, table, lens_t)
        torch.cuda.synchronize()
        if order == "timeout first":
            bad_append(h)
        st, site = b.fa_last_status(h)
        assert st == b.FA_ERR_DEVICE_TIMEOUT and site != 0 and site >> 8 != 9
        assert b.fa_last_status(h) == (b.FA_OK, 0)       # one reading clears both
        bad_append(h)
        assert b.fa_last_status(h) == (b.FA_ERR_INVALID_ARG, 0x0902)
        assert b.fa_last_status(h) == (b.FA_OK, 0)
        assert b.fa_debug_set_drop_v_load(h, False) == b.FA_OK
        o, lse = b.forward_paged(h, q, cache, table, lens_t)
        ok(h)
        assert_attention(o, lse, *paged_reference(q, k, v, None, None, table, lens, 1, 128 ** -0.5))
    finally:
        b.fa_destroy(h)


def test_counters_are_back_before_the_next_launch_on_any_stream():
    """fa_last_status puts the counters back that a launch which gave up left half-way; the next launch, on a stream that does not wait for the
    default one, finds them so."""
    from paper_2609_21264_b200 import binding as b
    lens = [700, 3000, 40]
    k, v, table, lens_t, _, _ = pool(lens, 16, 2, 128, 128, False, False, 36)
    q = torch.randn(3, 8, 128, device="cuda").bfloat16()
    cache, side = b.PagedCache(k, v), torch.cuda.Stream()
    h = b.fa_create(wait_limit_ms=20)
    try:
        want = b.forward_paged(h, q, cache, table, lens_t)
        ok(h)
        for _ in range(3):
            assert b.fa_debug_set_drop_v_load(h, True) == b.FA_OK
            with torch.cuda.stream(side):
                b.forward_paged(h, q, cache, table, lens_t)
            torch.cuda.synchronize()
            assert b.fa_debug_set_drop_v_load(h, False) == b.FA_OK
            assert b.fa_last_status(h)[0] == b.FA_ERR_DEVICE_TIMEOUT
            with torch.cuda.stream(side):
                o, lse = b.forward_paged(h, q, cache, table, lens_t)
            ok(h)
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    finally:
        b.fa_destroy(h)


def test_counters_of_a_new_handle_are_there_for_its_first_launch_on_any_stream():
    from paper_2609_21264_b200 import binding as b
    lens = [700, 3000, 40]
    k, v, table, lens_t, _, _ = pool(lens, 16, 2, 128, 128, False, False, 37)
    q = torch.randn(3, 8, 128, device="cuda").bfloat16()
    cache, side, want = b.PagedCache(k, v), torch.cuda.Stream(), None
    torch.cuda.synchronize()
    for _ in range(10):
        h = b.fa_create()
        with torch.cuda.stream(side):
            o, _ = b.forward_paged(h, q, cache, table, lens_t)
        ok(h)
        want = o if want is None else want
        assert torch.equal(o, want)
        b.fa_destroy(h)
    assert_attention(want, None, *paged_reference(q, k, v, None, None, table, lens, 1, 128 ** -0.5))


@pytest.mark.parametrize("max_pages", [0, 3])
def test_an_empty_batch_through_the_binding(handle, max_pages):
    """A server that has drained its batch goes on making the same calls."""
    from paper_2609_21264_b200 import binding as b
    k, v, _, _, _, _ = pool([20], 16, 2, 128, 128, False, False, 33)
    cache, before = b.PagedCache(k, v), b.fa_launch_count(handle)
    none = dict(dtype=torch.int32, device="cuda")
    table, lens, cu = torch.empty(0, max_pages, **none), torch.empty(0, **none), torch.zeros(1, **none)
    rows = lambda H: torch.empty(0, H, 128, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for offsets in (None, cu):
        out = b.append_paged(handle, rows(2), rows(2), cache, table, lens, cu_seqlens=offsets, q=rows(8))
        assert out.shape == (0, 8, 128)
    o, lse = b.forward_paged(handle, rows(8), cache, table, lens)
    assert o.shape == (0, 8, 128) and o.dtype == torch.bfloat16 and lse.shape == (8, 0)
    given = rows(8)
    assert b.forward_paged(handle, rows(8), cache, table, lens, out=given, want_lse=False) == (given, None)
    assert b.forward_paged_diff(handle, rows(8), cache, table, lens, torch.ones(8, device="cuda")).shape == (0, 8, 128)
    ok(handle)
    assert b.fa_launch_count(handle) == before
    with pytest.raises(ValueError):
        b.forward_paged(handle, torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda"), cache, table, lens)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[333, 64], [5000, 90]], ids=["whole", "split"])
def test_differential_probabilities_keep_their_bits_where_the_maps_are_nearly_equal(handle, e4m3, lens):
    """Maps that differ little, lambda close to 1: what is left of the difference is as small as one bf16 rounding of the
    probabilities.  Over a bf16 cache they keep two bf16 terms (2^-16 of the value), over an 8-bit one three e5m2 terms behind a rounding to
    fp16 (2^-8 + 2^-11, and 2^-27 of the largest weight).  With A = sum_j (p1 + lambda p2) |v_j| the other errors are: a score, 64
    products added with up to 2^-23 of their sizes' sum z each, turns into a relative error 64 * 2^-23 * z of its probability, with room for
    the exponential, the references and the division in z + 1; n / 16 additions to the accumulator, 2^-23 each; the output's bf16."""
    from paged_util import diff_rows, rows_of, softmax64
    from paper_2609_21264_b200 import binding as b
    Hq, Hkv = 8, 2
    k, v, table, lens_t, ks, vs = pool(lens, 16, Hkv, 128, 128, e4m3, False, 34)
    raw = k.view(torch.uint8) if e4m3 else k
    raw[..., 64:] = raw[..., :64].clone()
    q = torch.randn(2, Hq, 128, generator=torch.Generator().manual_seed(35))
    q[..., 64:] = q[..., :64] * (1 + 2.0 ** -6)
    q = q.to(torch.bfloat16).cuda()
    lam = torch.full((Hq,), 0.998, device="cuda")
    o = b.forward_paged_diff(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, lam, out_scale=0.5)
    ok(handle)
    one_term = 0.0
    for i, n in enumerate(lens):
        kd, vd, last = rows_of(k, ks, table, i, n), rows_of(v, vs, table, i, n), torch.tensor([n - 1])
        for h in range(Hq):
            x, kh, vh, lm = q[i:i + 1, h].cpu().double(), kd[h // 4], vd[h // 4], lam[h].item()
            y, a = diff_rows(x, kh, vh, lm, 0.125, last)
            z = max((x[:, s].abs() @ kh[:, s].abs().T).max().item() * 0.125 for s in (slice(0, 64), slice(64, 128)))
            tol = (2.0 ** -23 * (64 * (z + 1) + n / 8 + 32) + (2.0 ** -8 + 2.0 ** -11 if e4m3 else 2.0 ** -16)) * a
            if e4m3:
                tol = tol + 2.0 ** -26 * vh.abs().sum(0)
            tol = 0.5 * tol + 2.0 ** -8 * (0.5 * y).abs() + 1e-30
            assert_close(o[i, h], 0.5 * y[0], tol[0], "sequence %d head %d" % (i, h))
            # what one bf16 term would have given is outside of that
            p1, p2 = (softmax64(x[:, s], kh[:, s], 0.125, last)[0] for s in (slice(0, 64), slice(64, 128)))
            cut = lambda p: (p / p.max()).to(torch.bfloat16).double() * p.max()  # noqa: E731
            one_term = max(one_term, (((cut(p1) - lm * cut(p2)) @ vh - y).abs() * 0.5 / tol).max().item())
    assert e4m3 or one_term > 1.5
