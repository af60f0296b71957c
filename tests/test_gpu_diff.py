"""Differential attention over prompts (fa_forward_diff) against the definition in 64 bits."""
import ctypes

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


def heads(B, H, S, g, rows_first):
    x = torch.randn((B, S, H, 128) if rows_first else (B, H, S, 128), generator=g).to(torch.bfloat16).cuda()
    return x.permute(0, 2, 1, 3) if rows_first else x


def run(handle, B, Hq, Hkv, Sq, Sk, causal, weight=True, rows_first=False, seed=1, mult=1.0, lam=None, same=False):
    from paper_2609_21264_b200 import binding
    g = torch.Generator().manual_seed(seed)
    q, k, v = heads(B, Hq, Sq, g, rows_first) * mult, heads(B, Hkv, Sk, g, rows_first), heads(B, Hkv, Sk, g, rows_first)
    if same:                                     # both maps the same
        q[..., 64:] = q[..., :64]
        k[..., 64:] = k[..., :64]
    lam = (torch.rand(Hq, generator=g) * 1.6 - 0.4).cuda() if lam is None else torch.full((Hq,), lam, device="cuda")
    w = (1 + 0.2 * torch.randn(128, generator=g)).cuda() if weight else None
    o = binding.forward_diff(handle, q, k, v, lam, causal=causal, norm_weight=w, eps=1e-5, out_scale=0.7)
    ok(handle)
    assert o.stride() == q.stride()
    last = torch.arange(Sq) + (Sk - Sq) if causal else torch.full((Sq,), Sk)
    for b in range(B):
        for h in range(Hq):
            Y, A = diff_rows(q[b, h].cpu().double(), k[b, h // (Hq // Hkv)].cpu().double(), v[b, h // (Hq // Hkv)].cpu().double(),
                             lam[h].item(), 0.125, last)
            assert_close(o[b, h], *diff_norm(Y, A, w.cpu().double() if weight else None, 1e-5, 0.7), "b%d h%d" % (b, h))


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 300), (128, 128), (129, 129), (200, 333), (333, 200), (127, 640), (500, 500)])
def test_lengths(handle, causal, Sq, Sk):
    run(handle, 1, 2, 1, Sq, Sk, causal, seed=Sq)


@pytest.mark.parametrize("rows_first", [False, True], ids=["bhsd", "bshd"])
@pytest.mark.parametrize("weight", [False, True], ids=["plain", "normed"])
def test_batches_heads_and_layouts(handle, rows_first, weight):
    run(handle, 2, 6, 2, 257, 257, True, weight, rows_first, seed=3)
    run(handle, 3, 3, 3, 130, 190, False, weight, rows_first, seed=4)


def test_large_scores(handle):
    run(handle, 1, 2, 2, 400, 400, True, seed=5, mult=8.0)


def test_equal_maps(handle):
    """Both maps equal: lambda = 0.5 halves the result, lambda = 1 takes it away altogether (compared without normalisation)."""
    run(handle, 1, 2, 1, 300, 300, True, weight=True, seed=6, lam=0.5, same=True)
    run(handle, 1, 2, 1, 300, 300, True, weight=False, seed=7, lam=1.0, same=True)


def test_lambda_zero_is_ordinary_attention_over_the_first_half(handle):
    from paper_2609_21264_b200 import binding
    g = torch.Generator().manual_seed(8)
    q, k, v = heads(1, 4, 400, g, False), heads(1, 2, 400, g, False), heads(1, 2, 400, g, False)
    o = binding.forward_diff(handle, q, k, v, torch.zeros(4, device="cuda"), causal=True)
    q2, k2 = q.clone(), k.clone()
    q2[..., 64:] = 0
    want, _ = binding.forward(handle, q2, k2, v, causal=True, scale=0.125)
    ok(handle)
    # both round P and O once
    d = (o.double() - want.double()).abs()
    assert (d <= 2 * 2.0 ** -8 * want.double().abs() + 2 * 2.0 ** -8 * v.double().abs().max()).all()


def test_many_heads_and_items(handle):
    run(handle, 2, 16, 4, 300, 300, True, seed=9)


def test_captured_and_equal_bits(handle):
    from paper_2609_21264_b200 import binding
    g = torch.Generator().manual_seed(10)
    q, k, v = heads(1, 4, 600, g, True), heads(1, 4, 600, g, True), heads(1, 4, 600, g, True)
    lam, w = torch.rand(4, device="cuda"), torch.rand(128, device="cuda")
    want = binding.forward_diff(handle, q, k, v, lam, causal=True, norm_weight=w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = binding.forward_diff(handle, q, k, v, lam, causal=True, norm_weight=w)
    for _ in range(3):
        o.zero_()
        graph.replay()
        ok(handle)
        assert torch.equal(o, want)


def test_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    g = torch.Generator().manual_seed(11)
    q, k, v = heads(1, 4, 40, g, False), heads(1, 2, 40, g, False), heads(1, 2, 40, g, False)
    lam, o = torch.ones(4, device="cuda"), torch.empty_like(q)
    diff = b.fa_diff(ctypes.sizeof(b.fa_diff), 1e-5, lam.data_ptr(), None, 1.0, 0.0)

    def call(h=handle, d=diff, qp=q.data_ptr(), Hkv=2, dqk=128, dv=128, qs=(4 * 40 * 128, 40 * 128, 128), scale=0.0, Sq=40):
        ks = (2 * 40 * 128, 40 * 128, 128)
        return b.fa_forward_diff(h, qp, k.data_ptr(), v.data_ptr(), o.data_ptr(), 1, 4, Hkv, Sq, 40, dqk, dv, True, scale, d, qs, ks, ks,
                                 (4 * 40 * 128, 40 * 128, 128))

    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call() == b.FA_OK
    assert call(h=None) == bad and call(d=None) == bad and call(qp=None) == bad and call(Hkv=3) == bad and call(dqk=64, dv=64) == no
    assert call(dqk=192) == no and call(qs=(4 * 40 * 128, 40 * 128, 124)) == bad and call(scale=-1.0) == bad and call(Sq=0) == bad
    assert call(d=b.fa_diff(4, 1e-5, lam.data_ptr(), None, 1.0, 0.0)) == bad
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        b.forward_diff(handle, q, k, v[:, :1], lam, causal=True)
    with pytest.raises(ValueError):
        b.forward_diff(handle, q, k, v, lam[:3], causal=True)


def test_prompt_then_tokens_over_the_paged_cache():
    """A prompt through forward_diff and the same tokens one by one through the paged cache give the same rows (to the rounding of
    their probabilities)."""
    from paged_util import BF16_HALF, FP32_SLACK, rope_table
    from paper_2609_21264_b200 import binding as b
    Hq, Hkv, S, page = 4, 2, 45, 16
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.randn(S, H, 128, generator=g).to(torch.bfloat16).cuda() for H in (Hq, Hkv, Hkv))
    lam, w = torch.rand(Hq, device="cuda"), torch.rand(128, device="cuda") + 0.5
    kc, vc = (torch.zeros(3, page, Hkv, 128, dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3) for _ in range(2))
    cache, rope = b.PagedCache(kc, vc), b.Rope(rope_table(S, 64), span=64)        # each map of 64 rotated by itself
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    h = b.fa_create()
    rows = []
    qr = torch.empty_like(q)
    for t in range(S):
        lens = torch.tensor([t + 1], dtype=torch.int32, device="cuda")
        b.append_paged(h, k[t:t + 1], v[t:t + 1], cache, table, lens, q=q[t:t + 1], q_out=qr[t:t + 1], rope=rope)
        rows.append(b.forward_paged_diff(h, qr[t:t + 1], cache, table, lens, lam, norm_weight=w, out_scale=0.8))
    kr = torch.cat([kc[i].transpose(0, 1) for i in (2, 0, 1)])[:S]
    vr = torch.cat([vc[i].transpose(0, 1) for i in (2, 0, 1)])[:S]
    assert torch.equal(vr, v)
    one = lambda x: x.transpose(0, 1)[None]  # noqa: E731
    o = b.forward_diff(h, one(qr), one(kr), one(v), lam, causal=True, norm_weight=w, out_scale=0.8)
    ok(h)
    got = torch.cat(rows)
    for head in range(Hq):
        Y, A = diff_rows(qr[:, head].cpu().double(), kr[:, head // 2].cpu().double(), v[:, head // 2].cpu().double(), lam[head].item(), 0.125,
                         torch.arange(S))
        O, tol = diff_norm(Y, A, w.cpu().double(), 1e-5, 0.8)
        assert_close(got[:, head], O, tol, "paged")
        assert_close(o[0, head], O, tol, "prompt")
    b.fa_destroy(h)


def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers():
    from paper_2609_21264_b200 import binding as b
    g = torch.Generator().manual_seed(13)
    q, k, v = heads(2, 16, 400, g, False), heads(2, 4, 400, g, False), heads(2, 4, 400, g, False)
    lam = torch.rand(16, device="cuda")
    h, fresh = b.fa_create(flags=b.FA_FLAG_DEBUG_DROP_V_LOAD, wait_limit_ms=20), b.fa_create()
    try:
        want = b.forward_diff(fresh, q, k, v, lam, causal=True)
        ok(fresh)
        b.forward_diff(h, q, k, v, lam, causal=True)
        torch.cuda.synchronize()
        st, site = b.fa_last_status(h)
        assert st == b.FA_ERR_DEVICE_TIMEOUT and site != 0
        assert b.fa_debug_set_drop_v_load(h, False) == b.FA_OK
        for _ in range(3):
            o = b.forward_diff(h, q, k, v, lam, causal=True)
            ok(h)
            assert torch.equal(o, want)
    finally:
        b.fa_destroy(h)
        b.fa_destroy(fresh)


def test_a_query_that_is_no_number_shows_in_its_row_alone(handle):
    from paper_2609_21264_b200 import binding as b
    q, k, v = (torch.randn(1, 2, 300, 128, device="cuda").bfloat16() for _ in range(3))
    for half in (3, 100):
        x = q.clone()
        x[0, 1, 170, half] = float("nan")
        o = b.forward_diff(handle, x, k, v, torch.full((2,), 0.5, device="cuda"), causal=True)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_OK, 0)
        assert o[0, 1, 170].isnan().all()
        o[0, 1, 170] = 0
        assert o.isfinite().all()
