"""Attention and differential attention of the last tokens over a paged cache, against the definition in 64 bits.

Unused slots of the pages hold NaN and infinities, unused block table entries numbers that are no pages."""
import ctypes

import pytest
import torch

from paged_util import assert_attention, assert_close, diff_norm, diff_rows, ok, paged_reference, pool, rope_table, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["serial", "default"])
def handle(request):
    from paper_2609_21264_b200 import binding
    h = binding.fa_create(flags=binding.FA_FLAG_SERIAL_KERNEL if request.param == "serial" else 0)
    yield h
    binding.fa_destroy(h)


def run(handle, lens, Sq, Hq, Hkv, dqk, dv, page, e4m3=False, heads_first=False, seed=1, q_mult=1.0, shift=0.0, scale=0.0):
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, dqk, dv, e4m3, heads_first, seed, shift=shift)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(len(lens) * Sq, Hq, dqk, generator=g) * q_mult).to(torch.bfloat16).cuda()
    o, lse = binding.forward_paged(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, scale=scale)
    ok(handle)
    O, L, A = paged_reference(q, k, v, ks, vs, table, lens, Sq, scale or dqk ** -0.5)
    return assert_attention(o, lse, O, L, A), (q, k, v, ks, vs, table, lens_t, o, lse)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (3, 3), (14, 2), (16, 1)], ids=["g4", "g1", "g7", "g16"])
def test_lengths_around_tiles_and_pages(handle, dqk, dv, e4m3, Hq, Hkv):
    run(handle, [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 700], 1, Hq, Hkv, dqk, dv, 16, e4m3, heads_first=e4m3, seed=dqk + Hq)


@pytest.mark.parametrize("page", [16, 32, 48, 80, 128, 176, 256, 1024])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_page_sizes(handle, page, e4m3):
    run(handle, [1, 300, 47, 1100], 1, 8, 2, 128, 128, page, e4m3, heads_first=not e4m3, seed=page)


@pytest.mark.parametrize("Sq", [2, 3, 8, 16])
@pytest.mark.parametrize("dqk,dv,Hq,Hkv", [(128, 128, 8, 2), (64, 64, 14, 2), (192, 128, 4, 4), (128, 128, 16, 1)], ids=["d128", "d64", "d192", "mqa"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_several_new_tokens(handle, Sq, dqk, dv, Hq, Hkv, e4m3):
    """Causal among the new tokens; sequences shorter than Sq leave the first rows without a key."""
    run(handle, [Sq, Sq - 1, 0, 128, 129, 127 + Sq, 500], Sq, Hq, Hkv, dqk, dv, 32, e4m3, seed=Sq)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_one_long_sequence_and_many_short_ones(handle, e4m3):
    run(handle, [20000], 1, 8, 1, 128, 128, 64, e4m3, seed=5)
    run(handle, [(i * 53) % 260 for i in range(333)], 1, 2, 2, 64, 64, 16, e4m3, seed=6)
    run(handle, [3000] + [3] * 40 + [9000], 1, 8, 2, 128, 128, 16, e4m3, seed=7)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_large_scores_and_rising_maxima(handle, e4m3):
    """Scores in the hundreds (a softmax of a few keys) and keys whose scores rise along the sequence, so that the reference
    maximum moves again and again."""
    from paper_2609_21264_b200 import binding
    # (8-bit and 16-bit inputs are exact; a score of size s carries an fp32 error of about s * 2^-22, far below the slack at 300)
    run(handle, [1000, 77], 1, 8, 2, 128, 128, 16, e4m3, seed=8, q_mult=8.0)
    k, v, table, lens_t, ks, vs = pool([2000], 32, 2, 128, 128, e4m3, False, 9, poison=False)
    flat = torch.arange(2000, device="cuda")
    ramp = (flat.float() / 2000 * 4 - 2)
    kk = torch.zeros(k.shape, device="cuda")
    kk[table[0, flat // 32].long(), :, flat % 32] = ramp[:, None, None].expand(2000, 2, 128)
    k.copy_((kk * 20).to(k.dtype) if e4m3 else kk.to(k.dtype))
    q = torch.ones(1, 8, 128, device="cuda").bfloat16()
    q[:, ::2] *= -1
    o, lse = binding.forward_paged(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert_attention(o, lse, *paged_reference(q, k, v, ks, vs, table, [2000], 1, 128 ** -0.5))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_one_key_far_above_many_small_ones(handle, e4m3):
    """A key of weight about one half and thousands whose weights, each 2^-14 of it, make up the other half: the small ones
    keep their precision."""
    from paper_2609_21264_b200 import binding
    n = 16000
    k, v, table, lens_t, ks, vs = pool([n], 64, 1, 128, 128, e4m3, False, 10, poison=False, shift=0.5)
    one = 20.0 if e4m3 else 1.0
    k.copy_(torch.zeros(k.shape, device="cuda").to(k.dtype))
    kf = torch.zeros(k.shape, device="cuda")
    kf[int(table[0, 3]), 0, 5, :] = one
    k.copy_(kf.to(k.dtype))
    q = torch.zeros(1, 4, 128, device="cuda")
    q[:] = 9.7 * 128 ** 0.5 / 128
    q = q.bfloat16()
    o, lse = binding.forward_paged(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert_attention(o, lse, *paged_reference(q, k, v, ks, vs, table, [n], 1, 128 ** -0.5))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_queries_of_mixed_size(handle, e4m3):
    """Entries of a query spread over 2^20: the 8-bit terms of a query follow its largest entry."""
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, ks, vs = pool([400, 130], 16, 2, 128, 128, e4m3, False, 11)
    g = torch.Generator().manual_seed(12)
    q = torch.randn(2, 8, 128, generator=g) * 2.0 ** torch.randint(-20, 1, (2, 8, 128), generator=g)
    q[:, 1] *= 1e-3
    q[:, 2] *= 50
    q[:, 3] = 0
    q = q.to(torch.bfloat16).cuda()
    o, lse = binding.forward_paged(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert_attention(o, lse, *paged_reference(q, k, v, ks, vs, table, [400, 130], 1, 128 ** -0.5))


def run_diff(handle, lens, Sq, Hq, Hkv, page, e4m3=False, weight=True, seed=1, heads_first=False):
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, 128, 128, e4m3, heads_first, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(len(lens) * Sq, Hq, 128, generator=g).to(torch.bfloat16).cuda()
    lam = (torch.rand(Hq, generator=g) * 1.6 - 0.4).cuda()
    w = (1 + 0.2 * torch.randn(128, generator=g)).cuda() if weight else None
    o = binding.forward_paged_diff(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, lam, norm_weight=w, eps=1e-5, out_scale=0.7)
    ok(handle)
    Y, A = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b, n in enumerate(lens):
        kd, vd, here = rows_of(k, ks, table, b, n), rows_of(v, vs, table, b, n), slice(b * Sq, (b + 1) * Sq)
        for h in range(Hq):
            y, a = diff_rows(q[here, h].cpu().double(), kd[h // (Hq // Hkv)], vd[h // (Hq // Hkv)], lam[h].item(), 0.125, torch.arange(n - Sq, n))
            Y[here, h], A[here, h] = y, a
    assert_close(o, *diff_norm(Y, A, w.cpu().double() if weight else None, 1e-5, 0.7))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,Sq", [(8, 2, 1), (4, 4, 1), (16, 1, 1), (8, 2, 5), (16, 1, 16), (12, 2, 3)])
@pytest.mark.parametrize("weight", [False, True], ids=["plain", "normed"])
def test_differential(handle, e4m3, Hq, Hkv, Sq, weight):
    run_diff(handle, [0, 1, 17, 128, 129, 300, 2100], Sq, Hq, Hkv, 16, e4m3, weight, seed=Hq + Sq, heads_first=e4m3)


def test_strides_and_outputs_beside_other_data(handle):
    """q as a slice of one projection, O in the middle of a wider buffer that must stay as it was; no lse."""
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, _, _ = pool([100, 33, 0], 16, 2, 128, 128, False, False, 20)
    x = torch.randn(3, 12, 128, device="cuda").bfloat16()
    buf = torch.full((5, 10, 136), 3.0, dtype=torch.bfloat16, device="cuda")
    out = buf[1:4, 1:9, :128]
    o, lse = binding.forward_paged(handle, x[:, 2:10], binding.PagedCache(k, v), table, lens_t, out=out, want_lse=False)
    ok(handle)
    assert o is out and lse is None
    O, L, A = paged_reference(x[:, 2:10], k, v, None, None, table, [100, 33, 0], 1, 128 ** -0.5)
    assert_attention(out, None, O, L, A)
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[1:4, 1:9, :128] = False
    assert (buf[keep] == 3.0).all()


def test_shared_pages_and_repeated_calls_are_bit_equal(handle):
    """Two sequences whose first pages are the same ones; equal calls give equal bits, whatever ran in between."""
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, _, _ = pool([5000, 5000, 640], 64, 2, 128, 128, False, False, 21, poison=False)
    table[1, :40] = table[0, :40]
    table[2, :10] = table[0, :10]
    q = torch.randn(3, 16, 128, device="cuda").bfloat16()
    cache = binding.PagedCache(k, v)
    first = binding.forward_paged(handle, q, cache, table, lens_t)
    ok(handle)
    assert_attention(*first, *paged_reference(q, k, v, None, None, table, [5000, 5000, 640], 1, 128 ** -0.5))
    run(handle, [900, 31], 1, 8, 2, 64, 64, 16, seed=22)
    for _ in range(5):
        again = binding.forward_paged(handle, q, cache, table, lens_t)
        ok(handle)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("Hq,Hkv,dqk,dv,page,e4m3,diff", [(32, 8, 128, 128, 16, False, False), (32, 8, 128, 128, 64, True, False),
                                                          (16, 16, 192, 128, 48, False, False), (14, 2, 64, 64, 32, False, False),
                                                          (16, 4, 128, 128, 32, False, True), (16, 4, 128, 128, 32, True, True)])
def test_a_serving_batch_fills_the_gpu_and_repeats_bit_for_bit(Hq, Hkv, dqk, dv, page, e4m3, diff):
    """Lengths from 65 to 4096 that end anywhere in a tile, more row blocks than SMs, every page slot poisoned that is not a key's:
    against the plain kernel, and ten times the same bits (loads of K and V that overtake one another show here)."""
    from paper_2609_21264_b200 import binding as b
    lens = [65 + (i * 7919 + 4201) % 4032 for i in range(48)]
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, dqk, dv, e4m3, False, 60)
    q = torch.randn(48, Hq, dqk, device="cuda").bfloat16()
    lam, w = torch.rand(Hq, device="cuda"), torch.rand(128, device="cuda")
    cache = b.PagedCache(k, v, ks, vs)

    def call(h):
        if diff:
            return b.forward_paged_diff(h, q, cache, table, lens_t, lam, norm_weight=w), None
        return b.forward_paged(h, q, cache, table, lens_t)

    plain, h = b.fa_create(flags=b.FA_FLAG_SERIAL_KERNEL), b.fa_create()
    try:
        want, want_lse = call(plain)
        o, lse = call(h)
        ok(plain)
        ok(h)
        # both round once to bf16, the streaming kernel rounds its probabilities too: a row's values differ by less than that of the
        # largest of them
        scale = want.double().abs().amax(-1, keepdim=True)
        assert ((o.double() - want.double()).abs() <= 4 * 2.0 ** -8 * scale).all()
        if lse is not None:
            assert (lse - want_lse).abs().max() <= 3e-4
        for _ in range(10):
            again, again_lse = call(h)
            ok(h)
            assert torch.equal(again, o) and (lse is None or torch.equal(again_lse, lse))
    finally:
        b.fa_destroy(plain)
        b.fa_destroy(h)


def test_captured_step_with_the_append_follows_growing_lengths(handle):
    """One decode step (append with rotation, then attention), captured once and replayed while the sequences grow, against the
    eager calls on a copy."""
    from paper_2609_21264_b200 import binding
    lens0, Hq, Hkv, page = [3, 130, 0, 47], 8, 2, 16
    k, v, table, lens, _, _ = pool([n + 8 if n else 0 for n in lens0], page, Hkv, 128, 128, False, False, 30, poison=False)
    table = table.clamp(0, k.shape[0] - 1)
    tab = rope_table(256, 128)
    x = torch.randn(4, Hq + 2 * Hkv, 128, device="cuda").bfloat16()
    lens.copy_(torch.tensor(lens0, dtype=torch.int32))
    rope = binding.Rope(tab)

    def step(kc, vc):
        cache = binding.PagedCache(kc, vc)
        qr = binding.append_paged(handle, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], cache, table, lens, q=x[:, :Hq], rope=rope)
        return binding.forward_paged(handle, qr, cache, table, lens)

    k2, v2 = k.clone(), v.clone()
    step(k2.clone(), v2.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step(k, v)
    for i in range(6):
        lens.copy_(torch.tensor([n + i + 1 if n else 0 for n in lens0], dtype=torch.int32))
        x.copy_(torch.randn_like(x))
        graph.replay()
        ok(handle)
        oe, le = step(k2, v2)
        ok(handle)
        assert torch.equal(o, oe) and torch.equal(lse, le) and torch.equal(k, k2) and torch.equal(v, v2)
        assert (o[2] == 0).all() and torch.isneginf(lse[:, 2]).all()
    now = [n + 6 if n else 0 for n in lens0]
    qr = binding.append_paged(handle, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], binding.PagedCache(k, v), table, lens, q=x[:, :Hq], rope=rope)
    assert_attention(o, lse, *paged_reference(qr, k, v, None, None, table, now, 1, 128 ** -0.5))


def test_another_stream(handle):
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, _, _ = pool([700, 64], 16, 2, 128, 128, False, True, 40)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    cache = binding.PagedCache(k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = binding.forward_paged(handle, q, cache, table, lens_t)
    side.synchronize()
    ok(handle)
    assert_attention(o, lse, *paged_reference(q, k, v, None, None, table, [700, 64], 1, 128 ** -0.5))


def test_contents_the_device_refuses(handle):
    """Pages outside the pool and lengths the block table cannot hold are reported; nothing outside the pool is read, the
    other sequences' rows are right, and the handle goes on working."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([500, 40, 300], 16, 2, 128, 128, False, False, 50)
    q = torch.randn(3, 8, 128, device="cuda").bfloat16()
    cache = b.PagedCache(k, v)
    bad = table.clone()
    bad[0, 3], bad[0, 9] = -5, 2 ** 31 - 1
    o, lse = b.forward_paged(handle, q, cache, bad, lens_t)
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0902)
    O, L, A = paged_reference(q, k, v, None, None, table, [500, 40, 300], 1, 128 ** -0.5)
    assert_attention(o[1:], lse[:, 1:], O[1:], L[:, 1:], A[1:])
    far = lens_t.clone()
    far[1], far[2] = -3, 2 ** 30
    o, lse = b.forward_paged(handle, q, cache, table.clamp(0, k.shape[0] - 1), far)
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0901)
    assert_attention(o[:1], lse[:, :1], O[:1], L[:, :1], A[:1])
    o, lse = b.forward_paged(handle, q, cache, table, lens_t)
    ok(handle)
    assert_attention(o, lse, O, L, A)


def test_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens, _, _ = pool([20], 16, 2, 64, 64, False, False, 5)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    o, lam = torch.empty_like(q), torch.ones(4, device="cuda")
    cache = b.PagedCache(k, v)
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 1, table.data_ptr(), table.shape[1], lens.data_ptr(), table.shape[1], 0)

    def call(h=handle, qp=q.data_ptr(), op=o.data_ptr(), Hq=4, Sq=1, scale=0.0, qs=(256, 64), s=seqs, c=cache.c):
        return b.fa_forward_paged(h, c, s, qp, op, None, Hq, Sq, scale, qs, (256, 64))

    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call() == b.FA_OK
    assert call(h=None) == bad and call(qp=None) == bad and call(op=o.data_ptr() + 2) == bad and call(Hq=3) == bad and call(Sq=0) == bad
    assert call(Sq=b.FA_PAGED_MAX_SQ + 1) == no and call(scale=-1.0) == bad and call(scale=float("nan")) == bad and call(qs=(256, 60)) == bad
    diff = b.fa_diff(ctypes.sizeof(b.fa_diff), 1e-5, lam.data_ptr(), None, 1.0, 0.0)
    dcall = lambda d: b.fa_forward_paged_diff(handle, cache.c, seqs, q.data_ptr(), o.data_ptr(), 4, 1, 0.0, d, (256, 64), (256, 64))  # noqa: E731
    assert dcall(diff) == no                                   # two maps of 64 need heads of 128
    assert dcall(None) == bad and dcall(b.fa_diff(ctypes.sizeof(b.fa_diff), 1e-5, None, None, 1.0, 0.0)) == bad
    assert dcall(b.fa_diff(ctypes.sizeof(b.fa_diff), 0.0, lam.data_ptr(), lam.data_ptr(), 1.0, 0.0)) == bad
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        b.forward_paged(handle, q.float(), cache, table, lens)
    with pytest.raises(ValueError):
        b.forward_paged(handle, torch.cat([q, q, q]), cache, table.expand(2, -1).contiguous(), lens.expand(2).contiguous())
    with pytest.raises(b.FaError):
        b.forward_paged(handle, q[:, :3], cache, table, lens)
    with pytest.raises(ValueError):
        b.forward_paged_diff(handle, q, cache, table, lens, lam[:2])


def test_prompts_then_tokens_step_by_step():
    """The operators as a server uses them: ragged prompts are appended (rotated on the way) and attended to in one packed call, then
    four tokens a sequence are appended and attended to one at a time; every row against attention in 64 bits over the sequence's
    whole history, rotated in 64 bits from what was appended."""
    from paged_util import BF16_HALF, FP32_SLACK, rope_table, softmax64, turned
    from paper_2609_21264_b200 import binding as b
    Hq, Hkv, d, page = 8, 2, 128, 16
    prompts, steps = [37, 150, 16], 4
    B, G = len(prompts), 4
    final = [n + steps for n in prompts]
    k, v, table, _, _, _ = pool(final, page, Hkv, d, d, False, False, 70)
    cache, tab = b.PagedCache(k, v), rope_table(256, d)
    rope, cu = b.Rope(tab), torch.tensor([0, 37, 187, 203], dtype=torch.int32, device="cuda")
    history = [torch.zeros(0, Hq + 2 * Hkv, d, dtype=torch.float64) for _ in range(B)]
    h = b.fa_create()

    def check(seq, rows, o, lse):
        x = history[seq]
        n = x.shape[0]
        q, _ = turned(x[:, :Hq], tab[:n].cpu().double(), d, 0, d, False)
        kk, _ = turned(x[:, Hq:Hq + Hkv], tab[:n].cpu().double(), d, 0, d, False)
        for head in range(Hq):
            # queries and keys as they are after their rounding to bf16
            p, L = softmax64(q[n - rows:, head].bfloat16().double(), kk[:, head // G].bfloat16().double(), d ** -0.5, torch.arange(n - rows, n))
            O, A = p @ x[:, Hq + Hkv + head // G], p @ x[:, Hq + Hkv + head // G].abs()
            # a rotated value next to the middle between two bf16 numbers may be rounded either way: one step of one factor in a score
            slack = FP32_SLACK + 2 * BF16_HALF * 1e-1
            assert ((o[:, head].cpu().double() - O).abs() <= BF16_HALF * O.abs() + (BF16_HALF + slack) * A).all()
            assert ((lse[head].cpu().double() - L).abs() <= slack).all()

    x = torch.randn(203, Hq + 2 * Hkv, d, device="cuda").bfloat16()
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    qr = b.append_paged(h, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], cache, table, lens, cu_seqlens=cu, q=x[:, :Hq], rope=rope)
    kr = torch.cat([torch.cat([k[int(table[i, j])].transpose(0, 1) for j in range(-(-n // page))])[:n] for i, n in enumerate(prompts)])
    o, lse = b.forward_varlen(h, qr, kr.contiguous(), x[:, Hq + Hkv:].contiguous(), cu, cu, max(prompts), causal=True)
    ok(h)
    for i in range(B):
        here = slice(int(cu[i]), int(cu[i + 1]))
        history[i] = x[here].cpu().double()
        check(i, prompts[i], o[here], lse[:, here])
    for step in range(steps):
        x = torch.randn(B, Hq + 2 * Hkv, d, device="cuda").bfloat16()
        lens += 1
        qr = b.append_paged(h, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], cache, table, lens, q=x[:, :Hq], rope=rope)
        o, lse = b.forward_paged(h, qr, cache, table, lens)
        ok(h)
        for i in range(B):
            history[i] = torch.cat([history[i], x[i:i + 1].cpu().double()])
            check(i, 1, o[i:i + 1], lse[:, i:i + 1])
    b.fa_destroy(h)


@pytest.mark.parametrize("e4m3,diff", [(False, False), (True, False), (False, True)], ids=["bf16", "e4m3", "diff"])
def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(e4m3, diff):
    """The hook leaves out each CTA's first V tile: the launch returns, the host reads FA_ERR_DEVICE_TIMEOUT, and the next launch
    through the same handle (shared row blocks and their counters among its work) is right."""
    from paper_2609_21264_b200 import binding as b
    lens = [700, 3000, 40, 0, 129]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, 128, 128, e4m3, False, 80)
    q = torch.randn(len(lens), 8, 128, device="cuda").bfloat16()
    cache, lam = b.PagedCache(k, v, ks, vs), torch.rand(8, device="cuda")
    h, fresh = b.fa_create(flags=b.FA_FLAG_DEBUG_DROP_V_LOAD, wait_limit_ms=20), b.fa_create()

    def call(handle):
        if diff:
            return b.forward_paged_diff(handle, q, cache, table, lens_t, lam)
        return b.forward_paged(handle, q, cache, table, lens_t)[0]

    try:
        want = call(fresh)
        ok(fresh)
        call(h)
        torch.cuda.synchronize()
        st, site = b.fa_last_status(h)
        assert st == b.FA_ERR_DEVICE_TIMEOUT and site != 0
        assert b.fa_debug_set_drop_v_load(h, False) == b.FA_OK
        for _ in range(3):
            o = call(h)
            ok(h)
            assert torch.equal(o, want)
    finally:
        b.fa_destroy(h)
        b.fa_destroy(fresh)


def test_small_scratch_and_two_handles_on_two_streams():
    """A handle whose scratch holds a few partial results uses fewer CTAs; two handles may run at the same time."""
    from paper_2609_21264_b200 import binding as b
    lens = [9000, 200, 4000]
    k, v, table, lens_t, _, _ = pool(lens, 64, 2, 128, 128, False, True, 81)
    q = torch.randn(3, 16, 128, device="cuda").bfloat16()
    cache = b.PagedCache(k, v)
    ref = paged_reference(q, k, v, None, None, table, lens, 1, 128 ** -0.5)
    handles = [b.fa_create(scratch_bytes=6 * 16 * 130 * 4), b.fa_create()]
    streams = [torch.cuda.Stream() for _ in handles]
    try:
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        outs = []
        for _ in range(4):
            for h, s in zip(handles, streams):
                with torch.cuda.stream(s):
                    outs.append(b.forward_paged(h, q, cache, table, lens_t))
        for h in handles:
            ok(h)
        for o, lse in outs:
            assert_attention(o, lse, *ref)
        assert all(torch.equal(outs[0][0], outs[i][0]) for i in (2, 4, 6)) and all(torch.equal(outs[1][0], outs[i][0]) for i in (3, 5, 7))
        tiny = b.fa_create(scratch_bytes=1024)
        with pytest.raises(b.FaError) as e:
            b.forward_paged(tiny, q, cache, table, lens_t)
        assert e.value.status == b.FA_ERR_UNSUPPORTED
        b.fa_destroy(tiny)
    finally:
        torch.cuda.synchronize()
        for h in handles:
            b.fa_destroy(h)


def test_cache_of_more_than_2_31_elements(handle):
    """Pages whose elements lie behind 2^31, of a pool of either order."""
    from paper_2609_21264_b200 import binding
    pages, Hkv, page, d = 17000, 8, 128, 128
    for heads_first in (False, True):
        shape = (pages, Hkv, page, d) if heads_first else (pages, page, Hkv, d)
        k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        if not heads_first:
            k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
        table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
        for t in (k, v):
            t[table[0].long()] = torch.randn(3, Hkv, page, d, device="cuda").bfloat16()
        q = torch.randn(1, 16, d, device="cuda").bfloat16()
        lens = torch.tensor([300], dtype=torch.int32, device="cuda")
        o, lse = binding.forward_paged(handle, q, binding.PagedCache(k, v), table, lens)
        ok(handle)
        small_k, small_v = k[table[0].long()], v[table[0].long()]
        assert_attention(o, lse, *paged_reference(q, small_k, small_v, None, None, torch.tensor([[0, 1, 2]]), [300], 1, d ** -0.5))
        del k, v
        torch.cuda.empty_cache()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[200, 90], [6000, 90]], ids=["whole", "split"])
def test_a_key_that_is_no_number_shows_in_its_own_rows_alone(handle, e4m3, lens):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, 128, 128, e4m3, False, 60)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    at = lens[0] - 70
    k.view(torch.uint8 if e4m3 else torch.bfloat16)[int(table[0, at // 16]), 1, at % 16, 5] = 0x7F if e4m3 else float("nan")
    o, lse = b.forward_paged(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert o[0, 4:].isnan().all() and lse[4:, 0].isnan().all()
    assert o[0, :4].isfinite().all() and o[1].isfinite().all() and lse[:4].isfinite().all() and lse[:, 1].isfinite().all()
    # a query that is none, against keys that all are numbers
    q[1, 2, 7] = float("nan")
    o, lse = b.forward_paged(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert o[1, 2].isnan().all() and lse[2, 1].isnan() and o[1, [0, 1, 3]].isfinite().all()


def test_an_empty_batch_is_nothing(handle):
    from paper_2609_21264_b200 import binding as b
    c = b.PagedCache(*pool([20], 16, 2, 64, 64, False, False, 5)[:2])
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 0, None, 1, None, 1, 0)
    assert b.fa_forward_paged(handle, c.c, seqs, None, None, None, 4, 1, 0.0, (256, 64), (256, 64)) == b.FA_OK
