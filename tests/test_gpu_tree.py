"""fa_forward_paged_tree against the definition in 64 bits: trees, chains, masks that leave rows without a key, ragged batches.

Unused slots of the pages hold NaN and infinities, unused block table entries numbers that are no pages."""
import ctypes

import pytest
import torch

from draft_util import pack, random_parents, seen_by, tree_reference
from paged_util import assert_attention, ok, pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["serial", "default"])
def handle(request):
    from paper_2609_21264_b200 import binding
    h = binding.fa_create(flags=binding.FA_FLAG_SERIAL_KERNEL if request.param == "serial" else 0)
    yield h
    binding.fa_destroy(h)


def run(handle, lens, counts, Hq, Hkv, dqk, dv, page, e4m3=False, heads_first=False, seed=1, q_mult=1.0, shift=0.0, scale=0.0, masks="tree",
        most=0, pad=0, cu=True):
    """masks: "tree", "chain" (no mask), "random" (any bits, those of n and more set too), "none" (no bit at all)."""
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, dqk, dv, e4m3, heads_first, seed, shift=shift)
    g = torch.Generator().manual_seed(seed + 1)
    T = sum(counts) + pad
    most = most or max(1, max(counts))
    words = (most + 31) // 32
    q = (torch.randn(T, Hq, dqk, generator=g) * q_mult).to(torch.bfloat16).cuda()
    offsets = [0]
    for n in counts:
        offsets.append(offsets[-1] + n)
    seens, mask = [], torch.full((T, words), -1, dtype=torch.int32)
    for b, n in enumerate(counts):
        if masks == "tree":
            seen = seen_by(random_parents(n, g))[0]
        elif masks == "chain":
            seen = torch.ones(n, n).tril() > 0
        elif masks == "none":
            seen = torch.zeros(n, n) > 0
        else:
            seen = torch.rand(n, n, generator=g) < 0.4
        seens.append(seen)
        wide = torch.ones(n, 32 * words) > 0 if masks == "random" else torch.zeros(n, 32 * words) > 0
        wide[:, :n] = seen
        mask[offsets[b]:offsets[b + 1]] = pack(wide, words)
    out = torch.full((T, Hq, dv), 7.0, dtype=torch.bfloat16, device="cuda")
    o, lse = binding.forward_paged_tree(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, None if masks == "chain" else mask.cuda(),
                                        cu_seqlens=torch.tensor(offsets, dtype=torch.int32, device="cuda") if cu else None, max_tokens=most,
                                        scale=scale, out=out)
    assert o is out
    ok(handle)
    O, L, A = tree_reference(q[:offsets[-1]], k, v, ks, vs, table, lens, offsets, seens, scale or dqk ** -0.5)
    assert (o[offsets[-1]:] == 7).all()
    return assert_attention(o[:offsets[-1]], lse[:, :offsets[-1]], O, L, A)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (3, 3), (14, 2), (16, 1)], ids=["g4", "g1", "g7", "g16"])
def test_lengths_around_tiles_and_pages(handle, dqk, dv, e4m3, Hq, Hkv):
    lens = [5, 16, 17, 31, 127, 128, 129, 255, 256, 257, 700]
    run(handle, lens, [5, 3, 17, 1, 9, 12, 8, 0, 20, 2, 19], Hq, Hkv, dqk, dv, 16, e4m3, heads_first=e4m3, seed=dqk + Hq, pad=2)


@pytest.mark.parametrize("page", [16, 32, 48, 80, 128, 176, 256, 1024])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_page_sizes(handle, page, e4m3):
    run(handle, [7, 300, 47, 1100], [7, 26, 3, 16], 8, 2, 128, 128, page, e4m3, heads_first=not e4m3, seed=page)


@pytest.mark.parametrize("n", [1, 2, 16, 31, 32, 33, 63, 64, 65, 100, 128, 129, 200, 256])
@pytest.mark.parametrize("dqk,dv,Hq,Hkv", [(128, 128, 8, 2), (64, 64, 6, 1), (192, 128, 2, 2)], ids=["d128", "d64", "d192"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_numbers_of_drafts(handle, n, dqk, dv, Hq, Hkv, e4m3):
    """Trees whose drafts end at, before and behind a tile's border, begin in the tile before, or are all that there is."""
    run(handle, [n, n + 1, 384, 300 + n // 2, 385], [n] * 5, Hq, Hkv, dqk, dv, 32, e4m3, seed=n, cu=n % 2 == 0)


@pytest.mark.parametrize("masks", ["chain", "random", "none"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_other_masks(handle, masks, e4m3, dqk, dv):
    """A chain, any bits (rows that see nothing among them: sequences that have nothing but drafts), no bits; max_tokens above the
    counts, and words of the mask that no sequence needs."""
    run(handle, [40, 1, 9, 300, 512, 0, 130], [40, 1, 9, 40, 33, 0, 2], 8, 2, dqk, dv, 16, e4m3, seed=3, masks=masks, most=100, pad=1)


def test_sequences_shorter_than_their_drafts(handle):
    """The padding of a captured step: length 0, or fewer keys than drafts; what stands in front of position 0 is seen by nobody."""
    run(handle, [0, 3, 200, 0], [4, 4, 4, 4], 8, 2, 128, 128, 16, masks="random", cu=False)
    run(handle, [0, 3, 200, 0], [4, 4, 4, 4], 8, 2, 128, 128, 16, True, masks="chain", cu=False)
    run(handle, [60, 3, 200, 129], [64, 64, 64, 64], 8, 2, 128, 128, 16, masks="tree", cu=False)
    # a batch of nothing but padding: its rows are written all the same
    for dqk, dv, e4m3 in ((128, 128, False), (64, 64, True), (192, 128, False)):
        run(handle, [0], [4], 8, 2, dqk, dv, 16, e4m3, cu=False)
        run(handle, [0, 0, 0], [40, 0, 3], 8, 2, dqk, dv, 16, e4m3, pad=2)


@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (40, 1), (128, 1), (130, 1), (300, 2), (10, 2)])
def test_groups_of_any_size(handle, Hq, Hkv):
    """Groups that do not divide a tile's rows, and groups larger than a tile."""
    run(handle, [130, 50, 400], [5, 13, 30], Hq, Hkv, 128, 128, 16, seed=Hq)
    run(handle, [130, 50], [5, 13], Hq, Hkv, 64, 64, 16, True, seed=Hq)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_long_and_many(handle, e4m3):
    run(handle, [20000], [20], 8, 1, 128, 128, 64, e4m3, seed=5)
    run(handle, [9000], [70], 8, 2, 128, 128, 64, e4m3, seed=5)
    run(handle, [(i * 53) % 260 for i in range(200)], [min((i * 53) % 260, i % 9) for i in range(200)], 2, 2, 64, 64, 16, e4m3, seed=6)
    run(handle, [3000] + [3] * 40 + [9000], [30] + [3] * 40 + [12], 8, 2, 128, 128, 16, e4m3, seed=7)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_large_scores_and_rising_maxima(handle, e4m3):
    """Scores in the hundreds, keys whose scores rise along the sequence (the reference maximum moves again and again) and fall."""
    from paper_2609_21264_b200 import binding
    run(handle, [1000, 77], [30, 26], 8, 2, 128, 128, 16, e4m3, seed=8, q_mult=8.0)
    k, v, table, lens_t, ks, vs = pool([2000], 32, 2, 128, 128, e4m3, False, 9, poison=False)
    flat = torch.arange(2000, device="cuda")
    ramp = (flat.float() / 2000 * 4 - 2)
    kk = torch.zeros(k.shape, device="cuda")
    kk[table[0, flat // 32].long(), :, flat % 32] = ramp[:, None, None].expand(2000, 2, 128)
    k.copy_((kk * 20).to(k.dtype) if e4m3 else kk.to(k.dtype))
    q = torch.ones(40, 8, 128, device="cuda").bfloat16()
    q[:, ::2] *= -1
    o, lse = binding.forward_paged_tree(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, [2000], [0, 40], [torch.ones(40, 40).tril() > 0], 128 ** -0.5))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_one_key_far_above_many_small_ones(handle, e4m3):
    """A key of weight about one half and thousands whose weights, each 2^-14 of it, make up the other half."""
    from paper_2609_21264_b200 import binding
    n = 16000
    k, v, table, lens_t, ks, vs = pool([n], 64, 1, 128, 128, e4m3, False, 10, poison=False, shift=0.5)
    kf = torch.zeros(k.shape, device="cuda")
    kf[int(table[0, 3]), 0, 5, :] = 20.0 if e4m3 else 1.0
    k.copy_(kf.to(k.dtype))
    q = torch.full((12, 4, 128), 9.7 * 128 ** 0.5 / 128, device="cuda").bfloat16()
    o, lse = binding.forward_paged_tree(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, [n], [0, 12], [torch.ones(12, 12).tril() > 0], 128 ** -0.5))


@pytest.mark.parametrize("shift", [-118, -90, 0, 90, 118])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_queries_of_any_size_over_an_8_bit_cache(handle, shift, dqk, dv):
    """Queries of 2^shift, their entries spread over 2^20, against keys whose scale is 2^-shift: ordinary scores from numbers near
    either end of the range."""
    from paper_2609_21264_b200 import binding as b
    lens, counts = [150, 40], [11, 11]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, True, False, 30)
    g = torch.Generator().manual_seed(31)
    q = torch.randn(22, 8, dqk, generator=g) * 2.0 ** shift
    if shift == 0:
        q = q * 2.0 ** torch.randint(-20, 1, q.shape, generator=g)
        q[:, 3] = 0
    q = q.to(torch.bfloat16).cuda()
    ks = ks * 2.0 ** -shift
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, lens, [0, 11, 22], [torch.ones(n, n).tril() > 0 for n in counts], dqk ** -0.5))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_keys_that_are_no_numbers(handle, e4m3):
    """A draft's key of NaN or infinities that the mask hides changes nothing; one that a row sees makes that row NaN, no other."""
    from paper_2609_21264_b200 import binding as b
    n = 20
    k, v, table, lens_t, ks, vs = pool([150], 16, 1, 128, 128, e4m3, False, 12)
    seen, _ = seen_by(random_parents(n, torch.Generator().manual_seed(4)))
    q = torch.randn(n, 4, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    mask = pack(seen, 1).cuda()
    cache = b.PagedCache(k, v, ks, vs)
    o0, lse0 = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    at = 130 + 7                                         # draft 7
    page, slot = int(table[0, at // 16]), at % 16
    if e4m3:
        k.view(torch.uint8)[page, :, slot] = 0x7F
    else:
        k[page, :, slot] = float("nan")
        k[page, :, slot, ::3] = float("inf")
    o1, lse1 = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    hit = seen[:, 7].cuda()
    assert hit.any() and not hit.all()
    assert torch.equal(o1[~hit], o0[~hit]) and torch.equal(lse1[:, ~hit], lse0[:, ~hit])
    assert torch.isnan(o1[hit]).all() and torch.isnan(lse1[:, hit]).all()


def test_strides_of_queries_and_results(handle):
    """Slices of one projection's output, and a result in a wider buffer."""
    from paper_2609_21264_b200 import binding as b
    for dqk, dv, e4m3 in ((128, 128, False), (64, 64, True), (192, 128, False)):
        k, v, table, lens_t, ks, vs = pool([300, 40], 16, 2, dqk, dv, e4m3, False, 13)
        wide = torch.randn(2 * 9, 14, dqk, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
        q = wide[:, 2:10]
        out = torch.full((18, 11, dv + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        cache = b.PagedCache(k, v, ks, vs)
        o, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None, out=out[:, 3:, :dv])
        o2, lse2 = b.forward_paged_tree(handle, q.contiguous(), cache, table, lens_t, None)
        ok(handle)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert (out[:, :3] == 7).all() and (out[:, :, dv:] == 7).all()
        assert b.forward_paged_tree(handle, q, cache, table, lens_t, None, want_lse=False)[1] is None


def test_agrees_with_the_paged_call(handle):
    """Chains of up to 16 tokens are what fa_forward_paged computes."""
    from paper_2609_21264_b200 import binding as b
    for e4m3 in (False, True):
        k, v, table, lens_t, ks, vs = pool([300, 5, 129, 1000], 32, 2, 128, 128, e4m3, False, 14)
        q = torch.randn(4 * 5, 8, 128, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).cuda()
        cache = b.PagedCache(k, v, ks, vs)
        o, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
        o2, lse2 = b.forward_paged(handle, q, cache, table, lens_t)
        ok(handle)
        # two results that are each within one rounding of a probability and of the output: 4 * 2^-8 of values below 4
        assert (o.double() - o2.double()).abs().max() <= 4 * 4 * 2.0 ** -8 and (lse - lse2).abs().max() <= 6e-4


def test_equal_calls_give_equal_bits(handle):
    from paper_2609_21264_b200 import binding as b
    for e4m3, lens, n in ((False, [9000, 300, 4000], 40), (True, [9000, 300, 4000], 12), (False, [30000], 7)):
        k, v, table, lens_t, ks, vs = pool(lens, 64, 2, 128, 128, e4m3, False, 15)
        q = torch.randn(len(lens) * n, 8, 128, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
        cache = b.PagedCache(k, v, ks, vs)
        one = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
        for _ in range(5):
            two = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
            assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
        ok(handle)


def test_captured_call_follows_new_lengths_tables_and_masks(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool([700, 400], 16, 2, 128, 128, False, False, 16, poison=False)
    g = torch.Generator().manual_seed(9)
    q = torch.randn(40, 8, 128, generator=g).to(torch.bfloat16).cuda()
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (40, 1), generator=g, dtype=torch.int64).to(torch.int32).cuda()
    cu = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    cache, out = b.PagedCache(k, v), torch.zeros(40, 8, 128, dtype=torch.bfloat16, device="cuda")
    call = lambda: b.forward_paged_tree(handle, q, cache, table, lens_t, mask, cu_seqlens=cu, max_tokens=30, out=out)  # noqa: E731
    call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _, lse = call()
    lens_t.copy_(torch.tensor([123, 333], dtype=torch.int32))
    cu.copy_(torch.tensor([0, 11, 37], dtype=torch.int32))
    table.copy_(table.flip(0))
    mask.copy_(mask.flip(0))
    table.clamp_(0, k.shape[0] - 1)
    out.fill_(7)
    graph.replay()
    ok(handle)
    got, got_lse = out.clone(), lse[:, :37].clone()
    assert (got[37:] == 7).all()
    call()
    ok(handle)
    assert torch.equal(got, out)
    seens = [torch.tensor([[(int(w) >> j) & 1 for j in range(n)] for w in mask[a:a + n, 0].tolist()]) > 0 for a, n in ((0, 11), (11, 26))]
    assert_attention(got[:37], got_lse, *tree_reference(q[:37], k, v, None, None, table, [123, 333], [0, 11, 37], seens, 128 ** -0.5))


def test_another_stream(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool([500], 16, 2, 128, 128, False, False, 17)
    q = torch.randn(33, 8, 128, generator=torch.Generator().manual_seed(10)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v)
    want = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            x = torch.randn(2048, 2048, device="cuda")
            for _ in range(5):
                x = x @ x * 1e-3
            late = q * (1 + 0 * x[0, 0]).to(q.dtype).nan_to_num(1.0).clamp(1, 1)       # (depends on the work before it)
            got = b.forward_paged_tree(handle, late, cache, table, lens_t, None)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_contents_the_device_refuses(handle):
    """Pages outside the pool, lengths past the table, rows that are not the call's: reported, other sequences hold."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([40, 300], 16, 2, 64, 64, False, False, 18)
    q = torch.randn(12, 4, 64, generator=torch.Generator().manual_seed(11)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v)
    good, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    ok(handle)
    O, L, A = tree_reference(q, k, v, None, None, table, [40, 300], [0, 6, 12], [torch.ones(6, 6).tril() > 0] * 2, 0.125)
    # (other lengths deal the work out otherwise: the same values, within their rounding)
    holds = lambda o: assert_attention(o[6:], None, O[6:], L[:, 6:], A[6:]) <= 1  # noqa: E731
    assert assert_attention(good, lse, O, L, A) <= 1
    for page in (-1, k.shape[0], 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[0, 1] = page
        o, _ = b.forward_paged_tree(handle, q, cache, bad, lens_t, None)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0902) and holds(o)
    for n in (-1, -2 ** 31, 16 * table.shape[1] + 1, 2 ** 31 - 1):
        bad = lens_t.clone()
        bad[0] = n
        o, _ = b.forward_paged_tree(handle, q, cache, table.clamp(0, k.shape[0] - 1), bad, None)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0901) and holds(o)
    # (the second sequence keeps its rows 6 to 11 in each)
    for cu, most in (([-3, 6, 12], 10), ([7, 6, 12], 10), ([0, 6, 13], 10), ([0, 6, 2 ** 31 - 1], 10), ([-2 ** 31, 6, 12], 10), ([0, 6, 12], 5)):
        out = torch.full_like(good, 7)
        b.forward_paged_tree(handle, q, cache, table, lens_t, None, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), max_tokens=most, out=out)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0904)
        whole = cu[2] == 12 and most == 10
        assert holds(out) if whole else (out[6:] == 7).all()
    assert b.fa_last_status(handle) == (b.FA_OK, 0)


def test_empty_batches(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([40], 16, 2, 64, 64, False, False, 19)
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    cache = b.PagedCache(k, v)
    before = b.fa_launch_count(handle)
    o, lse = b.forward_paged_tree(handle, q[:0], cache, table[:0], lens_t[:0], None)
    assert o.shape == (0, 4, 64) and lse.shape == (4, 0)
    b.forward_paged_tree(handle, q[:0], cache, table, lens_t, None, cu_seqlens=torch.zeros(2, dtype=torch.int32, device="cuda"), max_tokens=3)
    assert b.fa_launch_count(handle) == before
    # rows, but none of them a sequence's
    out = torch.full((6, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    b.forward_paged_tree(handle, q, cache, table, lens_t, None, cu_seqlens=torch.zeros(2, dtype=torch.int32, device="cuda"), max_tokens=3, out=out)
    ok(handle)
    assert (out == 7).all()


def test_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([40], 16, 2, 64, 64, False, False, 20)
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    o = torch.empty_like(q)
    cache = b.PagedCache(k, v)
    mask = torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 1, table.data_ptr(), table.shape[1], lens_t.data_ptr(), table.shape[1], 0)
    size = ctypes.sizeof(b.fa_tree)

    def call(h=handle, tree=(size, 6, None, mask.data_ptr(), 1), total=6, Q=q.data_ptr(), O=o.data_ptr(), lse=None, Hq=4, scale=0.0, qs=(256, 64), os=(256, 64)):
        return b.fa_forward_paged_tree(h, cache.c, seqs, None if tree is None else b.fa_tree(*tree), total, Q, O, lse, Hq, scale, qs, os)

    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call() == b.FA_OK
    assert call(h=None) == bad and call(tree=None) == bad and call(total=-1) == bad and call(Q=None) == bad and call(O=None) == bad
    assert call(Q=q.data_ptr() + 2) == bad and call(lse=2) == bad and call(Hq=0) == bad and call(Hq=3) == bad and call(Hq=65538) == no
    assert call(scale=float("nan")) == bad and call(scale=-1.0) == bad and call(qs=(256, 60)) == bad and call(os=(0, 64)) == bad and call(qs=None) == bad
    for tree, want in (((8, 6, None, None, 1), bad), ((size, 0, None, None, 1), bad), ((size, -1, None, None, 1), bad), ((size, 257, None, None, 9), no),
                       ((size, 33, None, mask.data_ptr(), 1), bad), ((size, 6, 2, None, 1), bad), ((size, 6, None, 2, 1), bad), ((size, 5, None, None, 1), bad)):
        assert call(tree=tree) == want, tree
    torch.cuda.synchronize()
    for kw in ({"mask": mask.long()}, {"mask": mask[:5]}, {"max_tokens": 33}, {"cu_seqlens": torch.zeros(3, dtype=torch.int32, device="cuda"), "max_tokens": 6},
               {"cu_seqlens": torch.zeros(2, dtype=torch.int32, device="cuda")}, {"max_tokens": -1}, {"out": o[:5]}, {"mask": mask.cpu()}):
        kw = {"mask": mask, **kw}
        with pytest.raises(ValueError):
            b.forward_paged_tree(handle, q, cache, table, lens_t, kw.pop("mask"), **kw)
    with pytest.raises(b.FaError):
        b.forward_paged_tree(handle, q, cache, table, lens_t, mask, max_tokens=5)
    ok(handle)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_wait_that_runs_out(dqk, dv, e4m3):
    """The loading warps leave out their first V tile: the kernel returns with a status, and the next call of the handle is right."""
    from paper_2609_21264_b200 import binding as b
    lens, n = [700, 150], 20
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, e4m3, False, 21)
    q = torch.randn(2 * n, 8, dqk, generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v, ks, vs)
    h = b.fa_create(flags=b.FA_FLAG_DEBUG_DROP_V_LOAD, wait_limit_ms=20)
    try:
        b.forward_paged_tree(h, q, cache, table, lens_t, None)
        torch.cuda.synchronize()
        st, site = b.fa_last_status(h)
        assert st == b.FA_ERR_DEVICE_TIMEOUT and site != 0 and b.fa_last_kernel_name(h).startswith("fa_tree")
        b.fa_debug_set_drop_v_load(h, False)
        o, lse = b.forward_paged_tree(h, q, cache, table, lens_t, None)
        ok(h)
        assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, lens, [0, n, 2 * n], [torch.ones(n, n).tril() > 0] * 2, dqk ** -0.5))
    finally:
        b.fa_destroy(h)


def test_little_scratch(handle):
    """A handle with room for two partial results on one SM works on that one; with less, on none."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([700, 150], 16, 2, 128, 128, False, False, 22)
    q = torch.randn(2 * 40, 8, 128, generator=torch.Generator().manual_seed(13)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v)
    ref = tree_reference(q, k, v, None, None, table, [700, 150], [0, 40, 80], [torch.ones(40, 40).tril() > 0] * 2, 128 ** -0.5)
    for size, works in ((300 << 10, True), (1 << 20, True), (200 << 10, False)):
        h = b.fa_create(scratch_bytes=size)
        try:
            if works:
                o, lse = b.forward_paged_tree(h, q, cache, table, lens_t, None)
                ok(h)
                assert_attention(o, lse, *ref)
            else:
                with pytest.raises(b.FaError) as e:
                    b.forward_paged_tree(h, q, cache, table, lens_t, None)
                assert e.value.status == b.FA_ERR_UNSUPPORTED
        finally:
            b.fa_destroy(h)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_queries_that_are_no_numbers(handle, e4m3, dqk, dv):
    """A query of NaN makes its own row NaN, no other."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool([300, 150], 16, 2, dqk, dv, e4m3, False, 23)
    q = torch.randn(2 * 20, 8, dqk, generator=torch.Generator().manual_seed(14)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v, ks, vs)
    o0, lse0 = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    ok(handle)
    q[7, 3, 5] = float("nan")
    q[25, 0] = float("nan")
    o1, lse1 = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    ok(handle)
    hit = torch.zeros(40, 8, dtype=torch.bool, device="cuda")
    hit[7, 3] = hit[25, 0] = True
    assert torch.isnan(o1[hit]).all() and torch.isnan(lse1.T[hit]).all()
    assert torch.equal(o1[~hit], o0[~hit]) and torch.equal(lse1.T[~hit], lse0.T[~hit])


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [1e-30, 0.01, 1.0])
def test_scales(handle, e4m3, scale):
    """Scores that hardly differ (the mean of the values), and large ones; an 8-bit cache without scales of its own."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([300, 140, 20], 16, 2, 128, 128, e4m3, True, 24)
    if e4m3:
        k, v = ((x.float() / 16).nan_to_num(0.0).clamp(-3, 3).to(torch.float8_e4m3fn) for x in (k, v))
    q = torch.randn(3 * 15, 8, 128, generator=torch.Generator().manual_seed(15)).to(torch.bfloat16).cuda()
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v), table, lens_t, None, scale=scale)
    ok(handle)
    O, L, A = tree_reference(q, k, v, None, None, table, [300, 140, 20], [0, 15, 30, 45], [torch.ones(15, 15).tril() > 0] * 3, scale)
    assert_attention(o, lse, O, L, A)


def test_masked_values_near_the_largest_number(handle):
    """A draft whose values are 2^120, seen by a few: it weighs exactly nothing in the others."""
    from paper_2609_21264_b200 import binding as b
    n = 20
    k, v, table, lens_t, _, _ = pool([150], 16, 1, 128, 128, False, False, 25)
    seen, _ = seen_by(random_parents(n, torch.Generator().manual_seed(4)))
    q = torch.randn(n, 4, 128, generator=torch.Generator().manual_seed(16)).to(torch.bfloat16).cuda()
    mask, cache = pack(seen, 1).cuda(), b.PagedCache(k, v)
    o0, _ = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    at = 130 + 7
    v[int(table[0, at // 16]), :, at % 16] = 2.0 ** 120
    o1, _ = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    hit = seen[:, 7].cuda()
    assert torch.equal(o1[~hit], o0[~hit]) and not torch.equal(o1[hit], o0[hit])


def test_many_sequences(handle):
    """More sequences than a warp has lanes many times over, most of them short."""
    lens = [(i * 29) % 150 + (3000 if i % 97 == 5 else 0) for i in range(1500)]
    counts = [min(n, i % 4) for i, n in enumerate(lens)]
    run(handle, lens, counts, 2, 1, 64, 64, 16, seed=26, pad=1)


def test_launches_without_overlap_and_two_handles_at_once():
    from paper_2609_21264_b200 import binding as b
    cases = []
    for seed, (lens, n, e4m3) in enumerate((([5000, 300], 40, False), ([4000, 900, 20], 13, True))):
        k, v, table, lens_t, ks, vs = pool(lens, 32, 2, 128, 128, e4m3, False, 27 + seed)
        q = torch.randn(len(lens) * n, 8, 128, generator=torch.Generator().manual_seed(17)).to(torch.bfloat16).cuda()
        cases.append((q, b.PagedCache(k, v, ks, vs), table, lens_t))
    handles = [b.fa_create(), b.fa_create(flags=b.FA_FLAG_NO_DEPENDENT_LAUNCH)]
    try:
        want = [b.forward_paged_tree(handles[0], q, c, t, l, None) for q, c, t, l in cases]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in handles]
        got = [[], []]
        for _ in range(10):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    q, c, t, l = cases[i]
                    got[i].append(b.forward_paged_tree(handles[i], q, c, t, l, None))
        for h in handles:
            ok(h)
        for i in range(2):
            for o, lse in got[i]:
                assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])
    finally:
        for h in handles:
            b.fa_destroy(h)


# (drafts, query heads, K/V heads) up to 32 rows, the last of each group just above
FEW = [(1, 1, 1), (16, 2, 2), (32, 1, 1), (33, 1, 1), (8, 4, 2), (16, 4, 2), (17, 4, 2), (5, 9, 3), (8, 8, 2), (4, 14, 2), (5, 14, 2), (4, 8, 1), (2, 16, 1),
       (1, 31, 1), (1, 32, 1), (1, 33, 1), (3, 10, 1), (4, 10, 1)]


@pytest.mark.parametrize("most,Hq,Hkv", FEW)
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_few_rows(handle, most, Hq, Hkv, dqk, dv, e4m3):
    """Up to 32 rows and the first number above: ragged trees around the borders of a tile, sequences without drafts or without keys."""
    n = [min(most, x) for x in (3, 0, 1, 32, 2, 5, 0, 17, 33, 4)]
    lens = [700, 300, 1, 129, 128, 5, 0, 257, 33, 127]
    assert all(a <= x for a, x in zip(n, lens))
    run(handle, lens, n, Hq, Hkv, dqk, dv, 16, e4m3, heads_first=e4m3, seed=most + Hq, most=most, pad=2)


@pytest.mark.parametrize("masks", ["tree", "chain", "random", "none"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,most", [(2, 2, 32), (2, 2, 16), (8, 2, 8), (24, 1, 1)])
def test_masks_of_few_rows(handle, masks, e4m3, Hq, Hkv, most):
    """Rows that see nothing, in sequences that have nothing but drafts, or fewer keys than drafts; bits of n and more are not looked at."""
    n = [most, 1, min(most, 9), most, 0, 1, most, most]
    run(handle, [most, 1, 3, 300, 40, 0, 129, 128 + most // 2], n, Hq, Hkv, 128, 128, 32, e4m3, seed=9, masks=masks, most=most, pad=1)
    run(handle, [300, 0, 17], [most] * 3, Hq, Hkv, 64, 64, 16, e4m3, seed=10, masks=masks, cu=False)
    run(handle, [0, 0], [most] * 2, Hq, Hkv, 192, 128, 16, e4m3, seed=11, masks=masks, cu=False)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_few_rows_long_and_many(handle, e4m3):
    run(handle, [20000], [4], 8, 1, 128, 128, 64, e4m3, seed=5)
    run(handle, [9000, 20, 9100], [30, 2, 32], 2, 2, 64, 64, 48, e4m3, seed=5, most=32)
    run(handle, [(i * 53) % 260 for i in range(200)], [min((i * 53) % 260, i % 9) for i in range(200)], 4, 2, 192, 128, 16, e4m3, seed=6)
    run(handle, [3000] + [3] * 40 + [9000], [8] + [3] * 40 + [7], 8, 2, 128, 128, 16, e4m3, seed=7, q_mult=3.0)


def test_a_chain_of_few_drafts_is_the_paged_call():
    """Equally many drafts in a chain: the kernel of fa_forward_paged, and its bits where both cut the batch alike."""
    from paper_2609_21264_b200 import binding as b
    h = b.fa_create()
    try:
        for e4m3, dqk, dv, Hq, Hkv, n in ((False, 128, 128, 8, 2, 4), (True, 128, 128, 8, 2, 8), (False, 64, 64, 4, 4, 16), (True, 192, 128, 6, 1, 5)):
            k, v, table, lens_t, ks, vs = pool([700, 40, 768], 16, Hkv, dqk, dv, e4m3, False, 31)
            q = torch.randn(3 * n, Hq, dqk, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
            cache = b.PagedCache(k, v, ks, vs)
            want = b.forward_paged(h, q, cache, table, lens_t)
            got = b.forward_paged_tree(h, q, cache, table, lens_t, None)
            ok(h)
            assert b.fa_last_kernel_name(h) == ("fa_tree_few_e4m3" if e4m3 else "fa_tree_few")
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    finally:
        b.fa_destroy(h)


def test_few_rows_captured_with_other_contents(handle):
    """A captured call of few rows follows what lengths, offsets, masks and the table hold when it is replayed."""
    from paper_2609_21264_b200 import binding as b
    g = torch.Generator().manual_seed(41)
    first, then = ([500, 130, 0], [4, 7, 0]), ([260, 505, 9], [8, 1, 2])
    k, v, table, lens_t, _, _ = pool([520, 520, 520], 16, 2, 128, 128, False, False, 17)
    q = torch.randn(13, 8, 128, generator=g).to(torch.bfloat16).cuda()
    cu, mask, lens = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(13, 1, dtype=torch.int32, device="cuda"), torch.zeros_like(lens_t)
    out = torch.zeros(13, 8, 128, dtype=torch.bfloat16, device="cuda")
    cache = b.PagedCache(k, v)

    def fill(lengths, counts):
        seens, offsets = [torch.rand(n, n, generator=g) < 0.5 for n in counts], [0]
        for n in counts:
            offsets.append(offsets[-1] + n)
        rows = torch.full((13, 1), -1, dtype=torch.int32)
        for s, a, n in zip(seens, offsets, counts):
            rows[a:a + n] = pack(s, 1)
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        cu.copy_(torch.tensor(offsets, dtype=torch.int32))
        mask.copy_(rows)
        out.fill_(7.0)
        return tree_reference(q[:offsets[-1]], k, v, None, None, table, lengths, offsets, seens, 128 ** -0.5), offsets[-1]

    call = lambda: b.forward_paged_tree(handle, q, cache, table, lens, mask, cu_seqlens=cu, max_tokens=8, out=out)  # noqa: E731
    ref, n = fill(*first)
    call()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        _, lse = call()
    for what in (first, then, first):
        ref, n = fill(*what)
        graph.replay()
        torch.cuda.synchronize()
        ok(handle)
        assert_attention(out[:n], lse[:, :n], *ref)
        assert (out[n:] == 7).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,n", [(1, 20), (2, 8)], ids=["32rows", "16rows"])
def test_numbers_that_are_none_in_few_rows(handle, e4m3, Hq, n):
    """A draft's key of NaN or infinities and a query of NaN concern the rows that see the one and are the other; a masked value of 2^120 (bf16)
    weighs nothing."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool([150], 16, 1, 128, 128, e4m3, False, 12)
    seen, _ = seen_by(random_parents(n, torch.Generator().manual_seed(4)))
    q = torch.randn(n, Hq, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    mask, cache, draft = pack(seen, 1).cuda(), b.PagedCache(k, v, ks, vs), int(seen[:, :n - 1].sum(0).float().add(torch.arange(n - 1) * 1e-3).argmax())
    o0, lse0 = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    hit = seen[:, draft].cuda()
    assert hit.any() and not hit.all()
    at = 150 - n + draft
    page, slot = int(table[0, at // 16]), at % 16
    if not e4m3:
        kept = v[page, :, slot].clone()
        v[page, :, slot] = 2.0 ** 120
        o1, _ = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
        ok(handle)
        assert torch.equal(o1[~hit], o0[~hit]) and not torch.equal(o1[hit], o0[hit])
        v[page, :, slot] = kept
    if e4m3:
        k.view(torch.uint8)[page, :, slot] = 0x7F
    else:
        k[page, :, slot] = float("nan")
        k[page, :, slot, ::3] = float("inf")
    o1, lse1 = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    assert torch.equal(o1[~hit], o0[~hit]) and torch.equal(lse1[:, ~hit], lse0[:, ~hit])
    assert torch.isnan(o1[hit]).all() and torch.isnan(lse1[:, hit]).all()
    row = int((~hit).nonzero()[0])
    q[row, 0, 5] = float("nan")
    o2, lse2 = b.forward_paged_tree(handle, q, cache, table, lens_t, mask)
    ok(handle)
    rest = ~hit
    rest[row] = False
    assert torch.isnan(o2[row, 0]).all() and torch.isnan(lse2[0, row]) and torch.equal(o2[rest], o0[rest])


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_scores_of_few_rows(handle, e4m3):
    """Scores in the hundreds, rising maxima, one key far above thousands, scales near zero: as above, in few rows."""
    from paper_2609_21264_b200 import binding
    run(handle, [1000, 77], [7, 6], 8, 2, 128, 128, 16, e4m3, seed=8, q_mult=8.0)
    run(handle, [300, 90], [8, 3], 8, 2, 64, 64, 16, e4m3, seed=8, scale=1e-30)
    k, v, table, lens_t, ks, vs = pool([2000], 32, 2, 128, 128, e4m3, False, 9, poison=False)
    flat = torch.arange(2000, device="cuda")
    ramp = (flat.float() / 2000 * 4 - 2)
    kk = torch.zeros(k.shape, device="cuda")
    kk[table[0, flat // 32].long(), :, flat % 32] = ramp[:, None, None].expand(2000, 2, 128)
    k.copy_((kk * 20).to(k.dtype) if e4m3 else kk.to(k.dtype))
    q = torch.ones(8, 8, 128, device="cuda").bfloat16()
    q[:, ::2] *= -1
    o, lse = binding.forward_paged_tree(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, [2000], [0, 8], [torch.ones(8, 8).tril() > 0], 128 ** -0.5))
    n = 16000
    k, v, table, lens_t, ks, vs = pool([n], 64, 1, 128, 128, e4m3, False, 10, poison=False, shift=0.5)
    kf = torch.zeros(k.shape, device="cuda")
    kf[int(table[0, 3]), 0, 5, :] = 20.0 if e4m3 else 1.0
    k.copy_(kf.to(k.dtype))
    q = torch.full((6, 4, 128), 9.7 * 128 ** 0.5 / 128, device="cuda").bfloat16()
    o, lse = binding.forward_paged_tree(handle, q, binding.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, [n], [0, 6], [torch.ones(6, 6).tril() > 0], 128 ** -0.5))


def test_strides_of_few_rows(handle):
    from paper_2609_21264_b200 import binding as b
    for dqk, dv, e4m3 in ((128, 128, False), (64, 64, True), (192, 128, False)):
        k, v, table, lens_t, ks, vs = pool([300, 40], 16, 2, dqk, dv, e4m3, False, 13)
        wide = torch.randn(2 * 5, 14, dqk, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
        q = wide[:, 2:10]
        out = torch.full((10, 11, dv + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        cache = b.PagedCache(k, v, ks, vs)
        mask = torch.full((10, 3), 9, dtype=torch.int32, device="cuda")[:, :2]
        o, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, mask, out=out[:, 3:, :dv])
        o2, lse2 = b.forward_paged_tree(handle, q.contiguous(), cache, table, lens_t, mask.contiguous())
        ok(handle)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert (out[:, :3] == 7).all() and (out[:, :, dv:] == 7).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_few_rows_refuse_contents_and_give_up(e4m3):
    """Lengths, offsets and pages that cannot be are reported and their sequences left out; a load that never comes ends the call."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, ks, vs = pool([300, 140], 16, 2, 128, 128, e4m3, False, 14)
    q = torch.randn(12, 8, 128, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v, ks, vs)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    h = b.fa_create()
    try:
        good = b.forward_paged_tree(h, q, cache, table, lens_t, None, cu_seqlens=ints(0, 6, 12), max_tokens=8)[0]
        ok(h)
        for cu in (ints(0, 20, 12), ints(-1, 6, 12), ints(6, 3, 12)):
            out = torch.full_like(q, 7.0)
            b.forward_paged_tree(h, q, cache, table, lens_t, None, cu_seqlens=cu, max_tokens=8, out=out)
            torch.cuda.synchronize()
            assert b.fa_last_status(h) == (b.FA_ERR_INVALID_ARG, 0x0904)
        for n in (-1, 10 ** 6):
            o = b.forward_paged_tree(h, q, cache, table.clamp(0, k.shape[0] - 1), ints(n, 140), None, cu_seqlens=ints(0, 6, 12), max_tokens=8)[0]
            torch.cuda.synchronize()
            assert b.fa_last_status(h) == (b.FA_ERR_INVALID_ARG, 0x0901) and torch.equal(o[6:], good[6:])
        bad = table.clone()
        bad[0, 2] = k.shape[0]
        o = b.forward_paged_tree(h, q, cache, bad, lens_t, None, cu_seqlens=ints(0, 6, 12), max_tokens=8)[0]
        torch.cuda.synchronize()
        assert b.fa_last_status(h) == (b.FA_ERR_INVALID_ARG, 0x0902) and torch.equal(o[6:], good[6:])
    finally:
        b.fa_destroy(h)
    h = b.fa_create(flags=b.FA_FLAG_DEBUG_DROP_V_LOAD, wait_limit_ms=20)
    try:
        b.forward_paged_tree(h, q, cache, table, lens_t, None, cu_seqlens=ints(0, 6, 12), max_tokens=8)
        torch.cuda.synchronize()
        st, site = b.fa_last_status(h)
        assert st == b.FA_ERR_DEVICE_TIMEOUT and site != 0 and b.fa_last_kernel_name(h).startswith("fa_tree_few")
    finally:
        b.fa_destroy(h)
