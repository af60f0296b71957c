"""fa_forward_paged_tree with more than 32 rows, where the calls of other tests are few rows or say nothing about the kernel: every test looks
at the name of the kernel that ran."""
import pytest
import torch

from draft_util import pack, tree_reference
from paged_util import BF16_HALF, FP32_SLACK, assert_attention, ok, pool, rows_of
from test_gpu_tree import run

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


@pytest.mark.parametrize("dqk,dv,e4m3", [(64, 64, False), (128, 128, False), (192, 128, False), (128, 128, True), (192, 128, True)])
def test_contents_the_device_refuses(handle, dqk, dv, e4m3):
    """Pages outside the pool, lengths past the table, rows that are not the call's: reported, other sequences hold."""
    from paper_2609_21264_b200 import binding as b
    lens = [40, 300]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, e4m3, False, 42)
    q = torch.randn(12, 16, dqk, generator=torch.Generator().manual_seed(43)).to(torch.bfloat16).cuda()
    cache, pages = b.PagedCache(k, v, ks, vs), k.shape[0]
    good, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    ok(handle)
    kernel_was(handle, 48, e4m3)
    O, L, A = tree_reference(q, k, v, ks, vs, table, lens, [0, 6, 12], [torch.ones(6, 6).tril() > 0] * 2, dqk ** -0.5)
    assert_attention(good, lse, O, L, A)

    def holds(o, lse):           # (other lengths deal the work out otherwise: the same values, within their rounding)
        assert_attention(o[6:], lse[:, 6:], O[6:], L[:, 6:], A[6:])

    def reported(site):
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, site)

    for page in (-1, pages, 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[0, 1] = page
        o = b.forward_paged_tree(handle, q, cache, bad, lens_t, None)
        reported(0x0902)
        holds(*o)
    for n in (-1, -2 ** 31, 16 * table.shape[1] + 1, 2 ** 31 - 1):
        bad = lens_t.clone()
        bad[0] = n
        o = b.forward_paged_tree(handle, q, cache, table.clamp(0, pages - 1), bad, None)
        reported(0x0901)
        holds(*o)
    # (the second sequence keeps its rows 6 to 11 where its offsets are sound; with five drafts at most neither does)
    for cu, most in (([-3, 6, 12], 10), ([7, 6, 12], 10), ([0, 6, 13], 10), ([0, 6, 2 ** 31 - 1], 10), ([-2 ** 31, 6, 12], 10), ([0, 6, 12], 5)):
        out = torch.full_like(good, 7)
        _, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), max_tokens=most,
                                      out=out)
        reported(0x0904)
        kernel_was(handle, 8 * most, e4m3)
        if cu[2] == 12 and most == 10:
            holds(out, lse)
        else:
            assert (out[6:] == 7).all()
        if cu[:2] != [0, 6] or most == 5:
            assert (out[:6] == 7).all()
    assert b.fa_last_status(handle) == (b.FA_OK, 0)


@pytest.mark.parametrize("B,dqk,dv,e4m3", [(1500, 64, 64, False), (1500, 64, 64, True), (200, 192, 128, False), (200, 128, 128, True)])
def test_many_sequences(handle, B, dqk, dv, e4m3):
    """More sequences than a warp has lanes many times over, most of them short, some without drafts or without keys."""
    lens = [(i * 29) % 150 + (3000 if i % 97 == 5 else 0) for i in range(B)]
    counts = [min(n, i % 4) for i, n in enumerate(lens)]
    run(handle, lens, counts, 12, 1, dqk, dv, 16, e4m3, seed=26, pad=1)
    kernel_was(handle, 36, e4m3)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_agrees_with_the_paged_call(handle, e4m3, dqk, dv):
    """Chains of up to 16 tokens are what fa_forward_paged computes, by another kernel: both within their roundings of the definition, and so
    within twice that of each other."""
    from paper_2609_21264_b200 import binding as b
    lens, n = [300, 5, 129, 1000], 5
    k, v, table, lens_t, ks, vs = pool(lens, 32, 2, dqk, dv, e4m3, False, 44)
    q = torch.randn(4 * n, 16, dqk, generator=torch.Generator().manual_seed(45)).to(torch.bfloat16).cuda()
    cache = b.PagedCache(k, v, ks, vs)
    o, lse = b.forward_paged_tree(handle, q, cache, table, lens_t, None)
    ok(handle)
    kernel_was(handle, 8 * n, e4m3)
    o2, lse2 = b.forward_paged(handle, q, cache, table, lens_t)
    ok(handle)
    assert b.fa_last_kernel_name(handle) == ("fa_paged_e4m3" if e4m3 else "fa_paged")
    O, L, A = tree_reference(q, k, v, ks, vs, table, lens, [n * i for i in range(5)], [torch.ones(n, n).tril() > 0] * 4, dqk ** -0.5)
    for got in ((o, lse), (o2, lse2)):
        assert_attention(*got, O, L, A)
    tol = 2 * (BF16_HALF * O.abs() + (BF16_HALF + FP32_SLACK) * A) + 1e-30
    assert ((o.cpu().double() - o2.cpu().double()).abs() <= tol).all()


@pytest.mark.parametrize("n", [4, 10], ids=["32rows", "80rows"])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_bits_of_probabilities_over_an_8_bit_cache(handle, n, dqk, dv):
    """A key of weight 1 and 96 of weight w, a little below it, whose values (-96, and 1 each) all but cancel: what is left of the output is below
    what a probability of fewer bits is off by.

    P is held relative to the first key's, whose is a power of two, so its own rounding is nothing.  More than 32 rows: an fp16 number, off by 2^-11
    of it at most.  Up to 32: that number as three terms of three bits each, counted from each one's leading bit, so 9 of its 11 bits at least, and what
    is cut off is 3 * 2^-10 of the leading one at most.  Scores are a product of two numbers; the factor and the exponent, below 2^4 in size, are off
    by some 2^-19, the exponential by 2^-22."""
    from paper_2609_21264_b200 import binding as b
    keys = 97
    k, v, table, lens_t, _, _ = pool([keys + n], 16, 1, dqk, dv, True, False, 46, poison=False)
    kf, vf = torch.zeros(k.shape), torch.zeros(v.shape)
    at = torch.arange(keys)
    page, slot = table.cpu()[0, at // 16].long(), at % 16
    kf[page[1:], 0, slot[1:], 0] = -1.0
    vf[page[1:], 0, slot[1:]] = 1.0
    vf[page[0], 0, slot[0]] = -96.0
    k.copy_(kf.to(k.dtype))
    v.copy_(vf.to(v.dtype))
    q = torch.zeros(n, 8, dqk)
    q[:, :, 0] = torch.linspace(2.0 ** -9, 2.0 ** -5, n * 8).reshape(n, 8)
    q = q.to(torch.bfloat16)
    mask = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    o, lse = b.forward_paged_tree(handle, q.cuda(), b.PagedCache(k, v), table, lens_t, mask, scale=1.0)
    ok(handle)
    kernel_was(handle, 8 * n, True)
    O, L, A = tree_reference(q, k, v, None, None, table, [keys + n], [0, n], [torch.zeros(n, n) > 0], 1.0)
    few = 8 * n <= 32
    tol = BF16_HALF * O.abs() + (2.0 ** -11 + (3 * 2.0 ** -10 if few else 0.0) + 2.0 ** -16) * A
    w = torch.exp(-q[:, :, 0].double())
    short = torch.floor(w * 64) / 64 if few else w.to(torch.bfloat16).double()          # two terms, or bf16
    assert (((96 * short - 96) / (96 * w + 1) - O[:, :, 0]).abs() / tol[:, :, 0]).max() > 1.5          # (would be seen)
    worst = ((o.cpu().double() - O).abs() / tol).max().item()
    assert worst <= 1.0, worst
    assert ((lse.cpu().double() - L).abs() <= FP32_SLACK).all()


def far_scores(shift, n, dqk, dv, e4m3, below=False, seed=50):
    """Queries of 2^shift, so scores far beyond what the bits of a 32-bit number behind the point hold (below: all of them negative), and what comes
    out: the value of each row's best key, which leads by more than a score's 32-bit sum of products can be off by and e^30 has room for."""
    lens = [300, 40, 150] if below else [1500, 140, 700]
    k, v, table, lens_t, ks, vs = pool(lens, 16, 2, dqk, dv, e4m3, False, seed)
    q = torch.randn(3 * n, 8, dqk, generator=torch.Generator().manual_seed(seed + 1)).to(torch.bfloat16) * 2.0 ** shift
    if below:
        q = q.abs()
        k = (k.view(torch.uint8) | 0x80).view(k.dtype) if e4m3 else -k.abs()
    for b, keys in enumerate(lens):
        kd = rows_of(k, ks, table, b, keys)
        for h in range(8):
            x = q[b * n:(b + 1) * n, h].double()
            z = (x @ kd[h // 4].T).masked_fill(torch.arange(keys)[None] > torch.arange(keys - n, keys)[:, None], -float("inf"))
            best = z.topk(2, 1)
            off = (x.abs() @ kd[h // 4].abs().T).gather(1, best.indices).sum(1) * dqk * 2.0 ** -24
            assert ((best.values[:, 0] - best.values[:, 1] - off) * dqk ** -0.5 > 30).all()
    ref = tree_reference(q, k, v, ks, vs, table, lens, [0, n, 2 * n, 3 * n], [torch.ones(n, n).tril() > 0] * 3, dqk ** -0.5)
    return q.cuda(), (k, v, ks, vs), table, lens_t, ref


FAR = [20, 22, 23, 24, 25, 26, 27, 28, 30, 34, 60]


@pytest.mark.parametrize("shift", FAR)
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_scores_of_any_size_few_rows(handle, e4m3, dqk, dv, shift):
    from paper_2609_21264_b200 import binding as b
    q, (k, v, ks, vs), table, lens_t, ref = far_scores(shift, 4, dqk, dv, e4m3)
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    kernel_was(handle, 16, e4m3)
    assert_attention(o, lse, *ref)
    o, lse = b.forward_paged(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t)
    ok(handle)
    assert_attention(o, lse, *ref)


@pytest.mark.parametrize("shift", FAR)
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_scores_of_any_size(handle, e4m3, dqk, dv, shift):
    from paper_2609_21264_b200 import binding as b
    q, (k, v, ks, vs), table, lens_t, ref = far_scores(shift, 11, dqk, dv, e4m3)
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    kernel_was(handle, 44, e4m3)
    assert_attention(o, lse, *ref)


@pytest.mark.parametrize("shift", FAR)
@pytest.mark.parametrize("n", [4, 11], ids=["16rows", "44rows"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_scores_far_below_zero(handle, e4m3, n, shift):
    from paper_2609_21264_b200 import binding as b
    q, (k, v, ks, vs), table, lens_t, ref = far_scores(shift, n, 128, 128, e4m3, below=True, seed=60)
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, None)
    ok(handle)
    kernel_was(handle, 4 * n, e4m3)
    assert_attention(o, lse, *ref)


@pytest.mark.parametrize("shift", [10, 24, 28, 34])
@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_far_scores_of_rows_that_see_one_key(handle, e4m3, dqk, dv, shift):
    """Every token sees itself alone, so most rows see nothing of their first tile of keys: the only score is the reference, however far out it is
    (q = +-k, so half of them are far above zero and half far below)."""
    from paper_2609_21264_b200 import binding as b
    n = 200
    k, v, table, lens_t, ks, vs = pool([n], 16, 1, dqk, dv, e4m3, False, 70)
    keys = rows_of(k, None, table, 0, n)[0]
    sign = torch.where(torch.arange(n) % 3 == 0, -1.0, 1.0)
    q = ((keys * sign[:, None])[:, None].expand(n, 2, dqk) * 2.0 ** shift).to(torch.bfloat16).cuda()
    seen = torch.eye(n) > 0
    o, lse = b.forward_paged_tree(handle, q, b.PagedCache(k, v, ks, vs), table, lens_t, pack(seen, 7).cuda())
    ok(handle)
    kernel_was(handle, 400, e4m3)
    assert_attention(o, lse, *tree_reference(q, k, v, ks, vs, table, [n], [0, n], [seen], dqk ** -0.5))
