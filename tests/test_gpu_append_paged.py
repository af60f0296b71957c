"""fa_append_paged against the rotation in 64 bits: every stored value, every slot that must stay as it was, refusals."""
import ctypes

import pytest
import torch

from paged_util import BF16_HALF, E4M3_HALF, E4M3_MAX, ok, pool, rope_table, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    from paper_2609_21264_b200 import binding
    h = binding.fa_create()
    yield h
    binding.fa_destroy(h)


def check(handle, lens, counts, Hq, Hkv, dqk, dv, page, e4m3, rope, *, heads_first=False, pad=0, fused=False, in_place=False,
          cu=True, seed=1, stream=None):
    """Appends `counts` new tokens to sequences of the lengths `lens` (new ones included) and compares the whole cache."""
    from paper_2609_21264_b200 import binding
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, dqk, dv, e4m3, heads_first, seed)
    raw = lambda t: t.view(torch.uint8) if e4m3 else t.view(torch.int16)  # noqa: E731
    k0, v0 = raw(k).cpu().clone(), raw(v).cpu().clone()
    g = torch.Generator().manual_seed(seed + 1)
    rows = sum(counts) + pad
    if fused:
        x = torch.randn(rows, Hq + 2 * Hkv, dqk, generator=g).to(torch.bfloat16).cuda()
        q, kn, vn = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        q, kn, vn = (torch.randn(rows, H, d, generator=g).to(torch.bfloat16).cuda() for H, d in ((Hq, dqk), (Hkv, dqk), (Hkv, dv)))
    if e4m3:
        kn[0, 0, :8] = 4000.0         # saturates
        vn[0, 0, :8] = -4000.0
    q_in, kc, vc = q.cpu().double(), kn.cpu().double(), vn.cpu().double()
    q_out = q if in_place else torch.full((rows, Hq, dqk), 7.0, dtype=torch.bfloat16, device="cuda")
    q_before = q_out.cpu().clone()
    dim, offset, span, inter = rope if rope else (0, 0, dqk, False)
    tab = rope_table(max(max(lens), 1), dim) if rope else None
    offs = torch.zeros(len(counts) + 1, dtype=torch.int32)
    offs[1:] = torch.tensor(counts).cumsum(0)
    r = binding.append_paged(handle, kn, vn, binding.PagedCache(k, v, ks, vs), table, lens_t, cu_seqlens=offs.cuda() if cu else None,
                             q=q, q_out=q_out, rope=binding.Rope(tab, offset=offset, span=span, interleaved=inter) if rope else None)
    assert r is q_out
    ok(handle)
    k1, v1, qo = raw(k).cpu(), raw(v).cpu(), q_out.cpu()
    touched = torch.zeros(k.shape[0], page, dtype=torch.bool)
    q_row = torch.zeros(rows, dtype=torch.bool)
    for b, (n, m) in enumerate(zip(lens, counts)):
        for i in range(m):
            pos, t = n - m + i, int(offs[b]) + i
            if pos < 0:
                continue
            q_row[t] = True
            pg, slot = int(table[b, pos // page]), pos % page
            touched[pg, slot] = True
            trow = tab[pos:pos + 1].cpu().double() if rope else None
            kt, size = turned(kc[t:t + 1], trow, dim, offset, span, inter)
            qt, qsize = turned(q_in[t:t + 1], trow, dim, offset, span, inter)
            kg, vg = k.cpu()[pg, :, slot], v.cpu()[pg, :, slot]
            if e4m3:
                kw, vw = kt[0] / ks.cpu().double()[:, None], vc[t] / vs.cpu().double()[:, None]
                size = size / ks.cpu().double()[:, None]
                # one rounding to e4m3 (half of its smallest step, 2^-10, near zero), saturated at 448
                for got, want, s in ((kg, kw, size[0]), (vg, vw, vw.abs())):
                    want = want.clamp(-E4M3_MAX, E4M3_MAX)
                    assert ((got.float().double() - want).abs() <= E4M3_HALF * want.abs() + 2.0 ** -10 + 2.0 ** -20 * s).all()
            else:
                assert ((kg.double() - kt[0]).abs() <= BF16_HALF * kt[0].abs() + 2.0 ** -22 * size[0]).all()
                assert torch.equal(vg.double(), vc[t])
            assert ((qo[t].double() - qt[0]).abs() <= BF16_HALF * qt[0].abs() + 2.0 ** -22 * qsize[0]).all()
    keep = (~touched)[:, None, :, None].expand(k.shape)
    assert torch.equal(k1[keep], k0[keep]) and torch.equal(v1[(~touched)[:, None, :, None].expand(v.shape)], v0[(~touched)[:, None, :, None].expand(v.shape)])
    assert torch.equal(qo[~q_row], q_before[~q_row])          # padding rows and skipped tokens
    return k1, v1, qo


@pytest.mark.parametrize("dqk,dv,rope", [
    (128, 128, (128, 0, 128, False)), (128, 128, (128, 0, 128, True)), (128, 128, None), (128, 128, (64, 0, 64, False)),
    (64, 64, (32, 0, 64, False)), (64, 64, (16, 8, 64, True)), (192, 128, (64, 128, 192, True)), (192, 128, (48, 16, 96, False)),
], ids=["d128", "d128_inter", "d128_none", "d128_span64", "d64_half", "d64_inter_off", "d192_inter", "d192_span96"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_ragged_prompts(handle, dqk, dv, rope, e4m3):
    check(handle, [1, 17, 40, 130, 16], [1, 5, 40, 33, 16], 6, 2, dqk, dv, 16, e4m3, rope, pad=3, heads_first=e4m3)


@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("heads_first", [False, True])
def test_page_sizes_and_orders(handle, page, heads_first):
    check(handle, [300, 48, 49, 1], [2, 48, 1, 1], 4, 4, 128, 128, page, False, (128, 0, 128, False), heads_first=heads_first)


def test_slices_of_one_projection_and_queries_in_place(handle):
    check(handle, [9, 100, 33], [9, 1, 20], 8, 2, 128, 128, 32, False, (128, 0, 128, False), fused=True)
    check(handle, [9, 100, 33], [9, 1, 20], 8, 2, 128, 128, 32, True, (64, 64, 128, False), in_place=True)
    check(handle, [9, 100, 33], [9, 1, 20], 8, 2, 64, 64, 32, False, (64, 0, 64, True), in_place=True, fused=True)


def test_padded_batch_and_equal_counts(handle):
    """Sequences of length 0 (padding of a captured step) are skipped, with and without offsets; a sequence shorter than its new
    tokens stores the ones whose position is not negative."""
    check(handle, [5, 0, 77, 0], [1, 1, 1, 1], 4, 2, 128, 128, 16, False, (128, 0, 128, False), cu=False)
    check(handle, [5, 2, 77, 0], [3, 3, 3, 3], 4, 2, 128, 128, 16, True, (128, 0, 128, True), cu=False)
    check(handle, [5, 0, 77, 3], [1, 0, 4, 5], 4, 2, 128, 128, 16, False, (128, 0, 128, False), pad=2)


def test_many_sequences(handle):
    lens = [(i * 37) % 90 for i in range(300)]
    check(handle, lens, [min(n, 1 + i % 3) if i % 11 else 0 for i, n in enumerate(lens)], 2, 1, 64, 64, 16, False, (64, 0, 64, False), pad=1)


def test_cache_of_more_than_2_31_elements(handle):
    """A page whose elements lie behind 2^31: 64-bit offsets."""
    from paper_2609_21264_b200 import binding
    pages, Hkv, page, d = 17000, 8, 128, 128          # 2.2e9 elements a tensor
    k = torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    kn, vn = torch.randn(3, Hkv, d, device="cuda").bfloat16(), torch.randn(3, Hkv, d, device="cuda").bfloat16()
    lens = torch.tensor([128], dtype=torch.int32, device="cuda")
    binding.append_paged(handle, kn, vn, binding.PagedCache(k, v), table, lens)
    ok(handle)
    assert torch.equal(k[pages - 1, :, 125:].transpose(0, 1), kn) and torch.equal(v[pages - 1, :, 125:].transpose(0, 1), vn)


def test_captured_call_follows_new_lengths_and_tables(handle):
    from paper_2609_21264_b200 import binding
    k, v, table, lens, _, _ = pool([5, 40], 16, 2, 128, 128, False, False, 3, poison=False, spare=6)
    kn, vn, q = (torch.randn(2, H, 128, device="cuda").bfloat16() for H in (2, 2, 4))
    tab = rope_table(64, 128)
    cache, rope, out = binding.PagedCache(k, v), binding.Rope(tab), torch.empty_like(q)
    binding.append_paged(handle, kn, vn, cache, table, lens, q=q, q_out=out, rope=rope)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.append_paged(handle, kn, vn, cache, table, lens, q=q, q_out=out, rope=rope)
    lens.copy_(torch.tensor([6, 41], dtype=torch.int32))
    kn.copy_(torch.randn_like(kn))
    graph.replay()
    ok(handle)
    k2, v2 = k.clone(), v.clone()
    k.zero_()
    v.zero_()
    binding.append_paged(handle, kn, vn, cache, table, lens, q=q, q_out=out, rope=rope)
    ok(handle)
    for b, n in enumerate((6, 41)):
        pg, slot = int(table[b, (n - 1) // 16]), (n - 1) % 16
        assert torch.equal(k2[pg, :, slot], k[pg, :, slot]) and torch.equal(v2[pg, :, slot], v[pg, :, slot])
        assert k[pg, :, slot].abs().sum() > 0


def test_contents_the_device_refuses(handle):
    """A page outside the pool, a length past the block table, a position past the rotation table: reported, nothing stored."""
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens, _, _ = pool([20, 40], 16, 2, 64, 64, False, False, 4, poison=False)
    kn, vn = (torch.randn(2, 2, 64, device="cuda").bfloat16() for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    bad = table.clone()
    bad[0, 1], bad[1, 2] = -1, k.shape[0]
    b.append_paged(handle, kn, vn, b.PagedCache(k, v), bad, lens)
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0902) and torch.equal(k, k0) and torch.equal(v, v0)
    b.append_paged(handle, kn, vn, b.PagedCache(k, v), table, torch.full_like(lens, 1000))
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0901) and torch.equal(k, k0)
    b.append_paged(handle, kn, vn, b.PagedCache(k, v), table, lens, rope=b.Rope(rope_table(19, 64)))
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0903) and torch.equal(k, k0)
    assert b.fa_last_status(handle) == (b.FA_OK, 0)


def test_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens, _, _ = pool([20], 16, 2, 64, 64, False, False, 5)
    kn, vn, q = (torch.randn(1, H, 64, device="cuda").bfloat16() for H in (2, 2, 4))
    cache = b.PagedCache(k, v)
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 1, table.data_ptr(), table.shape[1], lens.data_ptr(), table.shape[1], 0)
    tab = rope_table(64, 64)

    def call(c=None, s=None, total=1, kp=kn.data_ptr(), qp=None, qo=None, Hq=0, st=(128, 64), rope=None, h=handle):
        return b.fa_append_paged(h, c or cache.c, s or seqs, None, total, kp, vn.data_ptr(), qp, qo, Hq, st, (128, 64), (256, 64), (256, 64), rope)

    def cache_with(**kw):
        c = b.fa_paged_cache.from_buffer_copy(cache.c)
        for name, x in kw.items():
            setattr(c, name, x)
        return c

    def seqs_with(**kw):
        c = b.fa_paged_seqs.from_buffer_copy(seqs)
        for name, x in kw.items():
            setattr(c, name, x)
        return c

    assert call() == b.FA_OK and call(total=0) == b.FA_OK
    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call(h=None) == bad and call(total=-1) == bad and call(kp=None) == bad and call(kp=kn.data_ptr() + 2) == bad
    assert call(st=(128, 60)) == bad and call(st=(0, 64)) == bad and call(qp=q.data_ptr()) == bad
    assert call(qp=q.data_ptr(), qo=q.data_ptr(), Hq=0) == bad
    for kw, want in (({"struct_size": 8}, bad), ({"type": 2}, bad), ({"k": None}, bad), ({"num_pages": 0}, bad), ({"page_size": 24}, no),
                     ({"dqk": 96}, no), ({"k_scale": tab.data_ptr()}, bad), ({"reserved": 1}, bad)):
        assert call(c=cache_with(**kw)) == want, kw
    for kw, want in (({"struct_size": 8}, bad), ({"B": -1}, bad), ({"block_table": None}, bad), ({"seq_lens": None}, bad),
                     ({"table_stride": 0}, bad), ({"max_pages": 0}, bad), ({"B": 0}, b.FA_OK),
                     ({"max_pages": 2 ** 30, "table_stride": 2 ** 30}, no)):
        assert call(s=seqs_with(**kw)) == want, kw
    size = ctypes.sizeof(b.fa_rope)
    for args, want in (((size, 64, tab.data_ptr(), 64, 0, 64, 0), b.FA_OK), ((size, 64, tab.data_ptr(), 24, 0, 64, 0), no),
                       ((size, 64, tab.data_ptr(), 64, 8, 64, 0), bad), ((size, 64, tab.data_ptr(), 32, 4, 64, 0), no),
                       ((size, 64, tab.data_ptr(), 32, 0, 48, 0), bad), ((size, 0, tab.data_ptr(), 64, 0, 64, 0), bad),
                       ((size, 64, None, 64, 0, 64, 0), bad), ((8, 64, tab.data_ptr(), 64, 0, 64, 0), bad)):
        assert call(rope=b.fa_rope(*args)) == want, args
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        b.append_paged(handle, kn.float(), vn, cache, table, lens)
    with pytest.raises(ValueError):
        b.append_paged(handle, kn, vn, cache, table.long(), lens)
    with pytest.raises(ValueError):
        b.append_paged(handle, kn[:, :1], vn[:, :1], cache, table, lens)
    with pytest.raises(ValueError):
        b.append_paged(handle, kn, vn, cache, table, lens, q_out=q)
    with pytest.raises(ValueError):
        b.PagedCache(k, v.float())
    with pytest.raises(b.FaError):
        b.append_paged(handle, torch.cat([kn, kn, kn]), torch.cat([vn, vn, vn]), cache, table.expand(2, -1).contiguous(), lens.expand(2).contiguous())


def test_negative_lengths_are_reported_and_empty_batches_are_nothing(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens, _, _ = pool([20, 40], 16, 2, 64, 64, False, False, 6, poison=False)
    kn, vn = (torch.randn(2, 2, 64, device="cuda").bfloat16() for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    cache = b.PagedCache(k, v)
    for least in (-1, -2 ** 31):
        b.append_paged(handle, kn, vn, cache, table, torch.full_like(lens, least))
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0901) and torch.equal(k, k0) and torch.equal(v, v0)
    b.append_paged(handle, kn[:0], vn[:0], cache, table[:0], lens[:0])
    assert b.append_paged(handle, kn[:0], vn[:0], cache, table[:0], lens[:0], q=kn[:0]).shape == (0, 2, 64)
    ok(handle)
    assert torch.equal(k, k0)


def test_more_heads_than_a_call_may_have(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens, _, _ = pool([20], 16, 2, 64, 64, False, False, 7)
    kn = torch.randn(1, 2, 64, device="cuda").bfloat16()
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 1, table.data_ptr(), table.shape[1], lens.data_ptr(), table.shape[1], 0)
    c = b.fa_paged_cache.from_buffer_copy(b.PagedCache(k, v).c)
    call = lambda Hq: b.fa_append_paged(handle, c, seqs, None, 1, kn.data_ptr(), kn.data_ptr(), kn.data_ptr(), kn.data_ptr(), Hq,  # noqa: E731
                                        (128, 64), (128, 64), (128, 64), (128, 64), None)
    assert call(65536) == b.FA_ERR_UNSUPPORTED and call(65535) == b.FA_ERR_UNSUPPORTED       # (too many 32-byte units a token)
    c.Hkv = 2 ** 31 - 1
    assert call(2) == b.FA_ERR_UNSUPPORTED


def test_one_rotation_for_two_head_sizes(handle):
    """span 0 is the whole head of whichever cache a call has."""
    from paper_2609_21264_b200 import binding as b
    rope, tab = None, rope_table(64, 64)
    rope = b.Rope(tab)
    for d, dv in ((64, 64), (192, 128), (128, 128), (64, 64)):
        k, v, table, lens, _, _ = pool([37], 16, 2, d, dv, False, False, 8, poison=False)
        kn = torch.randn(1, 2, d, device="cuda").bfloat16()
        b.append_paged(handle, kn, torch.randn(1, 2, dv, device="cuda").bfloat16(), b.PagedCache(k, v), table, lens, rope=rope)
        ok(handle)
        x, cs = kn[0].double(), tab[36].double()
        lo, hi, c, s = x[:, :32], x[:, 32:64], cs[:32], cs[32:]
        want = torch.cat([lo * c - hi * s, hi * c + lo * s, x[:, 64:]], 1)
        got = k[int(table[0, 2]), :, 4].double()
        # one rounding to bf16, fp32 products of numbers below 8 before it
        assert ((got - want).abs() <= want.abs() * 2.0 ** -8 + 8 * 2.0 ** -22).all()


def test_a_cache_of_one_page_and_head_with_strides_of_no_use(handle):
    from paper_2609_21264_b200 import binding as b
    store = torch.zeros(2, 64, 128, device="cuda").bfloat16()
    k, v = (x.as_strided((1, 1, 64, 128), (0, 3, 128, 1), x.storage_offset()) for x in store)
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")
    kn, vn, q = (torch.randn(5, 1, 128, device="cuda").bfloat16() for _ in range(3))
    cache = b.PagedCache(k, v)
    b.append_paged(handle, kn, vn, cache, table, lens)
    o, _ = b.forward_paged(handle, q[:1], cache, table, lens)
    ok(handle)
    assert torch.equal(store[0, :5], kn[:, 0]) and torch.equal(store[1, :5], vn[:, 0]) and not store[:, 5:].any()
    w = torch.softmax(q[0].double() @ kn[:, 0].double().t() * 128 ** -0.5, 1)
    want = w @ vn[:, 0].double()
    # probabilities and result rounded to bf16
    assert ((o[0].double() - want).abs() <= 2.0 ** -8 * (w @ vn[:, 0].double().abs() + want.abs()) + 3e-4).all()
