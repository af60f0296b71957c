"""Tree layout, append at given positions, compaction and page copies: every value of what they write, and what must stay."""
import ctypes

import pytest
import torch

from draft_util import pack, random_parents, seen_by, tree_reference
from paged_util import BF16_HALF, E4M3_HALF, E4M3_MAX, assert_attention, ok, pool, rope_table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    from paper_2609_21264_b200 import binding
    h = binding.fa_create()
    yield h
    binding.fa_destroy(h)


def offsets_of(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------- layout

@pytest.mark.parametrize("most", [1, 5, 32, 33, 64, 65, 128, 129, 200, 256])
@pytest.mark.parametrize("shape", ["random", "chain", "roots", "star"])
def test_layout(handle, most, shape):
    from paper_2609_21264_b200 import binding as b
    g = torch.Generator().manual_seed(most)
    counts = [most, max(1, most // 2), 0, 1, most - 1]
    lens = [most + 10, 500, 0, 1, max(0, most - 3)]          # the last has drafts in front of position 0
    make = {"random": lambda n: random_parents(n, g), "chain": lambda n: list(range(-1, n - 1)), "roots": lambda n: [-1] * n,
            "star": lambda n: [-1] + [0] * (n - 1) if n else []}[shape]
    trees = [make(n) for n in counts]
    offs = offsets_of(counts)
    parents = ints(sum(trees, []) + [5, 5])                   # two rows behind the last sequence
    words = (most + 31) // 32
    mask = torch.full((offs[-1] + 2, words + 1), 77, dtype=torch.int32, device="cuda")
    pos = torch.full((offs[-1] + 2,), 77, dtype=torch.int32, device="cuda")
    r = b.tree_layout(handle, parents, ints(lens), cu_seqlens=ints(offs), max_tokens=most, mask=mask, positions=pos)
    ok(handle)
    assert r[0] is mask and r[1] is pos
    for i, (t, n) in enumerate(zip(trees, lens)):
        seen, depth = seen_by(t)
        here = slice(offs[i], offs[i + 1])
        assert torch.equal(mask[here, :words].cpu(), pack(seen, words))
        assert pos[here].tolist() == [n - len(t) + d for d in depth]
    assert (mask[:, words:] == 77).all() and (mask[offs[-1]:] == 77).all() and (pos[offs[-1]:] == 77).all()


def test_layout_of_equal_trees_and_many_sequences(handle):
    from paper_2609_21264_b200 import binding as b
    g = torch.Generator().manual_seed(2)
    trees = [random_parents(9, g) for _ in range(300)]
    lens = [9 + i for i in range(300)]
    mask, pos = b.tree_layout(handle, ints(sum(trees, [])), ints(lens))
    ok(handle)
    assert mask.shape == (2700, 1)
    for i in (0, 1, 150, 299):
        seen, depth = seen_by(trees[i])
        assert torch.equal(mask[9 * i:9 * i + 9].cpu(), pack(seen, 1)) and pos[9 * i:9 * i + 9].tolist() == [i + d for d in depth]


def test_layout_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    parents, lens = ints([-1, 0, 1, 2]), ints([9, 9])
    for bad in (1, 3, -2, 2 ** 31 - 1):           # not smaller than its own number (draft 1 of the second sequence)
        p = parents.clone()
        p[3] = bad
        mask, pos = b.tree_layout(handle, ints([-1, 0, -1, bad]), lens)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0905)
        assert mask[:, 0].tolist() == [1, 3, 1, 2] and pos.tolist() == [7, 8, 7, 7]
    for cu in ([-1, 2, 4], [3, 2, 4], [0, 2, 5], [0, 2, 2 ** 31 - 1]):
        b.tree_layout(handle, ints([-1, 0, -1, 0]), lens, cu_seqlens=ints(cu), max_tokens=3)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0904)
    call = lambda h=handle, par=parents.data_ptr(), cu=None, total=4, B=2, ln=lens.data_ptr(), most=2, m=parents.data_ptr(), ms=1, p=None: b.fa_tree_layout(  # noqa: E731
        h, par, cu, total, B, ln, most, m, ms, p)
    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call(h=None) == bad and call(total=-1) == bad and call(B=-1) == bad and call(most=0) == bad and call(most=257, ms=9) == no
    assert call(par=None) == bad and call(par=2) == bad and call(most=33) == bad and call(total=5) == bad and call(total=6) == bad
    assert call(ln=None, p=parents.data_ptr()) == bad and call(total=0) == b.FA_OK and call(B=0) == b.FA_OK and call(m=None) == b.FA_OK
    for args, kw in (((parents.long(), lens), {}), ((parents, lens.long()), {}), ((parents.view(2, 2), lens), {}), ((parents, lens), {"max_tokens": -1}),
                     ((parents, lens), {"cu_seqlens": ints([0, 2, 4])}), ((parents, lens), {"mask": parents}), ((parents, lens), {"positions": lens})):
        with pytest.raises(ValueError):
            b.tree_layout(handle, *args, **kw)
    with pytest.raises(b.FaError):
        b.tree_layout(handle, parents[:3], lens)
    ok(handle)


# ------------------------------------------------------------------------------------------------- append at given positions

AXES = {"one": (1, lambda i, p: 0), "two halves": (2, lambda i, p: 2 * i // p), "three sections": (3, lambda i, p: min(2, (5 * i // p + 1) // 2)),
        "three in turns": (3, lambda i, p: i % 3), "four ragged": (4, lambda i, p: min(3, i // 5))}


@pytest.mark.parametrize("axes", list(AXES))
@pytest.mark.parametrize("dqk,dv,rope", [(128, 128, (128, 0, 128, False)), (128, 128, (128, 0, 128, True)), (64, 64, (16, 8, 64, True)),
                                         (128, 128, (64, 0, 64, False)), (192, 128, (192, 0, 192, False)), (192, 128, (48, 16, 96, True))])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_append_at_positions(handle, axes, dqk, dv, rope, e4m3):
    from paper_2609_21264_b200 import binding as b
    n_axes, axis = AXES[axes]
    dim, offset, span, inter = rope
    lens, counts, Hq, Hkv, pad = [1, 17, 0, 130, 16], [1, 5, 3, 33, 16], 6, 2, 2
    offs = offsets_of(counts)
    T = offs[-1] + pad
    k, v, table, lens_t, ks, vs = pool(lens, 16, Hkv, dqk, dv, e4m3, e4m3, 3)
    before = [x.view(torch.uint8 if e4m3 else torch.int16).clone() for x in (k, v)]
    g = torch.Generator().manual_seed(4)
    q, kn, vn = (torch.randn(T, H, d, generator=g).to(torch.bfloat16).cuda() for H, d in ((Hq, dqk), (Hkv, dqk), (Hkv, dv)))
    tab = rope_table(50, dim)
    pos = torch.randint(0, 50, (n_axes, T), generator=g).to(torch.int32)
    pos[:, offs[2]:offs[3]] = 99                              # (tokens in front of position 0 and padding: not looked at)
    pos[:, offs[-1]:] = -5
    wide = torch.zeros(n_axes, T + 3, dtype=torch.int32)
    wide[:, :T] = pos
    numbers = [axis(i, dim // 2) for i in range(dim // 2)]
    out = torch.full((T, Hq, dqk), 7.0, dtype=torch.bfloat16, device="cuda")
    positions = wide.cuda()[:, :T]
    b.append_paged(handle, kn, vn, b.PagedCache(k, v, ks, vs), table, lens_t, cu_seqlens=ints(offs), q=q, q_out=out,
                   rope=b.Rope(tab, offset=offset, span=span, interleaved=inter, axis_of_pair=numbers if n_axes > 1 else None),
                   positions=positions[0] if n_axes == 1 else positions)
    ok(handle)
    rows, half, tab64 = pos.clamp(0, 49), dim // 2, tab.cpu().double()
    cos = torch.stack([tab64[rows[numbers[i]].long(), i] for i in range(half)], 1)
    sin = torch.stack([tab64[rows[numbers[i]].long(), half + i] for i in range(half)], 1)

    def want(x):
        x = x.cpu().double()
        y, size = x.clone(), x.abs()
        for first in range(offset, dqk, span):
            for i in range(half):
                p, r = (first + 2 * i, first + 2 * i + 1) if inter else (first + i, first + half + i)
                c, s = cos[:, i, None], sin[:, i, None]
                y[:, :, p], y[:, :, r] = x[:, :, p] * c - x[:, :, r] * s, x[:, :, r] * c + x[:, :, p] * s
                size[:, :, p] = size[:, :, r] = x[:, :, p].abs() + x[:, :, r].abs()
        return y, size

    kw, k_size = want(kn)
    qw, q_size = want(q)
    live = torch.zeros(T, dtype=torch.bool)
    touched = torch.zeros(k.shape[0], 16, dtype=torch.bool)
    for i, (n, m) in enumerate(zip(lens, counts)):
        for j in range(m):
            t, at = offs[i] + j, n - m + j
            if at < 0:
                continue
            live[t] = True
            page, slot = int(table[i, at // 16]), at % 16
            touched[page, slot] = True
            for got, x, size, sc in ((k, kw[t], k_size[t], ks), (v, vn[t].cpu().double(), vn[t].cpu().double().abs(), vs)):
                y = got[page, :, slot].float().cpu().double()
                if e4m3:
                    x, size = (x / sc.cpu().double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX), size / sc.cpu().double()[:, None]
                    assert ((y - x).abs() <= E4M3_HALF * x.abs() + 2.0 ** -10 + 2.0 ** -20 * size).all()
                else:
                    assert ((y - x).abs() <= BF16_HALF * x.abs() + 2.0 ** -22 * size).all()
    o = out.cpu().double()
    assert ((o[live] - qw[live]).abs() <= BF16_HALF * qw[live].abs() + 2.0 ** -22 * q_size[live]).all()
    assert (o[~live] == 7).all()
    for x, old in zip((k, v), before):
        keep = (~touched)[:, None, :, None].expand(x.shape).cuda()
        assert torch.equal(x.view(old.dtype)[keep], old[keep])


def test_given_positions_that_follow_the_slots_change_nothing(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([40, 9], 16, 2, 128, 128, False, False, 5, poison=False)
    g = torch.Generator().manual_seed(6)
    kn, vn, q = (torch.randn(14, H, 128, generator=g).to(torch.bfloat16).cuda() for H in (2, 2, 6))
    cu, tab = ints([0, 7, 14]), rope_table(64, 128)
    one = b.append_paged(handle, kn, vn, b.PagedCache(k, v), table, lens_t, cu_seqlens=cu, q=q, rope=b.Rope(tab))
    k1 = k.clone()
    k.zero_()
    pos = ints(list(range(33, 40)) + list(range(2, 9)))
    two = b.append_paged(handle, kn, vn, b.PagedCache(k, v), table, lens_t, cu_seqlens=cu, q=q, rope=b.Rope(tab, axis_of_pair=[0, 1] * 32),
                         positions=pos.expand(2, 14).contiguous())
    ok(handle)
    assert torch.equal(one, two)
    for b_, (n, m) in enumerate(((40, 7), (9, 7))):
        for at in range(n - m, n):
            assert torch.equal(k[int(table[b_, at // 16]), :, at % 16], k1[int(table[b_, at // 16]), :, at % 16])


def test_append_at_positions_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([20, 40], 16, 2, 64, 64, False, False, 7, poison=False)
    kn, q = torch.randn(2, 2, 64, device="cuda").bfloat16(), torch.randn(2, 4, 64, device="cuda").bfloat16()
    cache, tab = b.PagedCache(k, v), rope_table(30, 64)
    rope3 = b.Rope(tab, axis_of_pair=[0, 1, 2, 0] * 8)
    k0 = k.clone()
    for axis in range(3):
        for bad in (-1, 30, 2 ** 31 - 1, -2 ** 31):
            pos = ints([[1, 2]] * 3)
            pos[axis, 0] = bad
            out = torch.full_like(q, 7)
            b.append_paged(handle, kn, kn, cache, table, lens_t, q=q, q_out=out, rope=rope3, positions=pos)
            torch.cuda.synchronize()
            assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0903)
            at = int(table[0, 1]), 3                     # the first sequence's token, position 19
            assert torch.equal(k[at[0], :, at[1]], k0[at[0], :, at[1]]) and (out[0] == 7).all() and (out[1] != 7).any()
    seqs = b.fa_paged_seqs(ctypes.sizeof(b.fa_paged_seqs), 2, table.data_ptr(), table.stride(0), lens_t.data_ptr(), table.shape[1], 0)
    rope = b.fa_rope(ctypes.sizeof(b.fa_rope), 30, tab.data_ptr(), 64, 0, 64, 0)
    numbers = (ctypes.c_uint8 * 32)(*[0, 1] * 16)
    pos = ints([[1, 2]] * 2)
    size = ctypes.sizeof(b.fa_positions)
    call = lambda p, r=rope: b.fa_append_paged_at(handle, cache.c, seqs, None, 2, kn.data_ptr(), kn.data_ptr(), None, None, 0, (128, 64), (128, 64),  # noqa: E731
                                                  None, None, r, p)
    good = (size, 2, pos.data_ptr(), 2, ctypes.addressof(numbers))
    bad, no = b.FA_ERR_INVALID_ARG, b.FA_ERR_UNSUPPORTED
    assert call(b.fa_positions(*good)) == b.FA_OK and call(None) == b.FA_OK and call(b.fa_positions(*good), None) == bad
    torch.cuda.synchronize()
    assert b.fa_last_status(handle) == (bad, 0x0903)          # (without given positions the second token's is 39)
    for i, x, want in ((0, 8, bad), (1, 0, bad), (1, -1, bad), (1, 5, no), (1, 1, bad), (2, None, bad), (2, 2, bad), (3, 1, bad)):
        assert call(b.fa_positions(*[x if j == i else y for j, y in enumerate(good)])) == want, (i, x)
    for kw in ({"positions": pos}, {"positions": pos, "rope": rope3}, {"positions": pos.long(), "rope": b.Rope(tab)}, {"positions": pos.cpu(), "rope": b.Rope(tab)},
               {"positions": ints([1]), "rope": b.Rope(tab)}, {"positions": ints([[1, 2]] * 5), "rope": b.Rope(tab)}):
        with pytest.raises(ValueError):
            b.append_paged(handle, kn, kn, cache, table, lens_t, **kw)
    for numbers in ([0] * 31, [0] * 31 + [4], [-1] * 32):
        with pytest.raises(ValueError):
            b.Rope(tab, axis_of_pair=numbers)
    ok(handle)


# ------------------------------------------------------------------------------------------------- compaction

def layers_of(k, v, n, b, ks=None, vs=None):
    """n layers of caches with contents of their own."""
    pools = [(k, v)] + [(k.clone(), v.clone()) for _ in range(n - 1)]
    for i, (x, y) in enumerate(pools):
        for t in (x, y):
            raw = t.view(torch.uint8)
            raw ^= (37 * i) % 256
    return pools, b.PagedCaches([b.PagedCache(x, y, ks, vs) for x, y in pools])


@pytest.mark.parametrize("dqk,dv,Hkv,page,e4m3,heads_first,layers", [
    (128, 128, 8, 16, False, False, 3), (128, 128, 2, 48, True, True, 5), (64, 64, 1, 256, False, True, 1), (192, 128, 3, 32, False, False, 2),
    (192, 128, 2, 16, True, False, 2), (64, 64, 2, 16, False, False, 130)])
def test_compaction(handle, dqk, dv, Hkv, page, e4m3, heads_first, layers):
    from paper_2609_21264_b200 import binding as b
    lens, counts = [26, 300, 40, 0, 7, 500, 90, 3], [26, 26, 26, 4, 0, 200, 64, 5]
    keep = [[0, 3, 4, 9, 25], [25], [], [], [], sorted(torch.randperm(200, generator=torch.Generator().manual_seed(1))[:50].tolist()), list(range(1, 64)), [2, 3, 4]]
    offs = offsets_of(counts)
    k, v, table, lens_t, ks, vs = pool(lens, page, Hkv, dqk, dv, e4m3, heads_first, 8, poison=False)
    pools, caches = layers_of(k, v, layers, b, ks, vs)
    raw = lambda t: t.view(torch.uint8).cpu()  # noqa: E731
    want = [(raw(x).clone(), raw(y).clone()) for x, y in pools]
    table_c = table.cpu()
    for x, y in want:
        for t in (x, y):
            old = t.clone()
            for i, (n, m) in enumerate(zip(lens, counts)):
                for to, frm in enumerate(keep[i]):
                    at, src = n - m + to, n - m + frm
                    if at >= 0:
                        t[int(table_c[i, at // page]), :, at % page] = old[int(table_c[i, src // page]), :, src % page]
    most = 70
    keep_t = torch.full((len(lens), most + 2), 2 ** 31 - 1, dtype=torch.int32)
    for i, x in enumerate(keep):
        keep_t[i, :len(x)] = torch.tensor(x, dtype=torch.int32)
    new = b.compact_paged(handle, caches, table, lens_t, keep_t.cuda()[:, :most], ints([len(x) for x in keep]), cu_seqlens=ints(offs))
    ok(handle)
    assert new.tolist() == [max(0, n - m + len(x)) for n, m, x in zip(lens, counts, keep)]
    for (x, y), (a, c) in zip(pools, want):
        assert torch.equal(raw(x), a) and torch.equal(raw(y), c)


def test_compaction_of_equal_trees_and_one_cache(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([30, 18], 16, 2, 128, 128, False, False, 9, poison=False)
    k0 = k.clone()
    new = torch.empty_like(lens_t)
    r = b.compact_paged(handle, b.PagedCache(k, v), table, lens_t, ints([[1, 4], [0, 2]]), ints([2, 1]), total=10, new_lens=new)
    ok(handle)
    assert r is new and new.tolist() == [27, 14]
    at = lambda t, s, j: t[int(table[s, j // 16]), :, j % 16]  # noqa: E731
    assert torch.equal(at(k, 0, 25), at(k0, 0, 26)) and torch.equal(at(k, 0, 26), at(k0, 0, 29)) and torch.equal(at(k, 1, 13), at(k0, 1, 13))


def test_compaction_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v, table, lens_t, _, _ = pool([30, 40], 16, 2, 128, 128, False, False, 10, poison=False)
    cache, k0, v0 = b.PagedCache(k, v), k.clone(), v.clone()
    cu = ints([0, 5, 10])
    for keep, count in (([3, 3, 4], 3), ([3, 2, 4], 3), ([-1, 2, 4], 3), ([0, 2, 5], 3), ([0, 2, 2 ** 31 - 1], 3), ([0, 1, 2], 4), ([0, 1, 2], -1),
                        ([0, 1, 2], 2 ** 31 - 1), ([-2 ** 31, 1, 2], 1)):
        new = b.compact_paged(handle, cache, table, lens_t, ints([keep, [0, 1, 2]]), ints([count, 2]), cu_seqlens=cu)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0906), (keep, count)
        assert new.tolist() == [30, 37] and torch.equal(k, k0) and torch.equal(v, v0)
    for off in ([-1, 5, 10], [6, 5, 10], [0, 300, 305]):
        b.compact_paged(handle, cache, table, lens_t, ints([[0, 1, 2]] * 2), ints([0, 2]), cu_seqlens=ints(off))
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0904) and torch.equal(k, k0)
    for page in (-1, k.shape[0]):
        bad = table.clone()
        bad[0, 1] = page                                  # positions 16 to 31
        b.compact_paged(handle, cache, bad, lens_t, ints([[1, 2, 4], [0, 1, 2]]), ints([3, 2]), cu_seqlens=cu)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0902) and torch.equal(k, k0)
    for n in (-1, 10 ** 6):
        b.compact_paged(handle, cache, table.clamp(0, k.shape[0] - 1), ints([n, 40]), ints([[0, 1, 2]] * 2), ints([0, 0]), cu_seqlens=cu)
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0901) and torch.equal(k, k0)
    keep, counts = ints([[0, 1, 2]] * 2), ints([1, 1])
    for kw in ({"keep": keep.long()}, {"keep": keep[:1]}, {"keep": keep[:, :0]}, {"keep_counts": counts[:1]}, {"keep_counts": counts.float()},
               {"new_lens": lens_t}, {"new_lens": counts[:1]}, {"cu_seqlens": cu[:2]}, {"keep": keep.t().contiguous().t()}):
        args = {"keep": keep, "keep_counts": counts, "cu_seqlens": cu, **kw}
        with pytest.raises(ValueError):
            b.compact_paged(handle, cache, table, lens_t, args.pop("keep"), args.pop("keep_counts"), **args)
    with pytest.raises(b.FaError):
        b.compact_paged(handle, cache, table, lens_t, keep, counts, total=5)
    other = b.PagedCache(*[torch.zeros(k.shape[0], 2, 32, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    with pytest.raises(b.FaError):
        b.compact_paged(handle, b.PagedCaches([cache, other]), table, lens_t, keep, counts, cu_seqlens=cu)
    with pytest.raises(ValueError):
        b.PagedCaches([])
    ok(handle)
    assert torch.equal(k, k0)


# ------------------------------------------------------------------------------------------------- page copies

@pytest.mark.parametrize("dqk,dv,Hkv,page,e4m3,order,layers", [
    (128, 128, 8, 16, False, "slots", 3), (128, 128, 2, 48, True, "heads", 5), (64, 64, 1, 256, False, "heads", 1), (192, 128, 3, 32, False, "slots", 2),
    (192, 128, 2, 16, True, "heads", 2), (64, 64, 2, 16, False, "slots", 130), (128, 128, 3, 32, False, "apart", 2), (64, 64, 2, 16, True, "apart", 2)])
@pytest.mark.parametrize("filled", [False, True], ids=["whole", "filled"])
def test_page_copies(handle, dqk, dv, Hkv, page, e4m3, order, layers, filled):
    from paper_2609_21264_b200 import binding as b
    pages, g = 23, torch.Generator().manual_seed(11)
    pools = []
    for _ in range(layers):
        pair = []
        for d in (dqk, dv):
            # "apart": rows of a head and slot with room between them
            shape = {"heads": (pages, Hkv, page, d), "slots": (pages, page, Hkv, d), "apart": (pages, Hkv, page, d + 16)}[order]
            x = torch.randint(0, 256, (*shape[:3], shape[3] * (1 if e4m3 else 2)), generator=g, dtype=torch.uint8).cuda()
            x = x if e4m3 else x.view(torch.bfloat16)
            pair.append(x.permute(0, 2, 1, 3) if order == "slots" else x[..., :d])
        pools.append(pair)
    raw = lambda t: t.view(torch.uint8) if e4m3 else t.view(torch.int16)  # noqa: E731
    src, dst = [3, -1, 22, 0, 5, 3, 7], [1, 2, 4, 9, -4, 6, 22 - 11]
    slots = [1, 5, page, page - 1, 3, 0, page + 9]
    want = []
    for pair in pools:
        for t in pair:
            w = raw(t).clone()
            for s, d, n in zip(src, dst, slots):
                if s >= 0 and d >= 0:
                    n = min(n, page) if filled else page
                    w[d, :, :n] = raw(t)[s, :, :n]
            want.append(w)
    caches = b.PagedCaches([b.PagedCache(*pair) for pair in pools])
    b.copy_pages(handle, caches, ints(src), ints(dst), slots=ints(slots) if filled else None)
    ok(handle)
    for t, w in zip([t for pair in pools for t in pair], want):
        assert torch.equal(raw(t), w)


def test_copies_into_a_pool_of_more_than_2_31_elements(handle):
    from paper_2609_21264_b200 import binding as b
    pages, Hkv, page, d = 17000, 8, 128, 128          # 2.2e9 elements a tensor
    k = torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    k[1], v[1] = torch.randn(Hkv, page, d, device="cuda"), torch.randn(Hkv, page, d, device="cuda")
    b.copy_pages(handle, b.PagedCache(k, v), ints([1]), ints([pages - 1]))
    ok(handle)
    assert torch.equal(k[-1], k[1]) and torch.equal(v[-1], v[1])
    table, lens = ints([[pages - 1]]), ints([100])
    b.compact_paged(handle, b.PagedCache(k, v), table, lens, ints([[4]]), ints([1]), total=7)
    ok(handle)
    assert torch.equal(k[-1, :, 93], k[1, :, 97]) and torch.equal(v[-1, :, 93], v[1, :, 97])


def test_copy_refusals(handle):
    from paper_2609_21264_b200 import binding as b
    k, v = (torch.randn(5, 2, 16, 64, device="cuda").bfloat16() for _ in range(2))
    cache, k0 = b.PagedCache(k, v), k.clone()
    for s, d in ((5, 1), (1, 5), (2 ** 31 - 1, 1), (1, 2 ** 31 - 1)):
        b.copy_pages(handle, cache, ints([s]), ints([d]))
        torch.cuda.synchronize()
        assert b.fa_last_status(handle) == (b.FA_ERR_INVALID_ARG, 0x0902) and torch.equal(k, k0)
    b.copy_pages(handle, cache, ints([]), ints([]))
    b.copy_pages(handle, cache, ints([1]), ints([2]), slots=ints([-3]))
    ok(handle)
    assert torch.equal(k, k0)
    one = ints([1])
    for kw in ({"src": one.long()}, {"dst": ints([1, 2])}, {"slots": ints([1, 2])}, {"dst": one.cpu()}, {"src": one.view(1, 1)}):
        args = {"src": one, "dst": ints([2]), **kw}
        with pytest.raises(ValueError):
            b.copy_pages(handle, cache, args.pop("src"), args.pop("dst"), **args)
    bad = b.FA_ERR_INVALID_ARG
    assert b.fa_copy_pages(None, cache.c, 1, one.data_ptr(), one.data_ptr(), None, 1) == bad
    assert b.fa_copy_pages(handle, cache.c, 0, one.data_ptr(), one.data_ptr(), None, 1) == bad
    assert b.fa_copy_pages(handle, cache.c, 1, None, one.data_ptr(), None, 1) == bad
    assert b.fa_copy_pages(handle, cache.c, 1, one.data_ptr(), one.data_ptr(), 2, 1) == bad
    assert b.fa_copy_pages(handle, cache.c, 1, one.data_ptr(), one.data_ptr(), None, -1) == bad
    ok(handle)


# ------------------------------------------------------------------------------------------------- a step of speculative decoding

@pytest.mark.parametrize("serial", [False, True], ids=["default", "serial"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_step_and_the_step_behind_it(serial, e4m3):
    """Layout, append at the tree's positions, attention, fork, compaction, then an ordinary token: its attention is that of a cache into
    which the accepted path was appended as a plain prompt.  The whole step captured into a graph and replayed."""
    from paper_2609_21264_b200 import binding as b
    h = b.fa_create(flags=b.FA_FLAG_SERIAL_KERNEL if serial else 0)
    try:
        g = torch.Generator().manual_seed(12)
        Hq, Hkv, d, page, ctx, n = 8, 2, 128, 16, [70, 5], 21
        lens = [c + n for c in ctx]
        k, v, table, lens_t, ks, vs = pool([x + 4 for x in lens], page, Hkv, d, d, e4m3, False, 13, poison=False, spare=8)
        lens_t = ints(lens)
        trees = [random_parents(n, g) for _ in ctx]
        parents = ints(sum(trees, []))
        kn, vn, q = (torch.randn(2 * n, H, d, generator=g).to(torch.bfloat16).cuda() for H in (Hkv, Hkv, Hq))
        # the longest path of each tree is accepted
        paths = []
        for t in trees:
            seen, depth = seen_by(t)
            paths.append(seen[depth.index(max(depth))].nonzero()[:, 0].tolist())
        most = max(len(p) for p in paths)
        keep, counts = ints([p + [0] * (most - len(p)) for p in paths]), ints([len(p) for p in paths])
        tab = rope_table(200, d)
        cache, rope = b.PagedCache(k, v, ks, vs), b.Rope(tab)
        start = k.clone(), v.clone()

        def step():
            mask, pos = b.tree_layout(h, parents, lens_t)
            qr = b.append_paged(h, kn, vn, cache, table, lens_t, q=q, rope=rope, positions=pos)
            o, lse = b.forward_paged_tree(h, qr, cache, table, lens_t, mask)
            return mask, pos, qr, o, lse, b.compact_paged(h, cache, table, lens_t, keep, counts, total=2 * n)

        mask, pos, qr, o, lse, new = step()
        ok(h)
        assert new.tolist() == [c + len(p) for c, p in zip(ctx, paths)]
        seens = [seen_by(t)[0] for t in trees]
        assert torch.equal(mask.cpu(), torch.cat([pack(s, 1) for s in seens]))
        # (attention was over the cache before the compaction: made again)
        after = k.clone(), v.clone()
        k.copy_(start[0]), v.copy_(start[1])
        b.append_paged(h, kn, vn, cache, table, lens_t, rope=rope, positions=pos)
        torch.cuda.synchronize()
        assert_attention(o, lse, *tree_reference(qr, k, v, ks, vs, table, lens, [0, n, 2 * n], seens, d ** -0.5))
        # the accepted path as a plain prompt into a cache of its own
        k.copy_(start[0]), v.copy_(start[1])
        rows = torch.cat([torch.tensor(p) + i * n for i, p in enumerate(paths)]).cuda()
        b.append_paged(h, kn[rows], vn[rows], cache, table, new, cu_seqlens=ints(offsets_of([len(p) for p in paths])), rope=rope)
        plain = k.clone(), v.clone()
        for i, m in enumerate(new.tolist()):
            for at in range(m):
                p, s = int(table[i, at // page]), at % page
                assert torch.equal(after[0][p, :, s].view(torch.uint8), plain[0][p, :, s].view(torch.uint8))
                assert torch.equal(after[1][p, :, s].view(torch.uint8), plain[1][p, :, s].view(torch.uint8))
        one = b.forward_paged(h, q[:2], cache, table, new)
        k.copy_(after[0]), v.copy_(after[1])
        two = b.forward_paged(h, q[:2], cache, table, new)
        ok(h)
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
        # a fork of the second sequence: its pages but the last shared, that one copied
        m = new.tolist()[1]
        last = (m - 1) // page
        free = [x for x in range(k.shape[0]) if x not in table[0, :-(-lens[0] // page) + 1].tolist() + table[1, :-(-lens[1] // page) + 1].tolist()][0]
        b.copy_pages(h, cache, table[1, last:last + 1].clone(), ints([free]), slots=ints([m - last * page]))
        forked = table.clone()
        forked[1, last] = free
        three = b.forward_paged(h, q[:2], cache, forked, new)
        ok(h)
        assert torch.equal(three[0], two[0])
        # the step as a graph
        k.copy_(start[0]), v.copy_(start[1])
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = step()
        for _ in range(2):
            k.copy_(start[0]), v.copy_(start[1])
            graph.replay()
            ok(h)
            for x, y in zip(captured, (mask, pos, qr, o, lse, new)):
                assert torch.equal(x, y)
            assert torch.equal(k.view(torch.uint8), after[0].view(torch.uint8)) and torch.equal(v.view(torch.uint8), after[1].view(torch.uint8))
    finally:
        b.fa_destroy(h)


def test_new_lengths_are_a_tensor_of_their_own(handle):
    """The CTAs of a sequence read lengths, offsets and kept numbers each in its own time: none of them may be written meanwhile."""
    from paper_2609_21264_b200 import binding as b
    k = torch.randn(4, 2, 16, 64, device="cuda").to(torch.bfloat16)
    v = torch.randn(4, 2, 16, 64, device="cuda").to(torch.bfloat16)
    k0, v0 = k.clone(), v.clone()
    table, lens, keep, counts, cu = ints([[0, 1], [2, 3]]), ints([20, 30]), ints([[1], [2]]), ints([1, 1]), ints([0, 5, 10])
    for new in (counts, cu[:2], keep.view(-1)):
        with pytest.raises(b.FaError) as e:
            b.compact_paged(handle, b.PagedCache(k, v), table, lens, keep, counts, cu_seqlens=cu, new_lens=new)
        assert e.value.status == b.FA_ERR_INVALID_ARG
    torch.cuda.synchronize()
    ok(handle)
    assert torch.equal(k, k0) and torch.equal(v, v0) and counts.tolist() == [1, 1] and cu.tolist() == [0, 5, 10] and keep.tolist() == [[1], [2]]
