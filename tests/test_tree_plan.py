"""The list of work of attention of drafted tokens, made on the host by the kernel's own code: every tile of every row tile once, no slot
twice, pieces in the order and the slots that the joining kernel expects."""
import random

import pytest

from paper_2609_21264_b200 import binding as b


def check(num_sms, lens, counts, Hq, Hkv, dqk, dv, **kw):
    info, pieces = b.fa_plan_paged_tree(num_sms, lens, counts, Hq, Hkv, dqk, dv, **kw)
    group, most = Hq // Hkv, kw.get("max_tokens") or max(1, max(counts))
    if group * most <= 32:
        return check_few(info, pieces, lens, counts, Hkv, 16 if group * most <= 16 else 32, num_sms)
    heads = min(group, 128)
    tokens, chunks, two = min(128 // heads, most), -(-group // heads), dqk != 192 and not kw.get("e4m3")
    assert info["rows_per_block"] == heads * tokens and info["pieces"] == len(pieces) and info["ctas"] <= num_sms
    seen, slots, blocks = {}, set(), {}
    for p in pieces:
        n, nt = counts[p["sequence"]], -(-lens[p["sequence"]] // 128)
        row_tiles = -(-n // tokens) * chunks
        mine = [p["row_block"]] + ([p["row_block"] + 1] if two and p["row_block"] + 1 < row_tiles else [])
        assert not two or p["row_block"] % 2 == 0
        for r in mine:
            for t in range(p["first_tile"], p["end_tile"]) if nt else [-1]:
                key = (p["sequence"], p["kv_head"], r, t)
                assert key not in seen
                seen[key] = True
        whole = p["slot"] < 0
        assert whole == (p["first_tile"] == 0 and p["end_tile"] == nt) and (p["pieces"] == 1) == whole
        if not whole:
            assert p["slot"] == 2 * p["cta"] + (1 if p["first_tile"] == 0 else 0) and p["slot"] not in slots
            slots.add(p["slot"])
            blocks.setdefault((p["sequence"], p["kv_head"], p["row_block"]), []).append(p)
    for group_pieces in blocks.values():
        first = group_pieces[0]
        assert [p["cta"] for p in group_pieces] == list(range(first["cta"], first["cta"] + first["pieces"])) and first["first_tile"] == 0
        assert all(p["pieces"] == len(group_pieces) and p["first_cta"] == first["cta"] for p in group_pieces)
        assert [p["first_tile"] for p in group_pieces[1:]] == [p["end_tile"] for p in group_pieces[:-1]]
    assert len({p["cta"] for group_pieces in blocks.values() for p in group_pieces[:1]}) == len(blocks)      # one join a CTA at most
    want = sum(Hkv * -(-n // tokens) * chunks * max(1, -(-x // 128)) for x, n in zip(lens, counts))
    assert len(seen) == want
    return info, pieces


def check_few(info, pieces, lens, counts, Hkv, rows, num_sms):
    """The streaming kernel's list: one block of rows, an empty tile for what has no keys or no drafts, two slots a CTA."""
    assert (info["rows_per_block"], info["row_blocks"]) == (rows, 1) and info["pieces"] == len(pieces) and info["ctas"] <= num_sms
    tiles = [max(1, -(-x // 128)) if n else 1 for x, n in zip(lens, counts)]
    seen, slots, blocks = set(), set(), {}
    for p in pieces:
        for t in range(p["first_tile"], p["end_tile"]):
            assert (p["sequence"], p["kv_head"], t) not in seen
            seen.add((p["sequence"], p["kv_head"], t))
        whole = p["slot"] < 0
        assert p["row_block"] == 0 and whole == (p["end_tile"] - p["first_tile"] == tiles[p["sequence"]]) and (p["pieces"] == 1) == whole
        if not whole:
            assert p["slot"] // 2 == p["cta"] and p["slot"] not in slots
            slots.add(p["slot"])
            blocks.setdefault((p["sequence"], p["kv_head"]), []).append(p)
    for group_pieces in blocks.values():
        assert [p["cta"] for p in group_pieces] == list(range(group_pieces[0]["first_cta"], group_pieces[0]["first_cta"] + group_pieces[0]["pieces"]))
        assert [p["first_tile"] for p in group_pieces[1:]] == [p["end_tile"] for p in group_pieces[:-1]] and group_pieces[0]["first_tile"] == 0
    assert len(seen) == Hkv * sum(tiles)
    return info, pieces


@pytest.mark.parametrize("seed", range(40))
def test_random_batches(seed):
    rng = random.Random(seed)
    B = rng.choice((1, 2, 5, 17, 60))
    most = rng.randint(1, 256)
    lens = [0 if rng.random() < 0.15 else rng.randint(1, rng.choice((500, 6000))) for _ in range(B)]
    counts = [0 if rng.random() < 0.2 else rng.randint(1, most) for _ in range(B)]
    counts[0] = counts[0] or 1
    if seed % 3 == 0:
        lens, counts = [max(1, lens[0])] * B, [counts[0]] * B
    Hkv = rng.randint(1, 6)
    dqk, dv = rng.choice(((64, 64), (128, 128), (192, 128)))
    check(rng.choice((1, 7, 148)), lens, counts, Hkv * rng.choice((1, 2, 4, 7, 8, 40, 130)), Hkv, dqk, dv, max_tokens=most, e4m3=rng.random() < 0.4)


@pytest.mark.parametrize("seed", range(40))
def test_random_batches_of_few_rows(seed):
    rng = random.Random(100 + seed)
    group = rng.choice((1, 2, 3, 4, 7, 8, 16, 32))
    most = rng.randint(1, 32 // group)
    B, Hkv = rng.choice((1, 2, 5, 17, 60)), rng.randint(1, 6)
    lens = [0 if rng.random() < 0.15 else rng.randint(1, rng.choice((500, 6000))) for _ in range(B)]
    counts = [0 if rng.random() < 0.2 else rng.randint(1, most) for _ in range(B)]
    counts[0] = counts[0] or 1
    dqk, dv = rng.choice(((64, 64), (128, 128), (192, 128)))
    check(rng.choice((1, 7, 148)), lens, counts, Hkv * group, Hkv, dqk, dv, max_tokens=most, e4m3=rng.random() < 0.4)


def test_small_batches_are_split_where_that_pays():
    whole = lambda pieces: all(p["slot"] < 0 for p in pieces)  # noqa: E731
    # 128 blocks of eight tiles on 148 SMs: a wave of whole blocks; eight blocks of eight tiles: four pieces each
    check(148, [1003] * 16, [8] * 16, 32, 8, 128, 128)
    assert whole(check(148, [1003] * 16, [9] * 16, 32, 8, 128, 128)[1])
    info, pieces = check(148, [1003], [26], 32, 8, 128, 128)
    assert {p["pieces"] for p in pieces} == {4} and len({p["cta"] for p in pieces}) == len(pieces) == 32
    assert whole(check(148, [100], [26], 32, 8, 128, 128)[1])


def test_an_equal_share_for_every_cta():
    info, pieces = check(148, [131072, 70] + [5000] * 20, [64] * 22, 32, 8, 128, 128)
    tiles = [0] * 148
    for p in pieces:
        tiles[p["cta"]] += p["end_tile"] - p["first_tile"]
    assert max(tiles) * 2 <= info["units_per_cta"] + 2 and info["units_per_cta"] * 148 >= info["units"] > info["units_per_cta"] * 147


def test_refused_batches():
    for args, kw in ((([100], [257], 8, 2, 128, 128), {}), (([100], [4], 8, 2, 96, 96), {}), (([100], [4], 65538, 2, 128, 128), {}),
                     (([2 ** 31 - 1000] * 200, [256] * 200, 65528, 8, 128, 128), {"page_size": 65536}), (([100], [4], 8, 2, 128, 128), {"scratch_bytes": 1000}),
                     (([100], [4], 8, 2, 128, 128), {"page_size": 24})):
        with pytest.raises(b.FaError) as e:
            b.fa_plan_paged_tree(148, *args, **kw)
        assert e.value.status == b.FA_ERR_UNSUPPORTED
    for args in (([100], [4], 7, 2, 128, 128), ([100], [0], 8, 2, 128, 128)):
        with pytest.raises(b.FaError) as e:
            b.fa_plan_paged_tree(148, *args)
        assert e.value.status == b.FA_ERR_INVALID_ARG
