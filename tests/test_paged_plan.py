"""The work list of the paged kernel on the CPU: its own walk, made by the library's host side with the device's functions.

Every tile of every sequence, head and row block is taken once; partial results go to slots inside the scratch, no two to the
same one; the pieces of a row block agree on their number and on the counter they meet at."""
import random
from collections import defaultdict

import pytest

from paper_2609_21264_b200 import binding as b


def check(num_sms, lens, Hq, Hkv, Sq, dqk, dv, e4m3=False, diff=False, page=16, scratch=0, max_pages=0):
    info, pieces = b.fa_plan_paged(num_sms, lens, Hq, Hkv, Sq, dqk, dv, page_size=page, e4m3=e4m3, diff=diff, scratch_bytes=scratch,
                                   max_pages=max_pages)
    rows = Hq // Hkv * Sq
    assert info["rows_per_block"] in (16, 32, 64) and info["row_blocks"] == -(-rows // info["rows_per_block"])
    assert 1 <= info["ctas"] <= num_sms and len(pieces) == info["pieces"]
    most = (max_pages or max(1, -(-max(lens) // page))) * page
    tiles = [max(1, -(-max(0, min(n, most)) // 128)) for n in lens]
    blocks = len(lens) * Hkv * info["row_blocks"]
    unsplit = max(tiles) <= 6 and blocks <= info["ctas"]
    aligned = unsplit or (len(lens) == 1 and 2 * blocks <= info["ctas"])        # a block's tiles count as a multiple of the share
    share = info["units_per_cta"] if aligned else 1
    assert info["units"] == sum(-(-n // share) * share + info["part_cost"] for n in tiles) * Hkv * info["row_blocks"]
    if unsplit:
        assert all(x["slot"] < 0 for x in pieces)               # a CTA for every row block, nothing split
    if aligned:
        assert info["part_cost"] == 0 and len({x["cta"] for x in pieces}) == len(pieces)      # a CTA has one part
    assert info["units_per_cta"] * info["ctas"] >= info["units"]
    states = info["rows_per_block"] * (2 if diff else 1)
    slots = (scratch or 32 << 20) // (states * (dv + 2) * 4)
    assert 2 * info["ctas"] <= slots
    taken, groups, used = defaultdict(list), defaultdict(list), set()
    load = defaultdict(int)
    for x in pieces:
        key = (x["sequence"], x["kv_head"], x["row_block"])
        assert 0 <= x["cta"] < info["ctas"] and 0 <= x["sequence"] < len(lens) and 0 <= x["kv_head"] < Hkv
        assert 0 <= x["row_block"] < info["row_blocks"] and x["first_tile"] < x["end_tile"]
        taken[key] += range(x["first_tile"], x["end_tile"])
        load[x["cta"]] += x["end_tile"] - x["first_tile"]
        if x["slot"] < 0:
            assert (x["first_tile"], x["end_tile"]) == (0, tiles[x["sequence"]])
        else:
            assert x["slot"] not in used and x["slot"] // 2 == x["cta"] and x["slot"] < 2 * info["ctas"]
            used.add(x["slot"])
            groups[key].append(x)
    assert len(taken) == len(lens) * Hkv * info["row_blocks"]
    for (s, _, _), t in taken.items():
        assert t == list(range(tiles[s]))
    assert max(load.values()) <= info["units_per_cta"]
    firsts = set()
    for parts in groups.values():
        assert len(parts) == parts[0]["pieces"] > 1
        assert [p["cta"] for p in parts] == list(range(parts[0]["first_cta"], parts[0]["first_cta"] + len(parts)))
        assert {(p["pieces"], p["first_cta"]) for p in parts} == {(parts[0]["pieces"], parts[0]["first_cta"])}
        assert parts[0]["first_cta"] not in firsts          # one counter per row block that several CTAs share
        firsts.add(parts[0]["first_cta"])
    return info, pieces


def test_shapes_of_the_gpu_tests():
    edge = [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 700]
    for dqk, dv in ((64, 64), (128, 128), (192, 128)):
        for Hq, Hkv in ((8, 2), (3, 3), (14, 2), (16, 1)):
            for Sq in (1, 3, 16):
                for e4m3 in (False, True):
                    check(148, edge, Hq, Hkv, Sq, dqk, dv, e4m3)
    check(148, [(i * 53) % 260 for i in range(333)], 2, 2, 1, 64, 64)
    check(148, [3000] + [3] * 40 + [9000], 8, 2, 1, 128, 128)
    check(148, [20000], 8, 1, 1, 128, 128)


def test_random_batches():
    rng = random.Random(17)
    for _ in range(300):
        Hkv = rng.choice((1, 2, 3, 8))
        dqk, dv = rng.choice(((64, 64), (128, 128), (192, 128)))
        diff = dqk == 128 and rng.random() < 0.3
        lens = [rng.choice((0, 1, rng.randint(0, 300), rng.randint(0, 20000))) for _ in range(rng.randint(1, 60))]
        check(rng.choice((1, 2, 148)), lens, Hkv * rng.choice((1, 2, 5, 8)), Hkv, rng.choice((1, 2, 16)), dqk, dv, rng.random() < 0.5, diff,
              rng.choice((16, 48, 128)))


def test_lengths_out_of_range_are_clamped_as_on_the_device():
    check(148, [-5, 2 ** 31 - 1, 77], 8, 2, 1, 128, 128, max_pages=30)


def test_small_scratch_means_fewer_ctas_and_none_is_refused():
    info, _ = check(148, [100000], 8, 1, 1, 128, 128, scratch=10 * 16 * 130 * 4)
    assert info["ctas"] == 5
    with pytest.raises(b.FaError) as e:
        b.fa_plan_paged(148, [1000], 8, 1, 1, 128, 128, scratch_bytes=1000)
    assert e.value.status == b.FA_ERR_UNSUPPORTED


def test_refusals():
    for kw, want in (({"Hq": 7}, b.FA_ERR_INVALID_ARG), ({"Sq": 17}, b.FA_ERR_UNSUPPORTED), ({"dqk": 96}, b.FA_ERR_UNSUPPORTED),
                     ({"page_size": 24}, b.FA_ERR_UNSUPPORTED), ({"diff": True, "dqk": 64, "dv": 64}, b.FA_ERR_UNSUPPORTED)):
        args = {"num_sms": 148, "seq_lens": [5], "Hq": 8, "Hkv": 2, "Sq": 1, "dqk": 128, "dv": 128, **kw}
        with pytest.raises(b.FaError) as e:
            b.fa_plan_paged(args.pop("num_sms"), args.pop("seq_lens"), args.pop("Hq"), args.pop("Hkv"), args.pop("Sq"), args.pop("dqk"),
                            args.pop("dv"), **args)
        assert e.value.status == want, kw


def test_lists_that_32_bits_cannot_count_are_refused():
    """(74 blocks of one sequence count up to twice their tiles.)"""
    with pytest.raises(b.FaError) as e:
        b.fa_plan_paged(148, [2 ** 31 - 256], 74, 74, 1, 64, 64, page_size=128)
    assert e.value.status == b.FA_ERR_UNSUPPORTED
    info, pieces = b.fa_plan_paged(148, [2 ** 31 - 256], 63, 63, 1, 64, 64, page_size=128)
    assert 63 * (2 ** 24 - 2) <= info["units"] < 2 ** 31 and sum(x["end_tile"] - x["first_tile"] for x in pieces) == 63 * (2 ** 24 - 2)
