"""The documented limit of the paged calls' list of work, at either side of it."""
import pytest

from paper_2609_21264_b200 import binding


def refused(B, Hq, Hkv, Sq, pages, page=16, **kw):
    try:
        binding.fa_plan_paged(148, [1] * B, Hq, Hkv, Sq, kw.pop("dqk", 128), 128, page_size=page, max_pages=pages, **kw)
    except binding.FaError as e:
        assert e.status == binding.FA_ERR_UNSUPPORTED
        return True
    return False


@pytest.mark.parametrize("Hq,Hkv,Sq,blocks,kw", [
    (8, 8, 1, 1, {}),
    (64, 4, 1, 1, {}),                             # 16 rows
    (16, 4, 5, 1, {}),                             # 20 rows: a block of 32
    (64, 4, 8, 2, {}),                             # 128 rows: blocks of 64
    (64, 4, 8, 4, {"e4m3": True}),                 # blocks of 32
    (64, 4, 8, 4, {"dqk": 192}),
    (64, 4, 8, 8, {"diff": True}),                 # blocks of 16
], ids=str)
def test_the_product_of_sequences_heads_blocks_and_tiles(Hq, Hkv, Sq, blocks, kw):
    """B * Hkv * blocks * (tiles + 3) <= 2^30."""
    B = 64
    tiles = (1 << 30) // (B * Hkv * blocks) - 3
    assert tiles * 128 < 2 ** 31 - 256
    assert not refused(B, Hq, Hkv, Sq, tiles * 8, **kw)
    assert refused(B, Hq, Hkv, Sq, tiles * 8 + 1, **kw)
    # half as many sequences may be twice as long
    assert not refused(B // 2, Hq, Hkv, Sq, min(2 * tiles * 8, (2 ** 31 - 256) // 16), **kw)
