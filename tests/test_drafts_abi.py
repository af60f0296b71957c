"""Entry points on drafted tokens without a GPU: structures and constants against the header, refusals that come before any launch."""
import ctypes
import os
import re

import pytest
import torch

from paper_2609_21264_b200 import binding as b

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fa.h")).read()
TYPES = {"uint32_t": ctypes.c_uint32, "int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "const int32_t*": ctypes.c_void_p,
         "const uint32_t*": ctypes.c_void_p, "const uint8_t*": ctypes.c_void_p}


@pytest.mark.parametrize("name", ["fa_positions", "fa_tree"])
def test_structure_matches_the_header(name):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), HEADER, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [(n.strip(), TYPES[t]) for t, names in re.findall(r"(const \w+\*|uint32_t|int32_t|int64_t)\s+([^;]+);", body) for n in names.split(",")]
    assert list(getattr(b, name)._fields_) == fields and len(fields) == 5


def test_constants_match_the_header():
    for name in ("FA_MAX_AXES", "FA_TREE_MAX_TOKENS"):
        assert getattr(b, name) == int(re.search(r"#define\s+%s\s+(\d+)" % name, HEADER).group(1))


def test_a_null_handle_is_refused():
    assert b.fa_tree_layout(None, None, None, 0, 0, None, 1, None, 0, None) == b.FA_ERR_INVALID_ARG
    assert b.fa_append_paged_at(None, None, None, None, 0, None, None, None, None, 0, None, None, None, None, None, None) == b.FA_ERR_INVALID_ARG
    assert b.fa_forward_paged_tree(None, None, None, None, 0, None, None, None, 1, 0.0, None, None) == b.FA_ERR_INVALID_ARG
    assert b.fa_compact_paged(None, None, 1, None, None, 0, None, 1, None, 1, None) == b.FA_ERR_INVALID_ARG
    assert b.fa_copy_pages(None, None, 1, None, None, None, 0) == b.FA_ERR_INVALID_ARG


def test_host_tensors_and_wrong_types_are_refused():
    x = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        b.tree_layout(0, x, x)
    with pytest.raises(ValueError):
        b.PagedCaches([])
    with pytest.raises(ValueError):
        b._check_mask(x, 4, 1, x.device)
    for mask, words in ((x[:, None].float(), 1), (x[:, None], 2), (x[:3, None], 1), (x[:2, None].expand(2, 2), 2), (x.view(2, 2).t(), 2)):
        with pytest.raises(ValueError):
            b._check_mask(mask, mask.shape[0] if mask.shape[0] != 3 else 4, words, x.device)
    b._check_mask(x.view(2, 2), 2, 2, x.device)
    assert b._offsets(None, 3, x.device) is None and b._offsets(x, 3, x.device) == x.data_ptr()
    for bad in (x[:3], x.long(), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            b._offsets(bad, 3, x.device)
    assert b._most_tokens(0, None, 12, 4) == 3 and b._most_tokens(7, None, 12, 4) == 7 and b._most_tokens(0, None, 0, 0) == 1
    for args in ((0, x, 12, 4), (-1, None, 12, 4)):
        with pytest.raises(ValueError):
            b._most_tokens(*args)
