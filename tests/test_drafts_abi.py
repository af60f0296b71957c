"""Entry points on drafted tokens without a GPU: structures and constants against the header, refusals that come before any launch."""
import ctypes
import os
import re
import types

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
    with pytest.raises(TypeError):
        b.tree_layout(0, [1, 2], x)
    with pytest.raises(ValueError):
        b.tree_layout(0, None, x)
    with pytest.raises(ValueError):
        b.PagedCaches([])
    cache = types.SimpleNamespace(address=0, index=0, count=1, dqk=64, dv=64, Hkv=1)
    q = torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: b.forward_paged_tree(0, q, cache, x.view(2, 2), x, None), lambda: b.compact_paged(0, cache, x.view(2, 2), x, x.view(2, 2), x),
                 lambda: b.copy_pages(0, cache, x, x), lambda: b.append_paged(0, q, q, cache, x.view(2, 2), x, positions=x)):
        with pytest.raises(ValueError):
            call()
    assert b._offsets(None, 3, x.device) is None and b._offsets(x, 3, x.device) == x.data_ptr()
    for bad in (x[:3], x.long(), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            b._offsets(bad, 3, x.device)


def test_the_calls_module_asks_for_its_arguments():
    calls = b._native()
    for f in (calls.tree_layout, calls.append_at, calls.paged_tree, calls.compact, calls.copy_pages):
        with pytest.raises(ValueError):
            f()
        with pytest.raises((TypeError, ValueError)):
            f(*["no"] * 18)
