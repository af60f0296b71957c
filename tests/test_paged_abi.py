"""The structures of the paged and differential entry points: the binding's against the header's, field by field."""
import ctypes
import os
import re

import pytest

from paper_2609_21264_b200 import binding

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fa.h")).read()
TYPES = {"uint32_t": ctypes.c_uint32, "int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "void*": ctypes.c_void_p,
         "const float*": ctypes.c_void_p, "const int32_t*": ctypes.c_void_p}


@pytest.mark.parametrize("name", ["fa_paged_cache", "fa_paged_seqs", "fa_rope", "fa_diff", "fa_paged_plan_info", "fa_paged_piece"])
def test_structure_matches_the_header(name):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), HEADER, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = []
    for ctype, names in re.findall(r"(const float\*|const int32_t\*|void\*|uint32_t|int32_t|int64_t|float)\s+([^;]+);", body):
        for n in names.split(","):
            n = n.strip()
            array = re.match(r"(\w+)\[(\d+)\]", n)
            fields.append((array.group(1), TYPES[ctype] * int(array.group(2))) if array else (n, TYPES[ctype]))
    mine = [(n.rstrip("_"), t) for n, t in getattr(binding, name)._fields_]
    assert mine == fields


def test_constants_match_the_header():
    for name in ("FA_CACHE_BF16", "FA_CACHE_E4M3", "FA_PAGED_MAX_SQ"):
        assert getattr(binding, name) == int(re.search(r"#define\s+%s\s+(\d+)" % name, HEADER).group(1))


def test_a_null_handle_is_refused_without_a_gpu():
    assert binding.fa_append_paged(None, None, None, None, 0, None, None, None, None, 0, None, None, None, None, None) == binding.FA_ERR_INVALID_ARG
    assert binding.fa_forward_paged(None, None, None, None, None, None, 1, 1, 0.0, None, None) == binding.FA_ERR_INVALID_ARG
    assert binding.fa_forward_paged_diff(None, None, None, None, None, 1, 1, 0.0, None, None, None) == binding.FA_ERR_INVALID_ARG
    assert binding.fa_forward_diff(None, None, None, None, None, 1, 1, 1, 1, 1, 128, 128, True, 0.0, None, None, None, None,
                                   None) == binding.FA_ERR_INVALID_ARG
    assert binding.fa_device(None) == -1


def test_host_tensors_are_refused():
    import torch
    k = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.PagedCache(k, k)
    with pytest.raises(ValueError):
        binding.PagedCache(k, k.float())
    with pytest.raises(ValueError):
        binding.Rope(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        binding.forward_diff(0, k, k, k, torch.zeros(1), causal=True)


@pytest.mark.parametrize("table_rows", ["shared", "overlapping", "columns"])
def test_block_tables_whose_rows_do_not_lie_apart_are_refused(table_rows):
    """(A row stride below the row's length would be read as the length: rows of another place in memory.)"""
    import types

    import torch
    t = torch.zeros(64, dtype=torch.int32)
    table = {"shared": t[:8].expand(4, 8), "overlapping": t.as_strided((4, 8), (4, 1)), "columns": t[:32].view(8, 4).t()}[table_rows]
    cache = types.SimpleNamespace(device=t.device)
    with pytest.raises(ValueError, match="block_table"):
        binding._seqs(None, cache, table, torch.ones(4, dtype=torch.int32))


def test_plans_of_more_heads_than_a_call_may_have_are_refused():
    with pytest.raises(binding.FaError) as e:
        binding.fa_plan_paged(148, [100], 1 << 28, 1, 16, 128, 128)
    assert e.value.status == binding.FA_ERR_UNSUPPORTED
