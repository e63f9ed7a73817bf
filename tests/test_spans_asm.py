"""The gfx950 code the compiler emits for rotated appends, attention through a window and over
shared prefixes (CPU: hipcc cross-compiles without a GPU): no scratch memory, no vector
registers spilled, and the workgroups per CU that their launch bounds ask for."""

import re

import pytest

from tests.test_kernel_asm import kernel_entries
from tests.test_pages_asm import check_all, compiled, number


def check_occupancy(entries):
    """Workgroups of 8 waves: two a CU at 64 dims, one at 128; of 4 waves: as few_per_cu says."""
    for n, e in entries.items():
        vgprs, lds = -(-number(e, "vgpr_count") // 8) * 8, number(e, "group_segment_fixed_size")
        form, few = re.search(r"FormILi(64|128)E", n), re.search(r"fewILi(64|128)ELi([12])E", n)
        if form:
            groups, most = (2 if form.group(1) == "64" else 1), 256
        else:
            d, c = map(int, few.groups())
            groups, most = (4 if d == 64 else 3) - (c - 1), 512
        assert groups * vgprs <= most, (n, vgprs)
        assert groups * lds <= 160 * 1024, (n, lds)


@pytest.mark.parametrize("name,many,few,rest", [
    ("flowkv_window", 16, 8, 12), ("flowkv_prefix", 20, 16, 20),
])
def test_attention_kernels(tmp_path_factory, name, many, few, rest):
    asm = compiled(name, tmp_path_factory)
    every = kernel_entries(asm, "_attn")
    joins = {n: e for n, e in every.items() if re.search(r"_attn_(join|merge)I", n)}
    fews = {n: e for n, e in every.items() if "_attn_fewI" in n}
    manys = {n: e for n, e in every.items() if re.search(r"_attnI", n)}
    assert (len(manys), len(fews), len(joins)) == (many, few, rest)
    assert len(every) == many + few + rest
    check_all(every)
    check_occupancy({**manys, **fews})


def body(asm, name):
    return re.search(rf"^{re.escape(name)}:.*?^\.Lfunc_end", asm, re.S | re.M).group(0)


def test_few_rows_read_k_and_v_past_the_caches(tmp_path_factory):
    """(A branch round the two kinds of load once cost the hint, and 8% of a decode step.)"""
    for name, kernel in (("flowkv_chunk", "chunk_attn_few"), ("flowkv_window", "window_attn_few"),
                         ("flowkv_prefix", "alone_attn_few")):
        asm = compiled(name, tmp_path_factory)
        for n in kernel_entries(asm, kernel):
            d = int(re.search(r"fewILi(64|128)E", n).group(1))
            past = len(re.findall(r"^\s+global_load_dword\S*\s.*\bnt\b", body(asm, n), re.M))
            assert past >= 2 * (d // 16 + 4), (n, past)


def test_rotated_append_kernels(tmp_path_factory):
    entries = kernel_entries(compiled("flowkv_rotate", tmp_path_factory), "kv_rotate")
    assert len(entries) == 18
    check_all(entries)
    for n, e in entries.items():        # 32 waves a CU
        assert number(e, "vgpr_count") <= 64, n
