"""The gfx950 code the compiler emits for the kernels that write into a pool's pages and
attend over them (CPU: hipcc cross-compiles without a GPU): no scratch memory, no vector
registers spilled, and the waves per SIMD that their launch bounds ask for."""

import os
import re
import subprocess

import pytest

from tests.test_kernel_asm import ROOT, hipcc, kernel_entries

CSRC_DIR = os.path.join(ROOT, "paper_2504_03775_amd", "csrc")


def compiled(name, tmp_path_factory):
    cc = hipcc()
    if cc is None:
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("asm") / (name + ".s")
    from paper_2504_03775_amd.build import HIP_FLAGS, INCLUDE, CSRC
    flags = [f for f in HIP_FLAGS if f not in ("-fPIC", "-Wall")]
    subprocess.run([cc, *flags, "--cuda-device-only", "-S", "-I", INCLUDE, "-I", CSRC,
                    os.path.join(CSRC_DIR, name + ".hip"), "-o", str(out)],
                   check=True, capture_output=True, timeout=900)
    return out.read_text()


def number(entry, field):
    return int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1))


def check_all(entries):
    for n, e in entries.items():
        assert number(e, "private_segment_fixed_size") == 0, n
        assert number(e, "vgpr_spill_count") == 0, n
        assert number(e, "kernarg_segment_size") <= 4096, n


def test_page_kernels(tmp_path_factory):
    asm = compiled("flowkv_pages", tmp_path_factory)
    append = kernel_entries(asm, "kv_append")
    copies = {**kernel_entries(asm, "kv_block_copy"), **kernel_entries(asm, "kv_block_stream")}
    assert len(append) == 2 and len(copies) == 8
    check_all({**append, **copies})
    for n, e in copies.items():     # 32 waves a CU
        assert number(e, "vgpr_count") <= 64, n


def test_chunk_attention_kernels(tmp_path_factory):
    asm = compiled("flowkv_chunk", tmp_path_factory)
    forms = kernel_entries(asm, r"10chunk_attnIN")
    few = kernel_entries(asm, "chunk_attn_few")
    rest = {**kernel_entries(asm, "chunk_attn_merge"), **kernel_entries(asm, "chunk_attn_join")}
    assert len(forms) == 8 and len(few) == 4 and len(rest) == 6
    check_all({**forms, **few, **rest})
    for n, e in forms.items():      # workgroups of 8 waves: two a CU at 64 dims, one at 128
        groups = 2 if "FormILi64E" in n else 1
        assert groups * (-(-number(e, "vgpr_count") // 8) * 8) <= 256, n
        assert groups * number(e, "group_segment_fixed_size") <= 160 * 1024, n
    for n, e in few.items():        # workgroups of 4 waves
        d, c = map(int, re.search(r"chunk_attn_fewILi(64|128)ELi([12])E", n).groups())
        groups = (4 if d == 64 else 3) - (c - 1)
        assert groups * (-(-number(e, "vgpr_count") // 8) * 8) <= 512, n
        assert groups * number(e, "group_segment_fixed_size") <= 160 * 1024, n
