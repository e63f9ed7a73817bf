"""Block copies' checks of their lists (CPU: every call returns before it touches a device)."""

import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2504_03775_amd import flowkv as fk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def check(blocks, src, dst):
    """The status of a copy of no token of each block, as the lists alone decide it."""
    p = fk.flowkv_pool(fk.LAYOUT_BLOCK_MAJOR, 2, blocks, 0, 16, (ctypes.c_void_p * 1)(1 << 20))
    s, d, k = (np.asarray(x, np.int32) for x in (src, dst, [0] * len(src)))
    return fk.lib().flowkv_copy_blocks(ctypes.byref(p), s.ctypes.data, d.ctypes.data, k.ctypes.data,
                                       len(s), 16, None)


@pytest.mark.parametrize("blocks", [40, 5000, 2**31 - 1])
def test_pairs_as_a_plain_form_says(blocks):
    g = np.random.default_rng(blocks)
    seen = {}
    for _ in range(3000):
        n = int(g.integers(1, 30))
        span = blocks if g.integers(2) else min(blocks, 64)
        src, dst = g.integers(0, span, n), g.permutation(min(span, 1 << 16))[:n] + (span >> 17)
        if len(dst) < n:
            continue
        what = g.integers(6)
        if what == 0:
            dst[g.integers(n)] = dst[0]
        if what == 1:
            src[g.integers(n)] = [-1, blocks if blocks < 2**31 - 1 else -5][g.integers(2)]
        if what >= 3:                       # sources away from the destinations
            src = np.setdiff1d(src, dst)
            dst = dst[:len(src)]
        want = fk.OK
        if any(not 0 <= x < blocks for x in [*src, *dst]):
            want = fk.ERANGE
        elif len(set(dst.tolist())) < len(dst) or set(dst.tolist()) & set(src.tolist()):
            want = fk.EDUP
        got = check(blocks, src, dst)
        if want == fk.ERANGE and got == fk.EDUP:     # (a repeated destination came first)
            assert len(set(dst.tolist())) < len(dst)
        else:
            assert got == want, (blocks, src, dst)
        seen[got] = seen.get(got, 0) + 1
    assert len(seen) == 3 and min(seen.values()) > 50, seen


def test_long_lists():
    n = 200_000
    ids = np.random.default_rng(1).permutation(2 * n)
    assert check(2 * n, ids[:n], ids[n:]) == fk.OK
    ids[n - 1] = ids[2 * n - 1]
    assert check(2 * n, ids[:n], ids[n:]) == fk.EDUP


def test_memory_goes_by_the_lists_and_not_by_the_pool():
    """Two pairs in a pool of 2^31 - 1 blocks, with 512 MiB of address space left."""
    script = """
import resource
from tests.test_copy_blocks_host import check, fk
check(8, [1], [2])
size = int([x for x in open("/proc/self/status") if x.startswith("VmSize")][0].split()[1]) * 1024
resource.setrlimit(resource.RLIMIT_AS, (size + (512 << 20),) * 2)
assert check(2**31 - 1, [1, 2], [2**31 - 2, 7]) == fk.OK
assert check(2**31 - 1, [1, 2], [7, 7]) == fk.EDUP
"""
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr
