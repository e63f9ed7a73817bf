"""The workspace that attention of new tokens asks for under the library's own rule (CPU):
bounded as include/flowkv.h says, whatever the batch is padded to."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2504_03775_amd import flowkv as fk
from tests.test_pages_host import chunk, pool

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = 34_080_772       # bytes, where requests bring more than 32 rows a KV head
workspace = fk.flowkv_chunk_attention_workspace


def records(n, hq, d, splits):
    return n * hq * splits * (d + 2) * 4 if splits > 1 else 0


@pytest.mark.parametrize("n,req,hq,hk,d,new,top", [
    (20000, 8, 8, 1, 128, 300, 32768),          # a captured batch, mostly padding
    (16384, 8, 8, 1, 128, 256, 32768), (16384, 8, 8, 2, 64, 256, 32768),
    (2000, 200, 8, 1, 128, 16, 1 << 20),        # long contexts
    (2000, 2, 32, 8, 128, 1000, 1 << 29), (64, 1, 8, 1, 64, 64, (1 << 31) - 5000),
    (20000, 1, 8, 1, 128, 40, 10000),           # few rows, and steps, in all
    (100000, 1, 32, 8, 128, 30, 500), (1 << 20, 4, 8, 8, 64, 40, 3000),
    (2**31 - 1000, 1, 1, 1, 128, 40, 100000),
])
def test_workspace_of_many_rows_has_a_bound(n, req, hq, hk, d, new, top):
    assert new * hq // hk > 32
    assert workspace(n, req, hq, hk, d, new, top) <= MOST


def test_workspace_of_many_rows_has_a_bound_over_random_batches():
    g = np.random.default_rng(60)

    def spread(most):
        return int(np.exp(g.uniform(0, np.log(most))))
    some = 0
    for _ in range(20000):
        hk, G, d = spread(16), spread(64), (64, 128)[int(g.integers(2))]
        new, req, top = spread(40000), spread(600), spread(1 << 30)
        n = min(spread(8) * new * req if g.integers(2) else spread(1 << 20), 1 << 24)
        if new * G <= 32:
            continue
        need = workspace(n, req, hk * G, hk, d, new, top)
        some += need > 0
        assert need <= MOST, (n, req, hk * G, hk, d, new, top)
    assert some > 1000


def test_workspace_of_few_rows_is_a_whole_number_of_splits():
    for n, req, hq, hk, d, new, top in ((5, 1, 32, 8, 128, 5, 13000), (120, 24, 32, 8, 128, 8, 16000),
                                        (64, 64, 8, 1, 128, 1, 4000), (7, 1, 8, 8, 64, 7, 1 << 20),
                                        (4096, 16, 8, 1, 128, 4, 32768)):
        assert new * hq // hk <= 32
        need = workspace(n, req, hq, hk, d, new, top)
        sizes = {records(n, hq, d, -(-top // s)) for s in range(128, 2049, 128)}
        assert need in sizes and need > 0, (need, n, req)


def test_workspace_of_a_given_split_counts_every_row():
    for split in (64, 128, 2048, 4096):
        for new in (1, 300):
            assert workspace(20000, 8, 8, 1, 128, new, 32768, split) == \
                records(20000, 8, 128, 32768 // split)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_splits_are_counted_to_the_end_of_32_bits(tmp_path):
    """As the join of a row's splits counts them: with more than 2^30 tokens in splits of
    about as many, the tokens and the split together pass 32 bits."""
    exe = str(tmp_path / "splits_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2504_03775_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "splits_check.cpp"), "-o", exe],
                   check=True, capture_output=True, timeout=120)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "counts ok" in r.stdout, r.stdout + r.stderr


def test_a_scale_that_passes_float32_in_powers_of_two_is_refused():
    """scale x log2(e) above float32's largest: every score would be 0 x inf."""
    p = pool()
    for scale in (3e38, 2.4e38):
        assert chunk(p, n=0, scale=2.3e38) == fk.OK
        assert chunk(p, n=0, scale=scale) == fk.EINVAL
