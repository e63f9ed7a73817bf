"""Attention over shared prefixes (GPU) in the plans that a batch's sizes lead to, against the
formula of attention over all of each request's tokens, with the bounds that
tests/span_batch.py derives."""

import pytest

from workloads import Geometry
from tests.gpu_helpers import BM
from tests.span_batch import check_span, group_batch
from tests.test_prefix_attention_gpu import attend, say, sizes
from tests.test_window_attention_gpu import queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("split", [64, 128, 1024, 4096])
@pytest.mark.parametrize("new", [1, 5, 90])
def test_split_tokens_with_nothing_to_share(new, split):
    """No group, and groups of a prefix without tokens."""
    reqs = [(new, new + 700), (1, 300), (1, 1), (0, 9)]
    b, bounds, prefixes = group_batch(Geometry("prealone", 1, 2, 128, 16, "bfloat16"), BM,
                                      [(0, reqs)], 24, pad=(2, 3))
    q = queries(b, 8, 24)
    most = sizes(b, bounds, prefixes)
    say(f"nothing shared: {new} new tokens, split {split}")
    check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, bounds, prefixes, split))
    # (in no group, a prefix that is told counts as tokens of a request)
    check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, [0], [], split, (*most[:3], 50)))


@pytest.mark.parametrize("hk,d,G,dtype", [(8, 128, 4, "bfloat16"), (1, 128, 8, "float16"),
                                          (4, 64, 2, "bfloat16")])
@pytest.mark.parametrize("new", [17, 100, 400])
def test_a_long_request_beside_single_tokens(new, hk, d, G, dtype):
    """Shared by the library's rule, with more rows than a tile of any kind holds."""
    groups = [(3500, [(1, 1 + 7 * i) for i in range(40)] + [(new, new + 130)]),
              (1200, [(new // 2, new), (1, 9), (0, 0), (1, 1)] * 6)]
    b, bounds, prefixes = group_batch(Geometry("premixed", 1, hk, d, 16, dtype), BM, groups, 25,
                                      pad=(2, 3))
    rows, most = b.n_tokens * G, sizes(b, bounds, prefixes)
    say(f"{new} new tokens beside single ones, {rows / len(b.new):.0f} rows a request")
    q = queries(b, hk * G, 25)
    for split in (0, 512):
        check_span(b, 0, q, d ** -0.5, attend(b, 0, q, d ** -0.5, bounds, prefixes, split))
    # sizes above what there is
    check_span(b, 0, q, d ** -0.5, attend(b, 0, q, d ** -0.5, bounds, prefixes, 0,
                                          (most[0], most[1], most[2] + 900, most[3] + 500)))
