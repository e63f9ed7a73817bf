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
