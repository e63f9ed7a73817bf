"""Attention over shared prefixes (GPU) in the plans that a batch's sizes lead to, against the
formula of attention over all of each request's tokens, with the bounds that
tests/span_batch.py derives."""

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM
from tests.paged_batch import U, Batch
from tests.span_batch import check_span, group_batch, half_step
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


def test_many_requests_with_room_for_long_ones():
    """Single tokens of 20,000 requests behind one prefix, in a call that has room for half a
    million tokens of their own: 5 million workgroups, nearly all with nothing to do.  Queries of
    zero weigh all tokens alike: an output is the mean of what its row sees, rounded once behind
    sums that bfloat16 values of these sizes leave exact but for float32's last bits."""
    n, p, bs, d, most_own = 20_000, 32, 16, 64, 500_000
    g = np.random.default_rng(26)
    own = g.integers(1, bs + 1, n)
    b = Batch(Geometry("premost", 1, 1, d, bs, "bfloat16"), BM, np.ones(n, int), own, 26)
    shared = np.arange(b.blocks, b.blocks + 2)
    t = torch.cat([b.pool.tensors[0], b.pool.tensors[0][:2]])
    b.blocks += 2
    b.pool = fk.KVPool(BM, t)
    b.tab = np.ascontiguousarray(np.concatenate([np.tile(shared, (n, 1)), b.tab[:, :1]], 1), np.int32)
    b.total = own + p
    b.upload()
    q = torch.zeros((n, 1, d), dtype=torch.bfloat16, device="cuda")
    say("20,000 requests with room for 500,000 tokens each")
    out = attend(b, 0, q, 0.1, [0, n], [p], 0, (1, n, most_own, p))
    v = b.layer_view(0)[1].double()[:, :, 0]                            # (blocks, bs, d)
    mine = v[torch.as_tensor(b.tab[:, 2].astype(np.int64), device="cuda")].cumsum(1)
    last = torch.as_tensor(own - 1, device="cuda")[:, None, None].expand(-1, 1, d)
    want = (mine.gather(1, last)[:, 0] + v[[int(x) for x in shared]].sum((0, 1)))
    count = torch.as_tensor(own + p, device="cuda")[:, None].double()
    size = v.abs().amax() * count                                       # of a sum's parts
    tol = half_step(torch.bfloat16) * (want / count).abs() + 64 * U * size / count
    assert ((out[:, 0].double() - want / count).abs() <= tol).all()
