"""Attention of new tokens (GPU): every token that a row sees counts once, and no other, at
lengths where a token more or less lies far inside the bounds of rounding.

With queries of zero every weight is 1 (2^0) and the weights' sum is the number n of tokens
seen, both exact.  V is 1 in dim c of the tokens of class c, a run of `run` tokens, and 0
elsewhere: out[c] is the bf16 nearest to (tokens of class c seen) / n, up to two roundings
of float32 (1 / n, and the product with the count): half a bf16 step and 2^-23, of itself.
One token of a whole class more or less is 1 / run of it: 2^-5 at runs of 32, eight times
2^-8."""

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import BF16_HALF_STEP, Batch
from tests.test_chunk_attention_gpu import LONGEST, say

pytestmark = pytest.mark.gpu
RUN = 32


def mark(b, first):
    """Dim c of V: 1 for the tokens of positions first + c x RUN .. first + (c + 1) x RUN."""
    view, bs, d = b.layer_view(0), b.geom.block_size, b.geom.head_dim
    view[0] = 0.5
    view[1] = 0
    for r in range(len(b.new)):
        p = np.arange(first, min(first + d * RUN, int(b.total[r])))
        if p.size:
            at = [torch.as_tensor(x, device="cuda")
                  for x in (b.tab[r, p // bs].astype(np.int64), p % bs, (p - first) // RUN)]
            view[1][at[0], at[1], :, at[2]] = 1


def counts(b, first):
    """(new tokens, dims) counts of tokens seen, a row per new token, and the tokens seen."""
    d = b.geom.head_dim
    edges = first + np.arange(d + 1) * RUN
    n = np.concatenate([b.total[r] - b.new[r] + 1 + np.arange(b.new[r])
                        for r in range(len(b.new))])
    return np.diff(np.minimum(edges[None], n[:, None]), axis=1).astype(np.float64), n


BATCHES = [
    ([3], [9000]), ([1, 8], [20000, 8191]), ([40, 1], [9001, 16385]), ([300], [20000]),
    ([130, 2, 61], [4097, 12288, 9999]), ([700, 700], [700, 10007]), ([2100], [2100]),
]


@pytest.mark.parametrize("form", ["rule", "pieces", "order", 64, 192, 2048, 4096])
@pytest.mark.parametrize("d,hk,G,layout,bs", [(128, 2, 4, BM, 16), (64, 1, 8, LM, 7),
                                              (128, 1, 5, LM, 33)])
def test_every_seen_token_counts_once(d, hk, G, layout, bs, form):
    for i, (new, total) in enumerate(BATCHES):
        if form == "order":                         # more tiles than CUs: 300 more requests
            new = new + [1 + 50 // G] * 300
            total = total + [60 + 11 * j for j in range(300)]
        b = Batch(Geometry("counts", 1, hk, d, bs, "bfloat16"), layout, new, total, 100 + i)
        max_len = LONGEST if form == "pieces" else b.max_len
        split = form if isinstance(form, int) else 0
        q = torch.zeros((b.n_tokens, hk * G, d), dtype=torch.bfloat16, device="cuda")
        out = torch.zeros_like(q)
        need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(b.new), hk * G, hk, d, b.max_new,
                                                   max_len, split)
        ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")
        worst = 0.0
        for first in range(0, b.max_len, d * RUN):
            mark(b, first)
            out.fill_(7)
            fk.flowkv_chunk_attention(b.pool, 0, q, *b.args(), b.max_new, max_len, 0.3, out, ws,
                                      split)
            seen, n = counts(b, first)
            want = torch.as_tensor(seen / n[:, None], device="cuda")[:, None, :]
            got = out.double()
            err = (got - want).abs()
            assert (err <= (BF16_HALF_STEP + 2.0 ** -23) * want).all(), \
                f"first {first}: rows {(err > BF16_HALF_STEP * want * 1.01).nonzero()[:8].tolist()}"
            worst = max(worst, float((err / want.clamp(min=1e-30)).max()))
        say(f"new {new[:4]} of {total[:4]} {form}: {need} bytes, error {worst:.2e} of the value")
