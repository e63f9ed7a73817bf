"""Which calls cut the tiles behind the last whole round into pieces (GPU): those leave records in
their workspace, whole tiles nothing.  Either way the outputs are the formula's, within the bounds
that tests/span_batch.py derives."""

import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch
from tests.span_batch import check_span
from tests.test_prefix_attention_gpu import i32, say
from tests.test_window_attention_gpu import queries

pytestmark = pytest.mark.gpu

CASES = [  # (KV heads, query heads per KV head, new tokens, tokens in all, cut)
    (8, 8, [1030], [4000], True),                   # 264 tiles of 256 rows: 1.03 rounds
    (8, 8, [1280], [2900], True),                   # 320
    (16, 4, [600, 600], [3000, 3000], True),        # 320
    (8, 8, [2040], [4000], False),                  # 512: no tail
    (8, 8, [1800], [4000], False),                  # 456: most of the last round in use
    (8, 8, [300] * 6, [2300] * 6, False),           # 480
    (8, 8, [1500], [2200], False),                  # 376, of 12 to 35 steps
    (8, 8, [2100], [2100], False),                  # 528, of 1 to 33 steps
]


@pytest.mark.parametrize("call", ["window", "prefix"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_tails_where_they_pay(case, call):
    hk, G, new, total, cut = CASES[case]
    b = Batch(Geometry("tails", 1, hk, 128, 16, ("bfloat16", "float16")[case % 2]),
              (BM, LM)[case % 2], new, total, 60 + case)
    q = queries(b, hk * G, 60 + case)
    shape = (b.n_tokens, len(new), hk * G, hk, 128)
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    longest = b.max_len
    say(f"{call} {hk} x {G} new {new} of {total}: {'a tail in pieces' if cut else 'whole tiles'}")
    if call == "window":
        need = fk.flowkv_window_attention_workspace(*shape, b.max_new, longest, 2**18, 4)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        fk.flowkv_window_attention(b.pool, 0, q, *b.args(), b.max_new, longest, 2**18, 4, 0.09, out,
                                   ws)
    else:
        need = fk.flowkv_prefix_attention_workspace(*shape, 0, b.max_new, 0, longest, 0)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        fk.flowkv_prefix_attention(b.pool, 0, q, *b.args(), i32([0]), i32([]), b.max_new, 0,
                                   longest, 0, 0.09, out, ws)
    torch.cuda.synchronize()
    assert bool((ws != 255).any()) == cut
    check_span(b, 0, q, 0.09, out)
