"""Attention of new tokens (GPU) where the host knows little of the batch: rows of padding
before and behind it, as a captured call has them, and a max_new below the requests' own."""

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch, check_attention
from tests.test_chunk_attention_gpu import BATCHES, LONGEST, MIXED, SHAPES, queries, say

pytestmark = pytest.mark.gpu


def attend_as(b, q, scale, max_new, split=0, max_len=None, layer=0):
    """The call with `max_new`; nothing behind its workspace, and no padding row, changes."""
    max_len = b.max_len if max_len is None else max_len
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(b.new), q.shape[1], b.geom.kv_heads,
                                               b.geom.head_dim, max_new, max_len, split)
    ws = torch.full((need + 65536,), 90, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    fk.flowkv_chunk_attention(b.pool, layer, q, *b.args(), max_new, max_len, scale, out,
                              ws[:need] if need else None, split)
    torch.cuda.synchronize()
    assert (ws[need:] == 90).all(), "written behind the workspace"
    inside = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
    inside[int(b.off[0]):int(b.off[-1])] = True
    assert (out[~inside] == 7).all(), "a row of no request was written"
    return out, need


PADS = [(0, 30000), (30000, 0), (9000, 20001)]


@pytest.mark.parametrize("pad", range(len(PADS)))
@pytest.mark.parametrize("d,hk,G,layout,new,total", [
    (128, 1, 8, BM, [300, 40, 200, 17], [5000, 40, 900, 3000]), (64, 2, 4, LM, [100, 290], [3000, 290]),
    (128, 2, 8, LM, [40], [10000]), (64, 1, 16, BM, [0, 60, 0, 3], [0, 60, 9, 7000]),
    (128, 8, 4, BM, [64] * 40 + [10] * 20, [64 + 30 * i for i in range(60)]),
    (64, 8, 2, LM, [120] * 20 + [1] * 30, [120 + 40 * i for i in range(50)]),
])
def test_padding_around_the_batch(d, hk, G, layout, new, total, pad):
    b = Batch(Geometry("padded", 1, hk, d, 16, "bfloat16"), layout, new, total, 70 + pad,
              pad=PADS[pad])
    q = queries(b, hk * G, 70)
    for max_len in (b.max_len, 32768, LONGEST):
        out, need = attend_as(b, q, d ** -0.5, b.max_new, max_len=max_len)
        say(f"  {need} bytes of workspace")
        assert need <= 34_080_772
        check_attention(b, 0, q, d ** -0.5, out, max_seq=max_len)


@pytest.mark.parametrize("split,longest", [(0, False), (0, True), (64, False), (4096, False)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rows_past_max_new_are_computed(shape, split, longest):
    L, hk, d, bs, G = SHAPES[shape]
    for i, (new, total) in enumerate(BATCHES[3:8:2] + MIXED[4:5] + MIXED[8:]):
        b = Batch(Geometry(f"past{shape}", L, hk, d, bs, "bfloat16"), (BM, LM)[(i + shape) % 2], new,
                  total, 80 + i, pad=(i % 3, shape % 4))
        q = queries(b, hk * G, 80 + i)
        for max_new in sorted({i % 2, max(b.max_new // 4, 1)}):
            say(f"shape {SHAPES[shape]} new {new} as if {max_new}, split {split}")
            max_len = LONGEST if longest else b.max_len
            out, _ = attend_as(b, q, d ** -0.5, max_new, split, max_len, L - 1)
            check_attention(b, L - 1, q, d ** -0.5, out, max_seq=max_len)


@pytest.mark.parametrize("d,hk,G,new,total,max_new,longest", [
    (128, 1, 8, [3000, 2990], [3000, 9000], 8, True),           # many tiles for two pieces' room
    (64, 2, 8, [3000, 10], [3100, 10], 5, True),
    (128, 8, 8, [1] * 29 + [121], [50 * i + 1 for i in range(29)] + [800], 5, True),
    # (33 tiles a head, 32 pieces)
    (128, 1, 8, [1] * 299 + [2000], [i + 1 for i in range(299)] + [2600], 5, False),
    (64, 2, 8, [5] * 199 + [2000], [i + 5 for i in range(199)] + [2600], 5, False),
])
def test_more_tiles_than_max_new_makes_room_for(d, hk, G, new, total, max_new, longest):
    b = Batch(Geometry("tilespast", 1, hk, d, 16, "bfloat16"), BM, new, total, 90, pad=(3, 500))
    q = queries(b, hk * G, 90)
    max_len = LONGEST if longest else b.max_len
    out, _ = attend_as(b, q, d ** -0.5, max_new, 0, max_len)
    check_attention(b, 0, q, d ** -0.5, out, max_seq=max_len)
    assert torch.isfinite(out[3:3 + sum(new)].float()).all()


def test_rows_past_what_a_join_could_launch():
    """2^26 output rows and more, most of them padding, in a call that joins no splits."""
    hq, d, n = 32, 64, (1 << 21) + 40
    b = Batch(Geometry("padmany", 1, 2, d, 16, "bfloat16"), BM, [30, 1], [300, 40], 95,
              pad=(n - 36, 5))
    assert b.n_tokens == n and n * hq > 1 << 26
    q = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda")
    first = int(b.off[0])
    q[first:] = torch.randn((n - first, hq, d), device="cuda",
                            generator=torch.Generator("cuda").manual_seed(95)).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    assert fk.flowkv_chunk_attention_workspace(n, 2, hq, 2, d, 30, 1 << 20, 1 << 20) == 0
    fk.flowkv_chunk_attention(b.pool, 0, q, *b.args(), 30, 1 << 20, 0.1, out, None, 1 << 20)
    torch.cuda.synchronize()
    check_attention(b, 0, q, 0.1, out, max_seq=1 << 20)
    assert (out[:first] == 7).all() and (out[-5:] == 7).all()
