"""Rotated appends of many tokens (GPU), where a lane takes two heads and, from 32 MiB of stores
on, they go past the caches: q and K against the formula in 64 bits within the roundings that
tests/span_batch.py counts, V and every other byte of the pool bit for bit."""

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from tests.gpu_helpers import BM, LM
from tests.span_batch import check_rotated, rotated_plain
from tests.test_rotate_gpu import NAMES, batch, positions, rows, say, table

pytestmark = pytest.mark.gpu

MIB = 1 << 20
FORMS = {"two heads a lane": 6 * MIB, "past the caches": 34 * MIB}     # bytes stored, at least
SHAPES = [  # (layers, KV heads, query heads, head_dim, rot_dim, block size, dtype)
    (1, 2, 5, 128, 128, 16, "bfloat16"), (2, 1, 8, 128, 64, 16, "bfloat16"),
    (1, 2, 3, 80, 48, 3, "bfloat16"), (1, 3, 9, 24, 16, 5, "bfloat16"),
    (2, 2, 7, 64, 64, 16, "float16"), (1, 4, 1, 64, 32, 7, "float16"), (1, 1, 0, 128, 16, 1, "float16"),
    (1, 2, 3, 72, 64, 9, "float16"), (1, 2, 4, 64, 64, 16, "float32"), (1, 1, 3, 20, 8, 4, "float32"),
    (2, 3, 2, 128, 96, 16, "float32"),
]


def lengths(n, seed):
    """New tokens and tokens in all of requests that have n new ones between them: single
    tokens, empty requests and long ones."""
    g = np.random.default_rng(seed)
    new = [1] * 40 + [0, 0]
    while (left := n - sum(new)) > 0:
        new.append(min(left, int(g.integers(1, max(2, n // 3)))))
    new = g.permutation(new)
    return new, new + g.integers(0, 500, len(new))


def check_long(b, layer, q, k, v, angles, interleaved, in_place):
    """The batch's rows that have a place in the table and the pool as the formula has them, all
    else unchanged."""
    bs, n = b.geom.block_size, b.n_tokens
    pos = positions(b)
    req = np.zeros(n, np.int64)
    req[int(b.off[0]):int(b.off[-1])] = np.repeat(np.arange(len(b.new)), b.new)
    done = (pos >= 0) & (pos < len(angles))
    at = np.clip(pos, 0, len(angles) - 1)
    blk = b.tab[req, np.clip(pos // bs, 0, b.tab.shape[1] - 1)].astype(np.int64)
    kept = done & (pos // bs < b.tab.shape[1]) & (blk >= 0) & (blk < b.blocks)
    done, at, blk, slot = (torch.as_tensor(x, device="cuda") for x in (done, at, blk, pos % bs))
    kept = torch.as_tensor(np.flatnonzero(kept), device="cuda")
    before = [t.clone() for t in b.pool.tensors]
    want_k, size_k = rotated_plain(k, at, angles, interleaved)
    out = None
    if q is not None:
        want_q, size_q = rotated_plain(q, at, angles, interleaved)
        out = q if in_place else torch.full_like(rows(b, q.shape[1], 0, 0, 16), 7.0)
        old = out[~done].clone()
    fk.flowkv_append_rotated(b.pool, layer, k, v, angles, *b.args(), q=q, q_out=out,
                             interleaved=interleaved)
    torch.cuda.synchronize()
    rot = angles.shape[1]
    if q is not None:
        assert torch.equal(out[~done], old), "a row that has no position was written"
        check_rotated(out[done], want_q[done], size_q[done], rot)
        del want_q, size_q
    view, old_view = b.layer_view(layer), b.layer_view(layer, before)
    blk, slot = blk[kept], slot[kept]
    got_k = view[0][blk, slot]
    check_rotated(got_k, want_k[kept], size_k[kept], rot)
    old_view[0][blk, slot] = got_k
    old_view[1][blk, slot] = v[kept]
    for x, y in zip(b.pool.tensors, before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), "other bytes of the pool"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_formula(shape, form, interleaved):
    L, hk, hq, d, rot, bs, dtype = SHAPES[shape]
    seed = 17 * shape + 2 * interleaved + len(form)
    head = d * (4 if dtype == "float32" else 2)
    heads = hq + 2 * hk
    n = FORMS[form] // (heads * head) + 1 + seed % 5
    # the sizes that the two forms begin at
    assert n * heads * -(-head // 32) > 1 << 17
    assert (n * heads * head > 32 * MIB) == (form == "past the caches")
    layout = (BM, LM)[seed % 2]
    b = batch(SHAPES[shape], layout, *lengths(n, seed), seed, pad=(seed % 3, seed % 4))
    say(f"rotated append, {form}, {NAMES[layout]} {SHAPES[shape]} {n} tokens")
    # a block outside the pool, two lists that end early by a -1, positions past the table
    b.tab[5 % len(b.new), 0] = b.blocks
    b.tab[-1, -1] = b.tab[len(b.new) // 2, 2 % b.tab.shape[1]] = -1
    b.upload()
    lead, tail = 16 * (seed % 2), 16 * (seed % 3)
    q = rows(b, hq, seed, lead, tail) if hq else None
    positions_ = max(1, b.max_len - (60 if shape % 3 == 0 else 0))
    check_long(b, L - 1, q, rows(b, hk, seed + 1, tail, lead), rows(b, hk, seed + 2),
               table(positions_, rot), interleaved, in_place=shape % 2 == 0)


def test_two_heads_a_lane_give_the_bits_of_one():
    """The same tokens in one call and in pieces of it that a lane takes one head of each."""
    b = batch(SHAPES[0], BM, *lengths(2600, 3), 3)
    k, v, q = rows(b, 2, 4), rows(b, 2, 5), rows(b, 5, 6)
    angles = table(b.max_len, 128)
    assert b.n_tokens * 9 * 8 > 1 << 17
    outs = [torch.empty_like(q) for _ in range(2)]
    fk.flowkv_append_rotated(b.pool, 0, k, v, angles, *b.args(), q=q, q_out=outs[0])
    torch.cuda.synchronize()
    ref = [t.clone() for t in b.pool.tensors]
    for t in b.pool.tensors:
        t.normal_()
    left = [t.clone() for t in b.pool.tensors]
    for r in range(len(b.new)):
        lo, hi = int(b.off[r]), int(b.off[r + 1])
        assert (hi - lo) * 9 * 8 <= 1 << 17
        if hi > lo:
            fk.flowkv_append_rotated(b.pool, 0, k[lo:hi], v[lo:hi], angles,
                                     torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda"),
                                     b.tables[r:r + 1], b.lens[r:r + 1], q=q[lo:hi],
                                     q_out=outs[1][lo:hi])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    pos, bs = positions(b), b.geom.block_size
    req = np.repeat(np.arange(len(b.new)), b.new)
    blk = torch.as_tensor(b.tab[req, pos // bs].astype(np.int64), device="cuda")
    slot = torch.as_tensor(pos % bs, device="cuda")
    view, old, was = b.layer_view(0), b.layer_view(0, ref), b.layer_view(0, left)
    assert torch.equal(view[:, blk, slot], old[:, blk, slot])
    was[:, blk, slot] = view[:, blk, slot]
    assert all(torch.equal(x, y) for x, y in zip(b.pool.tensors, left))
