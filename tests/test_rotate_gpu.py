"""Rotated appends (GPU): q and K against the formula in 64 bits within the roundings that
tests/span_batch.py counts, V and every other byte of the pool bit for bit."""

import sys

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch
from tests.span_batch import check_rotated, rotated_plain

pytestmark = pytest.mark.gpu
NAMES = {LM: "layer", BM: "block"}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def table(positions, rot, base=10000.0):
    freq = base ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    x = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * freq
    return torch.cat([x.cos(), x.sin()], 1).float().contiguous()


def batch(shape, layout, new, total, seed, pad=(0, 0)):
    L, hk, _, d, _, bs, dtype = shape
    b = Batch(Geometry("rot", L, hk, d, bs, "bfloat16"), layout, new, total, seed, pad=pad)
    if dtype != "bfloat16":
        b.pool = fk.KVPool(layout, [t.to(getattr(torch, dtype)) for t in b.pool.tensors])
    return b


def rows(b, heads, seed, lead=0, tail=0):
    """(n, heads, dim) as columns `lead` on of a matrix with `tail` more behind."""
    d, dtype = b.geom.head_dim, b.pool.dtype
    x = torch.randn((b.n_tokens, lead + heads * d + tail), device="cuda",
                    generator=torch.Generator("cuda").manual_seed(seed)).to(dtype)
    return x[:, lead:lead + heads * d].unflatten(1, (heads, d))


def positions(b):
    """Of every row of the batch; -1 for rows of no request."""
    pos = np.full(b.n_tokens, -1, np.int64)
    for r, i, row in b.rows():
        pos[row] = int(b.total[r] - b.new[r]) + i
    return pos


def check(b, layer, q, k, v, angles, interleaved, in_place=False, stream=None):
    hk = b.geom.kv_heads
    rot = angles.shape[1]
    pos = positions(b)
    done = torch.as_tensor((pos >= 0) & (pos < len(angles)), device="cuda")
    at = torch.as_tensor(pos, device="cuda").clamp(0, max(len(angles) - 1, 0))
    some = angles if len(angles) else angles.new_zeros((1, rot))
    want_k, size_k = rotated_plain(k, at, some, interleaved)
    before = [t.clone() for t in b.pool.tensors]
    out = None
    if q is not None:
        want_q, size_q = rotated_plain(q, at, some, interleaved)
        out = q if in_place else torch.full_like(rows(b, q.shape[1], 0, 0, 16), 7.0)
        old = out.clone()
    fk.flowkv_append_rotated(b.pool, layer, k, v, angles, *b.args(), q=q, q_out=out,
                             interleaved=interleaved, stream=stream)
    torch.cuda.synchronize()
    if q is not None:
        assert torch.equal(out[~done], old[~done]), "a row that has no position was written"
        check_rotated(out[done], want_q[done], size_q[done], rot)
    # the pool: V in its slots bit for bit, K within its bound, nothing else changed
    got_k, kept = k.clone(), []
    bs, view, old_view = b.geom.block_size, b.layer_view(layer), b.layer_view(layer, before)
    for r, i, row in b.rows():
        p = pos[row]
        if not 0 <= p < len(angles) or p // bs >= b.tab.shape[1]:
            continue
        blk = int(b.tab[r, p // bs])
        if 0 <= blk < b.blocks:
            got_k[row] = view[0, blk, p % bs]
            old_view[0, blk, p % bs], old_view[1, blk, p % bs] = got_k[row], v[row]
            kept.append(row)
    kept = torch.as_tensor(kept, dtype=torch.int64, device="cuda")
    check_rotated(got_k[kept], want_k[kept], size_k[kept], rot)
    for x, y in zip(b.pool.tensors, before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), "other bytes of the pool"


SHAPES = [  # (layers, KV heads, query heads, head_dim, rot_dim, block size, dtype)
    (2, 2, 8, 128, 128, 16, "bfloat16"), (3, 1, 8, 64, 64, 16, "float16"),
    (1, 8, 32, 128, 64, 1, "bfloat16"), (2, 3, 3, 64, 16, 7, "float16"),
    (2, 1, 0, 128, 128, 16, "bfloat16"), (1, 2, 5, 80, 48, 3, "bfloat16"),
    (2, 2, 2, 24, 16, 5, "float16"), (1, 2, 4, 64, 64, 16, "float32"), (2, 1, 3, 12, 8, 4, "float32"),
    (1, 4, 64, 256, 256, 16, "bfloat16"),
]
BATCHES = [  # (new tokens, tokens in all)
    ([1], [1]), ([1] * 70, list(range(1, 71))), ([0, 5, 0, 1, 0], [3, 5, 0, 90, 0]), ([300], [300]),
    ([40, 1, 260], [77, 1, 1000]), ([1] * 5, [0, -3, 17, 16, 33]), ([6, 4], [3, 1000]),
]


@pytest.mark.parametrize("case", range(len(BATCHES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_formula(shape, case):
    L, hk, hq, d, rot, bs, dtype = SHAPES[shape]
    seed = 13 * shape + case
    layout = (BM, LM)[seed % 2]
    b = batch(SHAPES[shape], layout, *BATCHES[case], seed, pad=(seed % 3, seed % 4))
    say(f"rotated append {NAMES[layout]} {SHAPES[shape]} new {b.new.tolist()[:8]}")
    lead, tail = 16 * (seed % 2), 16 * (seed % 3)
    q = rows(b, hq, seed, lead, tail) if hq else None
    check(b, L - 1, q, rows(b, hk, seed + 1, tail, lead), rows(b, hk, seed + 2),
          table(max(1, b.max_len), rot), bool(case % 2 ^ shape % 2), in_place=seed % 5 == 0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_past_the_table_and_blocks_outside_the_pool(interleaved):
    b = Batch(Geometry("rotout", 2, 2, 64, 16, "bfloat16"), BM, [40, 6, 3], [100, 50, 700], 5)
    b.tab[0, [4, 5]] = [-1, b.blocks]
    b.tab[1, 2] = 2**31 - 1
    b.total[2] = 710        # behind the block list's 44 blocks
    b.upload()
    for n in (0, 1, 48, 77, 705, 1000):
        check(b, 1, rows(b, 4, 6), rows(b, 2, 7), rows(b, 2, 8), table(n, 64), interleaved)


def test_no_block_list_rotates_queries_alone():
    b = Batch(Geometry("rotnone", 1, 1, 64, 16, "bfloat16"), LM, [3], [9], 9)
    b.tab = np.zeros((1, 0), np.int32)
    b.upload()
    check(b, 0, rows(b, 2, 6), rows(b, 1, 7), rows(b, 1, 8), table(9, 64), False)


def test_far_positions_use_their_own_row():
    """Angles as the table has them: any float32, not cosines of anything."""
    g = torch.Generator("cuda").manual_seed(3)
    angles = torch.randn((200_000, 32), device="cuda", generator=g)
    b = Batch(Geometry("rotfar", 1, 1, 64, 16, "bfloat16"), LM, [5, 2], [200_000, 131_073], 11)
    check(b, 0, rows(b, 2, 6), rows(b, 1, 7), rows(b, 1, 8), angles, False)


def test_infinities_and_nan_stay_in_their_pairs():
    b = Batch(Geometry("rotodd", 1, 1, 64, 16, "bfloat16"), LM, [3], [50], 12)
    k, v = rows(b, 1, 7).contiguous(), rows(b, 1, 8).contiguous()
    angles = table(50, 32)
    fk.flowkv_append_rotated(b.pool, 0, k, v, angles, *b.args())
    view, blk = b.layer_view(0), int(b.tab[0, 3])
    ref = view[0, blk, 0].clone()
    k[1, 0, 3], k[1, 0, 40] = float("nan"), float("inf")
    fk.flowkv_append_rotated(b.pool, 0, k, v, angles, *b.args())
    got = view[0, blk, 0, 0]
    bad = [3, 19, 40]
    assert torch.isnan(got[[3, 19]].float()).all() and got[40] == float("inf")
    rest = [i for i in range(64) if i not in bad]
    assert torch.equal(got[rest], ref[0, rest])


def test_many_requests_and_blocks_beyond_4_gib():
    g = np.random.default_rng(15)
    for n, geom, spare in ((65, Geometry("rotmany", 1, 1, 64, 16, "bfloat16"), 5),
                           (3000, Geometry("rotmany", 1, 2, 64, 16, "float16"), 5),
                           (9, Geometry("rotbig", 4, 8, 128, 16, "bfloat16"), 20_000)):
        new = g.integers(0, 4, n)
        for layout in (BM, LM):
            b = Batch(geom, layout, new, new + g.integers(0, 30, n), 15, spare=spare)
            say(f"rotated append of {n} requests, {b.blocks} blocks, {NAMES[layout]}")
            check(b, 0, rows(b, 2, 6), rows(b, geom.kv_heads, 7), rows(b, geom.kv_heads, 8),
                  table(40, 64), False)


def test_streams_and_a_replayed_graph():
    b = Batch(Geometry("rotgraph", 2, 2, 64, 16, "bfloat16"), LM, [40, 1, 9], [90, 500, 9], 17)
    angles = table(1000, 64)
    check(b, 1, rows(b, 4, 6), rows(b, 2, 7), rows(b, 2, 8), angles, False,
          stream=torch.cuda.Stream())
    q, k, v = rows(b, 4, 26), rows(b, 2, 27), rows(b, 2, 28)
    out = torch.zeros_like(q, memory_format=torch.contiguous_format)

    def call():
        fk.flowkv_append_rotated(b.pool, 1, k, v, angles, *b.args(), q=q, q_out=out)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, total in (([40, 1, 9], [91, 499, 9]), ([0, 30, 20], [90, 60, 20]),
                       ([10, 10, 30], [33, 512, 30])):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.tab = np.random.default_rng(sum(total)).permutation(b.blocks)[
            :b.tab.size].reshape(b.tab.shape).astype(np.int32) if b.blocks >= b.tab.size else b.tab
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.tables.copy_(torch.as_tensor(b.tab))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        for t in b.pool.tensors:
            t.normal_()
        out.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        got, left = out.clone(), [t.clone() for t in b.pool.tensors]
        for t in b.pool.tensors:
            t.normal_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[:int(b.off[-1])], out[:int(b.off[-1])])
        view = b.layer_view(1)
        old = b.layer_view(1, left)
        for r, i, row in b.rows():
            p = int(b.total[r] - b.new[r]) + i
            if p >= 0 and 0 <= b.tab[r, p // 16] < b.blocks:
                assert torch.equal(view[:, int(b.tab[r, p // 16]), p % 16],
                                   old[:, int(b.tab[r, p // 16]), p % 16])


def test_the_binding_refuses_other_types_shapes_and_devices():
    b = Batch(Geometry("rotrefuse", 1, 2, 64, 16, "bfloat16"), LM, [3], [9], 9)
    q, k, v, t = rows(b, 4, 6), rows(b, 2, 7), rows(b, 2, 8), table(9, 64)
    good = dict(k=k, v=v, cos_sin=t, q=q, q_out=torch.empty_like(q))

    def call(**c):
        a = {**good, **c}
        fk.flowkv_append_rotated(b.pool, 0, a["k"], a["v"], a["cos_sin"], *b.args(), q=a["q"],
                                 q_out=a["q_out"])
    call()
    for c in (dict(k=k.half()), dict(v=v[:2]), dict(cos_sin=t.double()), dict(cos_sin=t.cpu()),
              dict(cos_sin=t[:, ::2]), dict(q=q[:2]), dict(q_out=None), dict(q_out=k),
              dict(q=q.flatten(1)), dict(q=q.transpose(1, 2)), dict(k=k[:, :, :32])):
        with pytest.raises(ValueError):
            call(**c)
    for c in (dict(cos_sin=table(9, 72)[:, :72]), dict(cos_sin=table(9, 8))):
        with pytest.raises(fk.FlowKVError):
            call(**c)
