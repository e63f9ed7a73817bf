"""Attention of new tokens over the paged cache (GPU) against its formula in 64 bits, with
the bounds that tests/paged_batch.py derives; rows that see nothing, block IDs outside the
pool, infinities and NaN in places that a row does not see, streams and graphs."""

import sys

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch, check_attention

pytestmark = pytest.mark.gpu
NAMES = {LM: "layer", BM: "block"}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def queries(b, q_heads, seed, gain=2.0, lead=0):
    """q as a slice of a wider row (lead elements before it) when lead is not 0."""
    d = b.geom.head_dim
    x = torch.randn((b.n_tokens, lead + q_heads * d),
                    generator=torch.Generator("cuda").manual_seed(seed + 7), device="cuda")
    return (gain * x).to(torch.bfloat16)[:, lead:].unflatten(1, (q_heads, d))


def attend(b, layer, q, scale, split=0, out=None, max_len=None, stream=None):
    max_len = b.max_len if max_len is None else max_len
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(b.new), q.shape[1],
                                               b.geom.kv_heads, b.geom.head_dim, b.max_new,
                                               max_len, split)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    fk.flowkv_chunk_attention(b.pool, layer, q, *b.args(), b.max_new, max_len, scale, out, ws,
                              split, stream=stream)
    torch.cuda.synchronize()
    return out


SHAPES = [  # (layers, KV heads, head_dim, block size, query heads per KV head)
    (2, 2, 128, 16, 4), (3, 1, 128, 16, 8), (2, 4, 64, 7, 2), (1, 2, 64, 16, 1),
    (2, 2, 128, 1, 3), (1, 1, 64, 100, 5), (2, 1, 128, 64, 7), (1, 3, 64, 3, 16), (1, 1, 128, 5, 40),
]
BATCHES = [  # (new tokens, tokens in all) of each request
    ([1], [1]), ([1, 1, 1], [1, 64, 65]), ([5], [300]), ([0, 3, 0, 2, 0], [9, 40, 0, 2, 700]),
    ([200], [200]), ([31, 33, 1], [31, 500, 129]), ([128, 127, 129], [128, 400, 129]),
    ([1, 260, 1, 70], [1000, 260, 63, 900]), ([16] * 9, [16 * (i + 1) for i in range(9)]),
    ([2, 8, 4, 1], [1500, 700, 4, 2000]), ([700], [1400]), ([1, 2, 1], [5000, 2049, 2048]),
    ([3], [9000]),
]


@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_formula(shape, batch):
    L, hk, d, bs, G = SHAPES[shape]
    seed = 31 * shape + batch
    layout = (BM, LM)[seed % 2]
    split = [0, 64, 128, 0, 1024, 2048, 4096][seed % 7]
    geom = Geometry(f"chunk{shape}", L, hk, d, bs, "bfloat16")
    b = Batch(geom, layout, *BATCHES[batch], seed, pad=(seed % 3, seed % 4))
    say(f"chunk attention {NAMES[layout]} shape {SHAPES[shape]} new {b.new.tolist()} of "
        f"{b.total.tolist()} split {split}")
    q = queries(b, hk * G, seed, lead=(0, 8, 2 * d)[seed % 3])
    out = attend(b, L - 1, q, d ** -0.5, split)
    rel, worst = check_attention(b, L - 1, q, d ** -0.5, out)
    say(f"  relative error {rel:.2e}, worst error / bound {worst:.2f}")
    inside = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
    inside[int(b.off[0]):int(b.off[-1])] = True
    assert (out[~inside] == 7).all(), "a row of no request was written"


@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
@pytest.mark.parametrize("new,total", [(2000, 9000), (3, 20000), (600, 600)])
def test_llama8b_geometry(layout, new, total):
    geom = Geometry("chunk8b", 4, 8, 128, 16, "bfloat16")
    b = Batch(geom, layout, [new, 1, 40], [total, 777, 2500], 3)
    say(f"chunk attention 8b {NAMES[layout]} {new} of {total}")
    q = queries(b, 32, 3)
    rel, worst = check_attention(b, 2, q, 128 ** -0.5, attend(b, 2, q, 128 ** -0.5))
    say(f"  relative error {rel:.2e}, worst error / bound {worst:.2f}")


@pytest.mark.parametrize("split", [64, 192, 0])
def test_large_scores_and_rising_maxima(split):
    """Scores of some hundreds, the largest at the end: every step moves the reference."""
    geom = Geometry("chunkbig", 1, 1, 64, 16, "bfloat16")
    b = Batch(geom, BM, [40, 5], [600, 333], 5)
    t = b.layer_view(0)
    for r in range(2):
        for p in range(int(b.total[r])):
            t[0, b.tab[r, p // 16], p % 16] *= p / 60
    q = queries(b, 4, 5, gain=8.0)
    out = attend(b, 0, q, 1.0, split)
    check_attention(b, 0, q, 1.0, out)


def test_one_token_returns_its_v_exactly():
    geom = Geometry("chunkone", 2, 2, 128, 16, "bfloat16")
    b = Batch(geom, LM, [1] * 20, [1] * 20, 8)
    q = queries(b, 8, 8)
    out = attend(b, 1, q, 0.3)
    v = b.layer_view(1)[1, torch.as_tensor(b.tab[:, 0].astype(np.int64), device="cuda"), 0]
    assert torch.equal(out, v.repeat_interleave(4, 1))


@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing_are_zero(d, split):
    """Lengths shorter than the new tokens (positions below 0), lengths of 0 and below."""
    geom = Geometry("chunknone", 1, 2, d, 16, "bfloat16")
    b = Batch(geom, BM, [5, 3, 200, 150], [2, 0, 130, 150], 9)
    b.total[1] = -4
    b.upload()
    q = queries(b, 4, 9)
    out = attend(b, 0, q, 0.1, split, max_len=150)
    for r in (0, 1, 2):
        first = int(b.off[r])
        none = int(min(b.new[r], b.new[r] - max(b.total[r], 0)))
        assert (out[first:first + none] == 0).all(), f"request {r}"
    check_attention(b, 0, q, 0.1, out, max_seq=150)


@pytest.mark.parametrize("split", [0, 64])
def test_blocks_outside_the_pool_contribute_nothing(split):
    geom = Geometry("chunkbad", 1, 2, 128, 16, "bfloat16")
    b = Batch(geom, LM, [70, 3, 1, 20], [400, 320, 40, 20], 10)
    b.tab[0, [0, 5, 11]] = [-1, b.blocks, 2**31 - 1]
    b.tab[1, 3:9] = -7
    b.tab[2, :] = -2**31
    b.tab[3, 0] = b.blocks + 1
    b.upload()
    q = queries(b, 8, 10)
    out = attend(b, 0, q, 0.09, split)
    check_attention(b, 0, q, 0.09, out)
    assert (out[int(b.off[2])] == 0).all()


def test_lengths_past_the_table_and_past_max_seq_len():
    """Tokens beyond max_blocks x block_size or beyond max_seq_len are not read."""
    geom = Geometry("chunkclamp", 1, 1, 128, 16, "bfloat16")
    b = Batch(geom, BM, [30, 4], [500, 200], 11)
    b.total[1] = 505        # 32 blocks listed (both rows have the widest's)
    b.tab[1, :] = b.tab[0, :]
    b.upload()
    q = queries(b, 4, 11)
    check_attention(b, 0, q, 0.09, attend(b, 0, q, 0.09, max_len=480), max_seq=480)
    b.total[0] += 100       # past the 32 listed blocks
    b.upload()
    check_attention(b, 0, q, 0.09, attend(b, 0, q, 0.09, max_len=b.max_len), max_seq=b.max_len)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_odd_values_reach_only_the_rows_that_see_them(d, split, bad):
    """V and K of a new token hold bad values: earlier rows are as if they did not; slots
    behind the last token hold them too, and reach no row."""
    geom = Geometry("chunkodd", 1, 1, d, 16, "bfloat16")
    b = Batch(geom, BM, [150, 90], [210, 101], 12)
    q = queries(b, 4, 12)
    ref = attend(b, 0, q, 0.1, split)
    t = b.layer_view(0)
    for r, p in ((0, 209), (1, 100)):               # slots behind the last token
        t[:, int(b.tab[r, p // 16]), p % 16 + 1:] = bad
    assert torch.equal(attend(b, 0, q, 0.1, split), ref)
    at = 130                                        # a position in the middle of request 0
    t[1, int(b.tab[0, at // 16]), at % 16, 0, 5] = bad
    out = attend(b, 0, q, 0.1, split)
    sees = 210 - 150 + np.arange(150) >= at
    first = int(b.off[0])
    rows = torch.as_tensor(first + np.flatnonzero(~sees), device="cuda")
    assert torch.equal(out[rows], ref[rows])
    rows = torch.as_tensor(first + np.flatnonzero(sees), device="cuda")
    hit = out[rows][:, :, 5].float()
    assert (torch.isnan(hit) if bad != bad else hit == bad).all()
    rest = [i for i in range(d) if i != 5]
    assert torch.equal(out[rows][:, :, rest], ref[rows][:, :, rest])
    assert torch.equal(out[int(b.off[1]):], ref[int(b.off[1]):])
    t[1, int(b.tab[0, at // 16]), at % 16, 0, 5] = 0
    t[0, int(b.tab[0, at // 16]), at % 16, 0, :] = float("nan")     # now its K
    out = attend(b, 0, q, 0.1, split)
    rows = torch.as_tensor(first + np.flatnonzero(~sees), device="cuda")
    assert torch.equal(out[rows], ref[rows])
    rows = torch.as_tensor(first + np.flatnonzero(sees), device="cuda")
    assert torch.isnan(out[rows].float()).all()


@pytest.mark.parametrize("new", [3, 7, 60])
@pytest.mark.parametrize("d", [64, 128])
def test_odd_values_beside_missing_blocks_reach_every_row(d, new):
    """A block outside the pool in the middle of what every row sees: infinities of the
    tokens around it count as they do elsewhere."""
    geom = Geometry("chunkodd2", 1, 1, d, 4, "bfloat16")
    b = Batch(geom, LM, [new], [300], 19)
    t = b.layer_view(0)
    b.tab[0, 20] = b.blocks + 3
    b.upload()
    q = queries(b, 4, 19)
    ref = attend(b, 0, q, 0.1)
    check_attention(b, 0, q, 0.1, ref)
    t[1, int(b.tab[0, 19]), 2, 0, 7] = float("inf")         # tokens 78 and 85
    t[1, int(b.tab[0, 21]), 1, 0, 9] = float("-inf")
    out = attend(b, 0, q, 0.1)
    assert (out[:, :, 7].float() == float("inf")).all()
    assert (out[:, :, 9].float() == float("-inf")).all()
    rest = [i for i in range(d) if i not in (7, 9)]
    assert torch.equal(out[:, :, rest], ref[:, :, rest])


@pytest.mark.parametrize("split", [0, 64])
def test_infinite_scores(split):
    """A score of -inf weighs nothing, one of +inf makes its row NaN; all of -inf: zeros."""
    geom = Geometry("chunkinf", 1, 1, 64, 16, "bfloat16")
    b = Batch(geom, LM, [3, 2, 100], [200, 2, 150], 13)
    q = queries(b, 2, 13)
    q[:, 0, 3], q[:, 1, 3] = 1.0, -1.0
    t = b.layer_view(0)
    t[0, int(b.tab[0, 2]), 4, 0, 3] = float("-inf")
    for p in range(2):
        t[0, int(b.tab[1, 0]), p, 0, 3] = float("-inf")
    out = attend(b, 0, q, 0.2, split)
    a = int(b.off[0])
    assert torch.isfinite(out[a:a + 3, 0].float()).all()
    assert torch.isnan(out[a:a + 3, 1].float()).all()
    a = int(b.off[1])
    assert (out[a:a + 2, 0] == 0).all()
    assert torch.isnan(out[a:a + 2, 1].float()).all()
    assert torch.isfinite(out[int(b.off[2]):].float()).all()


def test_blocks_beyond_4_gib_into_the_pool():
    geom = Geometry("chunkfar", 1, 8, 128, 16, "bfloat16")
    for layout in (BM, LM):
        b = Batch(geom, layout, [20, 300], [1500, 700], 14, spare=140_000)
        q = queries(b, 32, 14)
        check_attention(b, 0, q, 0.09, attend(b, 0, q, 0.09))
        say(f"  {NAMES[layout]} ok")
        del b
        torch.cuda.empty_cache()


def test_many_requests():
    """More requests than one round of the search for a tile's request looks at."""
    g = np.random.default_rng(15)
    for n in (65, 700, 5000):
        geom = Geometry("chunkmany", 1, 1, 64, 16, "bfloat16")
        new = g.integers(0, 4, n)
        b = Batch(geom, BM, new, new + g.integers(0, 30, n), 15)
        say(f"chunk attention over {n} requests, {b.n_tokens} new tokens")
        q = queries(b, 2, 15)
        out = attend(b, 0, q, 0.1)
        view = b.layer_view(0)
        pick = g.choice(n, 40, replace=False)
        for r in pick:
            if b.new[r] == 0:
                continue
            one = Batch.__new__(Batch)
            one.__dict__.update(b.__dict__)
            one.new, one.total, one.tab = b.new[r:r + 1], b.total[r:r + 1], b.tab[r:r + 1]
            one.off, one.max_len = b.off[r:r + 2], b.max_len
            check_attention(one, 0, q, 0.1, out)
        assert torch.isfinite(out[:int(b.off[-1])].float()).all()


def test_same_result_on_another_stream_and_for_two_calls_at_once():
    geom = Geometry("chunkstream", 2, 2, 128, 16, "bfloat16")
    b = Batch(geom, BM, [50, 3], [3000, 4000], 16)
    q = queries(b, 8, 16)
    ref = [attend(b, l, q, 0.09, 512) for l in range(2)]
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, 2, 8, 2, 128, b.max_new, b.max_len, 512)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(r) for r in ref]
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(10):
        for l in range(2):
            fk.flowkv_chunk_attention(b.pool, l, q, *b.args(), b.max_new, b.max_len, 0.09, outs[l],
                                      ws[l], 512, stream=streams[l])
    torch.cuda.synchronize()
    for l in range(2):
        assert torch.equal(outs[l], ref[l])


def test_replayed_graph_follows_the_lengths_on_the_device():
    """Captured once, replayed with other lengths, offsets and tables in the same memory."""
    geom = Geometry("chunkgraph", 2, 2, 64, 16, "bfloat16")
    b = Batch(geom, LM, [40, 1, 9], [900, 500, 9], 17)
    q = queries(b, 4, 17)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    need = fk.flowkv_chunk_attention_workspace(50, 3, 4, 2, 64, 50, 1000, 128)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call():
        fk.flowkv_chunk_attention(b.pool, 1, q, b.offsets, b.tables, b.lens, 50, 1000, 0.1, out,
                                  ws, 128)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, total in (([40, 1, 9], [900, 500, 9]), ([0, 30, 20], [900, 60, 20]),
                       ([1, 1, 1], [2, 512, 9]), ([10, 10, 30], [900, 512, 30])):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        out.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(b, 1, q, 0.1, out, max_seq=1000)
        assert torch.isnan(out[int(b.off[-1]):].float()).all()


LONGEST = 400_000       # a length that the caller has to allow for, whatever the batch holds


def pieces_bytes(b, hk, G, d):
    """Workspace of a call whose tiles are cut by the lengths on the device."""
    rows, pieces = (256, 256) if d == 128 else (128, 512)
    return (pieces * rows * (d + 2) + b.n_tokens * G // rows + len(b.new) + 1) * 4


MIXED = [  # as BATCHES, with more than 32 rows of a request in every shape
    ([200], [200]), ([31, 64, 1], [31, 500, 129]), ([128, 127, 129], [128, 400, 129]),
    ([1, 260, 1, 70], [1000, 260, 63, 900]), ([0, 3, 0, 40, 0, 0], [9, 40, 0, 40, 700, 0]),
    ([700], [1400]), ([40] * 12, [40 + 150 * i for i in range(12)]), ([50], [9000]),
    ([1] * 30 + [90], [333 * i + 1 for i in range(30)] + [300]),
]


@pytest.mark.parametrize("batch", range(len(MIXED)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_pieces_by_the_lengths_against_the_formula(shape, batch):
    L, hk, d, bs, G = SHAPES[shape]
    seed = 29 * shape + batch
    layout = (BM, LM)[seed % 2]
    b = Batch(Geometry(f"pieces{shape}", L, hk, d, bs, "bfloat16"), layout, *MIXED[batch], seed,
              pad=(seed % 3, seed % 4))
    say(f"pieces {NAMES[layout]} shape {SHAPES[shape]} new {b.new.tolist()} of {b.total.tolist()}")
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(b.new), hk * G, hk, d, b.max_new,
                                               LONGEST)
    rows = 256 if d == 128 else 128
    tiles = hk * min(len(b.new) * -(-b.max_new * G // rows), b.n_tokens * G // rows + len(b.new))
    assert need == (pieces_bytes(b, hk, G, d) if tiles < 256 else 0)    # (whole tiles from there)
    q = queries(b, hk * G, seed, lead=(0, 8, 2 * d)[seed % 3])
    out = attend(b, L - 1, q, d ** -0.5, max_len=LONGEST)
    rel, worst = check_attention(b, L - 1, q, d ** -0.5, out, max_seq=LONGEST)
    say(f"  relative error {rel:.2e}, worst error / bound {worst:.2f}")
    inside = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
    inside[int(b.off[0]):int(b.off[-1])] = True
    assert (out[~inside] == 7).all(), "a row of no request was written"


@pytest.mark.parametrize("hk,d,G,n_req,top", [(4, 64, 2, 130, 40), (8, 64, 2, 20, 120),
                                              (8, 128, 4, 20, 64), (2, 128, 8, 150, 30),
                                              (8, 128, 4, 60, 100), (1, 64, 5, 400, 17)])
@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_tiles_in_the_order_of_the_lengths(layout, hk, d, G, n_req, top):
    """More tiles than CUs, of requests of every length, some with no token."""
    g = np.random.default_rng(n_req + d)
    new = g.integers(0, top + 1, n_req)
    new[n_req // 2] = top
    b = Batch(Geometry("order", 1, hk, d, 16, "bfloat16"), layout, new,
              new + g.integers(0, 600, n_req), 23)
    say(f"order {NAMES[layout]} {n_req} requests of up to {top}, {hk} x {d}, group {G}")
    q = queries(b, hk * G, 23)
    out = attend(b, 0, q, d ** -0.5)
    check_attention(b, 0, q, d ** -0.5, out)
    assert torch.equal(attend(b, 0, q, d ** -0.5, split=1 << 20), out)     # one piece a tile too


@pytest.mark.parametrize("rule", [
    lambda: [test_rows_that_see_nothing_are_zero(d, 0) for d in (64, 128)],
    lambda: [test_blocks_outside_the_pool_contribute_nothing(0)],
    lambda: [test_odd_values_reach_only_the_rows_that_see_them(d, 0, bad)
             for d in (64, 128) for bad in (float("nan"), float("inf"), float("-inf"))],
    lambda: [test_odd_values_beside_missing_blocks_reach_every_row(d, 60) for d in (64, 128)],
    lambda: [test_infinite_scores(0)],
    lambda: [test_large_scores_and_rising_maxima(0)],
], ids=["nothing", "missing", "odd", "odd-missing", "infinite", "large"])
def test_pieces_keep_the_rules(rule, monkeypatch):
    plain = attend
    monkeypatch.setitem(globals(), "attend",
                        lambda b, layer, q, scale, split=0, out=None, max_len=None, stream=None:
                        plain(b, layer, q, scale, 0, out, LONGEST, stream))
    rule()


def test_pieces_in_a_replayed_graph_and_on_two_streams():
    """One capture, other lengths in the same memory; two calls at once, a workspace each."""
    geom = Geometry("piecesgraph", 2, 2, 128, 16, "bfloat16")
    b = Batch(geom, LM, [40, 1, 9], [900, 500, 9], 17)
    q = queries(b, 8, 17)
    out = [torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    need = fk.flowkv_chunk_attention_workspace(50, 3, 8, 2, 128, 50, LONGEST)
    assert need == pieces_bytes(b, 2, 4, 128)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(l=1, stream=None):
        fk.flowkv_chunk_attention(b.pool, l, q, b.offsets, b.tables, b.lens, 50, LONGEST, 0.1,
                                  out[l], ws[l], stream=stream)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for new, total in (([40, 1, 9], [900, 500, 9]), ([0, 30, 20], [900, 60, 20]),
                       ([1, 1, 1], [2, 512, 9]), ([10, 10, 30], [900, 512, 30])):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        for l in range(2):
            out[l].fill_(float("nan"))
            ws[l].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(b, 1, q, 0.1, out[1], max_seq=LONGEST)
        assert torch.isnan(out[1][int(b.off[-1]):].float()).all()
        once = out[1].clone()
        for _ in range(5):
            for l in range(2):
                call(l, streams[l])
        torch.cuda.synchronize()
        check_attention(b, 0, q, 0.1, out[0], max_seq=LONGEST)
        assert torch.equal(out[1][:int(b.off[-1])], once[:int(b.off[-1])])


@pytest.mark.parametrize("max_len,split", [(LONGEST, 0), (4000, 128), (4000, 0)])
def test_two_graphs_share_a_workspace(max_len, split):
    """Replayed in turn on one stream, with eager work between: each call writes all of the
    workspace that it reads."""
    geom = Geometry("sharedws", 1, 2, 128, 16, "bfloat16")
    runs, need = [], 0
    for k, (new, total) in enumerate((([90, 1, 7], [300, 2000, 7]), ([2, 64], [3900, 64]))):
        b = Batch(geom, BM, new, total, 40 + k)
        q = queries(b, 8, 40 + k)
        runs.append((b, q, torch.zeros_like(q)))
        need = max(need, fk.flowkv_chunk_attention_workspace(b.n_tokens, len(new), 8, 2, 128,
                                                             b.max_new, max_len, split))
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def call(k):
        b, q, out = runs[k]
        fk.flowkv_chunk_attention(b.pool, 0, q, *b.args(), b.max_new, max_len, 0.09, out, ws, split)

    graphs, want = [], []
    for k in range(2):
        call(k)
        torch.cuda.synchronize()
        check_attention(runs[k][0], 0, runs[k][1], 0.09, runs[k][2], max_seq=max_len)
        want.append(runs[k][2].clone())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            call(k)
    for i in range(6):
        k = i % 2
        runs[k][2].fill_(float("nan"))
        graphs[k].replay()
        torch.cuda.synchronize()
        assert torch.equal(runs[k][2], want[k])
        if i % 3 == 2:
            ws.fill_(255)


def test_refused_by_the_binding():
    geom = Geometry("chunkref", 2, 2, 64, 16, "bfloat16")
    b = Batch(geom, BM, [4, 3], [40, 30], 18)
    q = queries(b, 4, 18)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")

    def call(q=q, out=out, offsets=b.offsets, tables=b.tables, lens=b.lens, ws=None, split=0,
             layer=0, max_len=40, scale=0.1, pool=b.pool):
        fk.flowkv_chunk_attention(pool, layer, q, offsets, tables, lens, 4, max_len, scale, out,
                                  ws, split)

    call()
    for bad in (dict(q=q.float()), dict(out=out.float()), dict(out=out[:, :2]), dict(q=q[0]),
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(lens=b.lens.long()),
                dict(offsets=b.offsets[:-1]), dict(tables=b.tables[:1]), dict(lens=b.lens.cpu()),
                dict(q=torch.zeros((7, 4, 128), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    half = fk.KVPool(BM, torch.zeros((4, 1, 2, 16, 2, 64), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        call(pool=half)
    for code, bad in ((fk.EINVAL, dict(layer=2)), (fk.EINVAL, dict(scale=float("nan"))),
                      (fk.EINVAL, dict(split=100)), (fk.EINVAL, dict(q=q[:, :3], out=out[:, :3])),
                      (fk.EINVAL, dict(max_len=-1)), (fk.EINVAL, dict(split=64, max_len=100)),
                      (fk.ECAP, dict(split=64, max_len=100,
                                     ws=torch.empty(100, dtype=torch.uint8, device="cuda")))):
        if "out" in bad:
            bad["out"] = bad["out"].contiguous()
        with pytest.raises(fk.FlowKVError) as e:
            call(**bad)
        assert e.value.code == code, bad
    torch.cuda.synchronize()
