"""Attention through a window with first tokens that stay visible (GPU) against its formula in
64 bits, with the bounds that tests/span_batch.py derives."""

import sys

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch
from tests.span_batch import check_span, half_step, visible
from tests.test_chunk_attention_gpu import BATCHES, LONGEST, MIXED, SHAPES

pytestmark = pytest.mark.gpu
NAMES = {LM: "layer", BM: "block"}
ALL = 2**31 - 1
WINDOWS = [(1, 0), (3, 1), (17, 4), (64, 0), (100, 70), (33, 300), (1000, 4), (5, 64), (ALL, 0),
           (129, 1), (700, 31)]


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def queries(b, q_heads, seed, gain=2.0, lead=0):
    d = b.geom.head_dim
    x = torch.randn((b.n_tokens, lead + q_heads * d),
                    generator=torch.Generator("cuda").manual_seed(seed + 7), device="cuda")
    return (gain * x).to(b.pool.dtype)[:, lead:].unflatten(1, (q_heads, d))


def attend(b, layer, q, scale, window, sinks, split=0, max_len=None, max_new=None, stream=None):
    """The call; nothing behind its workspace and no row of no request changes."""
    max_len = b.max_len if max_len is None else max_len
    max_new = b.max_new if max_new is None else max_new
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    need = fk.flowkv_window_attention_workspace(b.n_tokens, len(b.new), q.shape[1],
                                                b.geom.kv_heads, b.geom.head_dim, max_new,
                                                max_len, window, sinks, split)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    fk.flowkv_window_attention(b.pool, layer, q, *b.args(), max_new, max_len, window, sinks, scale,
                               out, ws[:need] if need else None, split, stream=stream)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all(), "written behind the workspace"
    inside = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
    inside[int(b.off[0]):int(b.off[-1])] = True
    assert (out[~inside] == 7).all(), "a row of no request was written"
    return out


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_formula(shape, batch, dtype):
    L, hk, d, bs, G = SHAPES[shape]
    seed = 31 * shape + batch + 500 * (dtype == "float16")
    layout = (BM, LM)[seed % 2]
    split = [0, 64, 128, 0, 1024, 2048, 4096][seed % 7]
    b = Batch(Geometry(f"win{shape}", L, hk, d, bs, dtype), layout, *BATCHES[batch], seed,
              pad=(seed % 3, seed % 4))
    q = queries(b, hk * G, seed, lead=(0, 8, 2 * d)[seed % 3])
    for window, sinks in (WINDOWS[seed % 11], WINDOWS[(seed + 4) % 11]):
        say(f"window {window} + {sinks} {dtype} {NAMES[layout]} shape {SHAPES[shape]} new "
            f"{b.new.tolist()} of {b.total.tolist()} split {split}")
        out = attend(b, L - 1, q, d ** -0.5, window, sinks, split)
        rel, worst = check_span(b, L - 1, q, d ** -0.5, out, window, sinks)
        say(f"  relative error {rel:.2e}, worst error / bound {worst:.2f}")


@pytest.mark.parametrize("batch", range(len(MIXED)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_pieces_by_the_lengths_and_more_rows_than_max_new(shape, batch):
    L, hk, d, bs, G = SHAPES[shape]
    seed = 29 * shape + batch
    layout = (BM, LM)[seed % 2]
    b = Batch(Geometry(f"winp{shape}", L, hk, d, bs, ("bfloat16", "float16")[batch % 2]), layout,
              *MIXED[batch], seed, pad=(seed % 3, seed % 4))
    q = queries(b, hk * G, seed)
    for window, sinks in ((2**18, 5), (64 + seed, seed % 70)):
        say(f"pieces: window {window} + {sinks} {NAMES[layout]} shape {SHAPES[shape]} new "
            f"{b.new.tolist()} of {b.total.tolist()}")
        out = attend(b, L - 1, q, d ** -0.5, window, sinks, max_len=LONGEST)
        check_span(b, L - 1, q, d ** -0.5, out, window, sinks, max_seq=LONGEST)
        for split in (0, 64):
            out = attend(b, L - 1, q, d ** -0.5, window, sinks, split, max_new=batch % 3)
            check_span(b, L - 1, q, d ** -0.5, out, window, sinks)


@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
@pytest.mark.parametrize("new,total", [(2000, 9000), (3, 20000), (1, 20000)])
def test_llama8b_geometry(layout, new, total):
    b = Batch(Geometry("win8b", 4, 8, 128, 16, "bfloat16"), layout, [new, 1, 40],
              [total, 777, 2500], 3)
    q = queries(b, 32, 3)
    for window, sinks in ((4096, 4), (1024, 128)):
        check_span(b, 2, q, 128 ** -0.5, attend(b, 2, q, 128 ** -0.5, window, sinks), window, sinks)


@pytest.mark.parametrize("hk,d,G,n_req,top", [(4, 64, 2, 130, 40), (8, 128, 4, 60, 100),
                                              (1, 64, 5, 400, 17)])
def test_tiles_in_the_order_of_the_lengths(hk, d, G, n_req, top):
    g = np.random.default_rng(n_req + d)
    new = g.integers(0, top + 1, n_req)
    new[n_req // 2] = top
    b = Batch(Geometry("winorder", 1, hk, d, 16, "bfloat16"), BM, new,
              new + g.integers(0, 600, n_req), 23)
    q = queries(b, hk * G, 23)
    for window, sinks in ((300, 4), (20, 100)):
        check_span(b, 0, q, d ** -0.5, attend(b, 0, q, d ** -0.5, window, sinks), window, sinks)


TAILS = [  # (KV heads, query heads per KV head, new tokens, tokens in all): from 256 tiles of 256 rows on
    (8, 8, [1030], [4000]),                             # 33 tiles a head: one behind a round
    (8, 8, [700, 40, 300, 1], [3000, 5000, 300, 2900]), (8, 8, [2040], [2600]),     # 64: no tail
    (16, 4, [1500, 9], [1500, 8000]), (5, 16, [900, 0, 100], [2500, 9, 4000]),
    (2, 40, [600, 333], [3100, 2400]), (8, 8, [200] * 9, [2000 + 300 * i for i in range(9)]),
]


def tail_bytes(tiles):
    """Workspace of 256 pieces of 256 rows, and of the pieces before each tile slot."""
    return (256 * 256 * 130 + tiles + 1) * 4


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(TAILS)))
def test_whole_tiles_and_a_tail_in_pieces(case, dtype):
    hk, G, new, total = TAILS[case]
    b = Batch(Geometry("wintail", 1, hk, 128, 16, dtype), (BM, LM)[case % 2], new, total, 40 + case,
              pad=(case % 3, 2 * case))
    q = queries(b, hk * G, 40 + case)
    for window, sinks in ((2**18, 3), (2300, 40)):
        slots = b.n_tokens * G // 256 + len(new)
        assert fk.flowkv_window_attention_workspace(b.n_tokens, len(new), hk * G, hk, 128, b.max_new,
                                                    8000, window, sinks) == tail_bytes(slots)
        say(f"tail {hk} x {G} new {new} of {total} window {window} + {sinks} {dtype}")
        out = attend(b, 0, q, 128 ** -0.5, window, sinks, max_len=8000)
        check_span(b, 0, q, 128 ** -0.5, out, window, sinks, max_seq=8000)
        # rows that the host was not told of: whole tiles
        out = attend(b, 0, q, 128 ** -0.5, window, sinks, max_len=8000, max_new=b.max_new - 9)
        check_span(b, 0, q, 128 ** -0.5, out, window, sinks, max_seq=8000)


def test_a_tail_keeps_the_rules():
    """NaN and infinities that no row sees, missing blocks, rows that see nothing."""
    b = Batch(Geometry("wintailodd", 1, 8, 128, 16, "bfloat16"), BM, [1030, 60], [4000, 40], 47)
    q = queries(b, 64, 47)
    window, sinks = 2500, 5
    ref = attend(b, 0, q, 0.09, window, sinks, max_len=8000)
    check_span(b, 0, q, 0.09, ref, window, sinks, max_seq=8000)
    view, base = b.layer_view(0), 4000 - 1030
    for p in range(sinks, base - window + 1):
        view[:, int(b.tab[0, p // 16]), p % 16] = float("nan")
    assert torch.equal(attend(b, 0, q, 0.09, window, sinks, max_len=8000), ref)
    at = base - window + 300                    # (seen by the first 300 rows)
    view[1, int(b.tab[0, at // 16]), at % 16, :, 7] = float("inf")
    out = attend(b, 0, q, 0.09, window, sinks, max_len=8000)
    assert (out[:300, :, 7].float() == float("inf")).all()
    assert torch.equal(out[300:], ref[300:])
    b.tab[0, 100:140] = -1
    b.upload()
    view[1][view[1] == float("inf")] = 0
    check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, window, sinks, max_len=8000), window, sinks,
               max_seq=8000)


def test_a_tail_in_a_replayed_graph_and_on_two_streams():
    b = Batch(Geometry("wintailgraph", 2, 8, 128, 16, "bfloat16"), BM, [1030, 60], [4000, 3000], 48)
    q = queries(b, 64, 48)
    ref = [attend(b, l, q, 0.09, 2500, 4, max_len=8000) for l in range(2)]
    need = tail_bytes(1090 * 8 // 256 + 2)
    out = [torch.zeros_like(r) for r in ref]
    ws = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def call(l=1, stream=None):
        fk.flowkv_window_attention(b.pool, l, q, *b.args(), 1090, 8000, 2500, 4, 0.09, out[l], ws[l],
                                   stream=stream)
    for i in range(5):
        for l in range(2):
            call(l, streams[l])
    torch.cuda.synchronize()
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, total in (([1030, 60], [4000, 3000]), ([0, 1024], [9, 4000]), ([545, 545], [700, 545]),
                       ([3, 2], [3000, 3999])):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        out[1].fill_(float("nan"))
        ws[1].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check_span(b, 1, q, 0.09, out[1], 2500, 4, max_seq=8000)
        assert torch.isnan(out[1][int(b.off[-1]):].float()).all()


@pytest.mark.parametrize("split", [0, 64, 2048])
@pytest.mark.parametrize("new,total", [([3], [700]), ([200, 1, 40], [700, 64, 300]),
                                       ([700], [700]), ([1] * 30, [50 * i + 1 for i in range(30)])])
def test_a_window_that_hides_nothing_gives_the_same_bits(new, total, split):
    b = Batch(Geometry("winall", 1, 2, 128, 16, "bfloat16"), BM, new, total, 24)
    q = queries(b, 8, 24)
    want = torch.empty_like(q)
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(new), 8, 2, 128, b.max_new, b.max_len,
                                               split)
    ws = torch.empty(max(need, 4), dtype=torch.uint8, device="cuda")
    fk.flowkv_chunk_attention(b.pool, 0, q, *b.args(), b.max_new, b.max_len, 0.09, want, ws, split)
    for window, sinks in ((ALL, 0), (ALL, ALL), (1, ALL), (b.max_len, 0), (1, b.max_len)):
        assert torch.equal(attend(b, 0, q, 0.09, window, sinks, split), want), (window, sinks)


RUN = 32


@pytest.mark.parametrize("split", [0, 64, 192, 2048])
@pytest.mark.parametrize("d,hk,G,layout,bs", [(128, 2, 4, BM, 16), (64, 1, 8, LM, 7)])
def test_every_seen_token_counts_once(d, hk, G, layout, bs, split):
    """Queries of zero: every weight is 1, the sum the number n of tokens seen, both exact.  V is
    1 in dim c of the tokens of class c, a run of 32, and 0 elsewhere: out[c] is the bf16
    nearest to (tokens of class c seen) / n, up to two roundings of float32.  One token of a
    whole class more or less is 2^-5 of it, eight times half a step."""
    for i, (new, total) in enumerate([([3], [9000]), ([1, 8], [20000, 8191]), ([300], [20000]),
                                      ([130, 2, 61], [4097, 12288, 9999]), ([2100], [2100])]):
        b = Batch(Geometry("wincounts", 1, hk, d, bs, "bfloat16"), layout, new, total, 100 + i)
        q = torch.zeros((b.n_tokens, hk * G, d), dtype=torch.bfloat16, device="cuda")
        for window, sinks in ((1500, 4), (333, 100), (5000, 2000)):
            see = [visible(T, m, T, window, sinks) for m, T in zip(new, total)]
            for first in range(0, b.max_len, d * RUN):
                view = b.layer_view(0)
                view[0], view[1] = 0.5, 0
                want = []
                for r, (m, T) in enumerate(zip(new, total)):
                    p = np.arange(first, min(first + d * RUN, T))
                    if p.size:
                        at = [torch.as_tensor(x, device="cuda")
                              for x in (b.tab[r, p // bs].astype(np.int64), p % bs,
                                        (p - first) // RUN)]
                        view[1][at[0], at[1], :, at[2]] = 1
                    s = torch.zeros((m, d * RUN), device="cuda", dtype=torch.float64)
                    s[:, :max(0, min(T - first, d * RUN))] = see[r][:, first:first + d * RUN]
                    want.append(s.view(m, d, RUN).sum(2) / see[r].sum(1, keepdim=True))
                want = torch.cat(want)[:, None]
                err = (attend(b, 0, q, 0.3, window, sinks, split).double() - want).abs()
                assert (err <= (half_step(torch.bfloat16) + 2.0 ** -23) * want).all(), \
                    (window, sinks, first)
        say(f"new {new} of {total} split {split} ok")


@pytest.mark.parametrize("d,G,dtype", [(128, 4, "bfloat16"), (64, 2, "float16"), (64, 40, "bfloat16")])
@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("new,total", [([1], [900]), ([7, 1], [900, 333]), ([200, 50], [900, 700])])
def test_blocks_that_no_row_sees_are_not_looked_up(new, total, split, d, G, dtype):
    """Freed blocks in the list, and NaN and infinities in every token that no row sees."""
    for window, sinks in ((100, 4), (257, 0), (64, 33)):
        b = Batch(Geometry("winfree", 1, 2, d, 16, dtype), LM, new, total, 25)
        q = queries(b, 2 * G, 25)
        ref = attend(b, 0, q, 0.09, window, sinks, split)
        check_span(b, 0, q, 0.09, ref, window, sinks)
        view = b.layer_view(0)
        for r, (m, T) in enumerate(zip(new, total)):
            low = max(sinks, T - m - window + 1)
            for p in list(range(sinks, low)) + list(range(T, -(-T // 16) * 16)):
                view[:, int(b.tab[r, p // 16]), p % 16] = [float("nan"), float("inf")][p % 2]
        assert torch.equal(attend(b, 0, q, 0.09, window, sinks, split), ref)
        bad = [-1, b.blocks, 2**31 - 1, -2**31, 3]
        for r, (m, T) in enumerate(zip(new, total)):
            low = max(sinks, T - m - window + 1)
            for j in range(-(-sinks // 16), low // 16):
                b.tab[r, j] = bad[j % 5]
        b.upload()
        assert torch.equal(attend(b, 0, q, 0.09, window, sinks, split), ref)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("d,new,dtype", [(64, 150, "bfloat16"), (128, 150, "float16"),
                                         (128, 5, "bfloat16"), (64, 3, "float16")])
def test_odd_values_reach_only_the_rows_that_see_them(d, new, dtype, split, bad):
    """V, then K, of one token holds bad values: among the first tokens, before the window of
    some rows, among the new tokens; beside a missing block and not."""
    total, window, sinks = 510, 170, 6
    for missing in (False, True):
        b = Batch(Geometry("winodd", 1, 1, d, 16, dtype), BM, [new, 9], [total, 30], 12)
        if missing:
            b.tab[0, 400 // 16] = -1
            b.upload()
        q = queries(b, 4, 12)
        ref = attend(b, 0, q, 0.1, window, sinks, split)
        view = b.layer_view(0)
        base = total - new
        for at in (2, sinks, base - window + 1, base - window // 2, 395, base - window + 40,
                   total - 1, base + new // 2):
            see = (visible(total, new, total, window, sinks)[:, at]).cpu().numpy()
            first = int(b.off[0])
            unseen = torch.as_tensor(first + np.flatnonzero(~see), device="cuda")
            seen = torch.as_tensor(first + np.flatnonzero(see), device="cuda")
            slot = int(b.tab[0, at // 16]), at % 16, 0
            if slot[0] < 0:
                continue
            keep = view[:, slot[0], slot[1], 0].clone()
            view[1][slot + (5,)] = bad
            out = attend(b, 0, q, 0.1, window, sinks, split)
            assert torch.equal(out[unseen], ref[unseen]), at
            hit = out[seen][:, :, 5].float()
            assert (torch.isnan(hit) if bad != bad else hit == bad).all(), at
            rest = [i for i in range(d) if i != 5]
            assert torch.equal(out[seen][:, :, rest], ref[seen][:, :, rest]), at
            view[:, slot[0], slot[1], 0] = keep
            view[0][slot] = float("nan")
            out = attend(b, 0, q, 0.1, window, sinks, split)
            assert torch.equal(out[unseen], ref[unseen]), at
            assert torch.isnan(out[seen].float()).all(), at
            assert torch.equal(out[int(b.off[1]):], ref[int(b.off[1]):])
            view[:, slot[0], slot[1], 0] = keep


@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("d,dtype", [(64, "float16"), (128, "bfloat16")])
def test_rows_that_see_nothing_are_zero(d, dtype, split):
    """Positions below 0, lengths of 0 and below, windows whose blocks are all missing."""
    b = Batch(Geometry("winnone", 1, 2, d, 16, dtype), BM, [5, 3, 200, 150, 2], [2, 0, 130, 150, 90],
              9)
    b.total[1] = -4
    b.tab[4, 3:] = -1
    b.upload()
    q = queries(b, 4, 9)
    for window, sinks in ((1, 0), (20, 0), (20, 3)):
        out = attend(b, 0, q, 0.1, window, sinks, split, max_len=150)
        for r in (0, 1, 2):
            first = int(b.off[r])
            none = int(min(b.new[r], b.new[r] - max(b.total[r], 0)))
            assert (out[first:first + none] == 0).all(), f"request {r}"
        check_span(b, 0, q, 0.1, out, window, sinks, max_seq=150)
        if sinks == 0:
            assert (out[int(b.off[4]):] == 0).all()


def test_lengths_past_the_table_and_past_max_seq_len():
    b = Batch(Geometry("winclamp", 1, 1, 128, 16, "bfloat16"), BM, [30, 4], [500, 200], 11)
    b.total[1] = 505        # 32 blocks listed (both rows have the widest's)
    b.tab[1, :] = b.tab[0, :]
    b.upload()
    q = queries(b, 4, 11)
    for window, sinks in ((100, 4), (20, 0), (10, 500)):
        out = attend(b, 0, q, 0.09, window, sinks, max_len=480)
        check_span(b, 0, q, 0.09, out, window, sinks, max_seq=480)
    b.total[0] += 100       # past the 32 listed blocks
    b.upload()
    for window, sinks in ((130, 4), (20, 0), (10, 600)):
        out = attend(b, 0, q, 0.09, window, sinks)
        check_span(b, 0, q, 0.09, out, window, sinks, max_seq=b.max_len)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("split", [64, 192, 0])
def test_large_scores_and_rising_maxima(split, dtype):
    b = Batch(Geometry("winbig", 1, 1, 64, 16, dtype), BM, [40, 5], [600, 333], 5)
    t = b.layer_view(0)
    for r in range(2):
        for p in range(int(b.total[r])):
            t[0, b.tab[r, p // 16], p % 16] *= p / 60
    q = queries(b, 4, 5, gain=8.0)
    check_span(b, 0, q, 1.0, attend(b, 0, q, 1.0, 250, 9, split), 250, 9)


def test_small_weights_of_many_fp16_tokens_add_up():
    """One token 2^24.9 above each of 200,000 others, which together are 0.6% of the sum: fp16
    weights of 2^-24.9 would be rounded to 2^-24, 1.9 of each, ten times the bound."""
    b = Batch(Geometry("winsmall", 1, 1, 64, 16, "float16"), BM, [1, 40], [200_001, 200_040], 6)
    t = b.layer_view(0)
    t[0], t[1] = 0, 1
    q = torch.zeros((b.n_tokens, 2, 64), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1
    for r in range(2):
        t[0, int(b.tab[r, 0]), 3, 0, 0] = 24.9 * np.log(2)
        t[1, int(b.tab[r, 0]), 3, 0] = -1
    for window, sinks in ((ALL, 0), (150_000, 4)):
        check_span(b, 0, q, 1.0, attend(b, 0, q, 1.0, window, sinks), window, sinks)


def test_blocks_beyond_4_gib_into_the_pool():
    for layout in (BM, LM):
        b = Batch(Geometry("winfar", 1, 8, 128, 16, "bfloat16"), layout, [20, 300], [1500, 700], 14,
                  spare=140_000)
        q = queries(b, 32, 14)
        check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, 200, 5), 200, 5)
        del b
        torch.cuda.empty_cache()


def test_many_requests():
    g = np.random.default_rng(15)
    for n in (65, 700, 5000):
        new = g.integers(0, 4, n)
        b = Batch(Geometry("winmany", 1, 1, 64, 16, "bfloat16"), BM, new, new + g.integers(0, 30, n),
                  15)
        q = queries(b, 2, 15)
        check_span(b, 0, q, 0.1, attend(b, 0, q, 0.1, 7, 2), 7, 2)


def test_padding_around_the_batch():
    b = Batch(Geometry("winpad", 1, 1, 128, 16, "bfloat16"), BM, [300, 40, 200, 17],
              [5000, 40, 900, 3000], 70, pad=(9000, 20001))
    q = queries(b, 8, 70)
    for max_len in (b.max_len, 32768, LONGEST):
        for window, sinks in ((2000, 4), (100000, 0)):
            out = attend(b, 0, q, 0.09, window, sinks, max_len=max_len)
            check_span(b, 0, q, 0.09, out, window, sinks, max_seq=max_len)


def test_two_calls_at_once_and_a_replayed_graph():
    b = Batch(Geometry("wingraph", 2, 2, 64, 16, "float16"), LM, [40, 1, 9], [900, 500, 9], 17)
    q = queries(b, 4, 17)
    ref = [attend(b, l, q, 0.09, 200, 3, 128) for l in range(2)]
    need = fk.flowkv_window_attention_workspace(50, 3, 4, 2, 64, 50, 1000, 200, 3, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [torch.zeros_like(r) for r in ref]
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()

    def call(l=1, stream=None):
        fk.flowkv_window_attention(b.pool, l, q, *b.args(), 50, 1000, 200, 3, 0.09, out[l], ws[l],
                                   128, stream=stream)
    for i in range(10):
        for l in range(2):
            call(l, streams[l])
    torch.cuda.synchronize()
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, total in (([40, 1, 9], [900, 500, 9]), ([0, 30, 20], [900, 60, 20]),
                       ([1, 1, 1], [2, 512, 9]), ([10, 10, 30], [900, 512, 30])):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        out[1].fill_(float("nan"))
        ws[1].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check_span(b, 1, q, 0.09, out[1], 200, 3, max_seq=1000)
        assert torch.isnan(out[1][int(b.off[-1]):].float()).all()


def test_the_binding_refuses_other_types():
    b = Batch(Geometry("winrefuse", 1, 2, 64, 16, "float16"), LM, [3], [9], 9)
    q = queries(b, 4, 6)
    for a in ((q.bfloat16(), torch.empty_like(q)), (q, torch.empty_like(q).bfloat16()),
              (q, torch.empty_like(q)[:2]), (q.flatten(1), q.flatten(1))):
        with pytest.raises(ValueError):
            fk.flowkv_window_attention(b.pool, 0, a[0], *b.args(), 3, 9, 5, 0, 0.1, a[1])
    with pytest.raises(fk.FlowKVError):
        fk.flowkv_window_attention(b.pool, 0, q, *b.args(), 3, 9, 0, 0, 0.1, torch.empty_like(q))
