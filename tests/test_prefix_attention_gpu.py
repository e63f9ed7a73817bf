"""Attention over shared prefixes (GPU) against the formula of attention over all of each
request's tokens in 64 bits, with the bounds that tests/span_batch.py derives."""

import sys

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.span_batch import check_span, group_batch
from tests.test_window_attention_gpu import queries

pytestmark = pytest.mark.gpu
NAMES = {LM: "layer", BM: "block"}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def sizes(b, bounds, prefixes):
    """max_new, max_group, max_own, max_prefix of a batch."""
    own = b.total.copy()
    for g, p in enumerate(prefixes):
        own[bounds[g]:bounds[g + 1]] -= p
    group = [int(b.new[bounds[g]:bounds[g + 1]].sum()) for g in range(len(prefixes))]
    return (b.max_new, max(group, default=0), int(max(own.max(initial=0), 0)),
            int(max(prefixes, default=0)))


def attend(b, layer, q, scale, bounds, prefixes, split=0, most=None, stream=None):
    """The call; nothing behind its workspace and no row of no request changes."""
    most = sizes(b, bounds, prefixes) if most is None else most
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    need = fk.flowkv_prefix_attention_workspace(b.n_tokens, len(b.new), q.shape[1],
                                                b.geom.kv_heads, b.geom.head_dim, len(prefixes),
                                                *most, split)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    fk.flowkv_prefix_attention(b.pool, layer, q, *b.args(), i32(bounds), i32(prefixes), *most, scale,
                               out, ws[:need] if need else None, split, stream=stream)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all(), "written behind the workspace"
    inside = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
    inside[int(b.off[0]):int(b.off[-1])] = True
    assert (out[~inside] == 7).all(), "a row of no request was written"
    return out


SHAPES = [  # (layers, KV heads, head_dim, block size, query heads per KV head)
    (2, 2, 128, 16, 4), (3, 1, 128, 16, 8), (2, 4, 64, 7, 2), (1, 2, 64, 16, 1), (2, 2, 128, 1, 3),
    (1, 1, 64, 100, 5), (1, 3, 64, 3, 16), (1, 1, 128, 5, 40),
]
GROUPS = [  # (prefix, [(new tokens, tokens behind the prefix)] of each request) of each group
    [(130, [(1, 1), (1, 9), (1, 30), (1, 2)])],
    [(1, [(1, 1), (1, 1)])],
    [(1000, [(1, 1 + 17 * i) for i in range(20)])],
    [(500, [(3, 5), (1, 200), (8, 8)]), (0, [(1, 40), (2, 2)]), (77, [(5, 60)])],
    [(2050, [(1, 5)] * 9), (64, [(1, 70)] * 3), (300, []), (65, [(0, 4), (0, 0), (2, 2)])],
    [(700, [(30, 40), (33, 33), (1, 900), (0, 10)]), (129, [(12, 12)] * 12)],
    [(300, [(200, 300), (150, 150)]), (40, [(70, 500)])],
    [(512, [(1, 600)] * 40), (100, [(1, 1)] * 70)],
    [(9000, [(2, 2), (1, 40)])],
    [(1500, [(6, 100 + 30 * i) for i in range(12)])] * 3,
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("groups", range(len(GROUPS)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_formula(shape, groups, dtype):
    L, hk, d, bs, G = SHAPES[shape]
    seed = 31 * shape + groups + 500 * (dtype == "float16")
    layout = (BM, LM)[seed % 2]
    b, bounds, prefixes = group_batch(Geometry(f"pre{shape}", L, hk, d, bs, dtype), layout,
                                      GROUPS[groups], seed, pad=(seed % 3, seed % 4))
    q = queries(b, hk * G, seed, lead=(0, 8, 2 * d)[seed % 3])
    for split in (0, [64, 128, 1024][seed % 3], 4096):
        say(f"prefix {dtype} {NAMES[layout]} shape {SHAPES[shape]} groups {groups} split {split}")
        out = attend(b, L - 1, q, d ** -0.5, bounds, prefixes, split)
        rel, worst = check_span(b, L - 1, q, d ** -0.5, out)
        say(f"  relative error {rel:.2e}, worst error / bound {worst:.2f}")


@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
@pytest.mark.parametrize("groups", [[(13000, [(1, 1 + 9 * i) for i in range(32)])],
                                    [(4000, [(1, 100 + 30 * i) for i in range(64)])],
                                    [(3000, [(4, 50)] * 10), (6000, [(1, 2000)] * 3)],
                                    [(2000, [(300, 300), (700, 700)])]])
def test_llama8b_geometry(layout, groups):
    b, bounds, prefixes = group_batch(Geometry("pre8b", 4, 8, 128, 16, "bfloat16"), layout, groups, 3)
    q = queries(b, 32, 3)
    check_span(b, 2, q, 128 ** -0.5, attend(b, 2, q, 128 ** -0.5, bounds, prefixes))


@pytest.mark.parametrize("hk,d,G,dtype,groups", [
    (8, 128, 4, "bfloat16", [(13000, [(1, 1 + i) for i in range(130)])]),
    (4, 64, 4, "float16", [(9000, [(4, 5 + i) for i in range(60)]),
                           (11000, [(3, 9 + 20 * i) for i in range(55)])]),
])
def test_prefixes_in_tiles_of_128_rows(hk, d, G, dtype, groups):
    """So much of prefixes that the library's rule takes wide tiles, in several splits."""
    b, bounds, prefixes = group_batch(Geometry("prewide", 1, hk, d, 16, dtype), BM, groups, 21)
    most = sizes(b, bounds, prefixes)
    rows, slot = b.n_tokens * G, hk * d * 4
    assert (rows // 32) * most[3] * slot >= 400 << 20
    q = queries(b, hk * G, 21)
    check_span(b, 0, q, d ** -0.5, attend(b, 0, q, d ** -0.5, bounds, prefixes))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_prompts_behind_prefixes_each_by_itself(dtype):
    """Many rows a request: whole tiles, and a tail of them in pieces."""
    groups = [(2100, [(300, 300), (130, 130), (64, 90)]), (3000, [(500, 500), (90, 90)])]
    b, bounds, prefixes = group_batch(Geometry("prealone", 1, 8, 128, 16, dtype), LM, groups, 22)
    q = queries(b, 64, 22)
    out = attend(b, 0, q, 0.09, bounds, prefixes)
    check_span(b, 0, q, 0.09, out)


@pytest.mark.parametrize("split", [0, 64, 1024, 4096])
def test_rows_past_the_sizes_that_the_host_tells(split):
    """max_new and max_group below the requests' own, and sizes far above them."""
    groups = [(700, [(30, 40), (3, 33), (1, 900)]), (129, [(12, 12)] * 12)]
    b, bounds, prefixes = group_batch(Geometry("prepast", 1, 2, 128, 16, "bfloat16"), BM, groups, 4,
                                      pad=(3, 500))
    q = queries(b, 8, 4)
    _, _, own, longest = sizes(b, bounds, prefixes)
    for most in ((0, 0, own, longest), (1, 4, own, longest), (1, 2000, own + 3000, longest + 9000),
                 (500, 700, 5000, 20000)):
        check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, bounds, prefixes, split, most))


@pytest.mark.parametrize("split", [0, 64, 4096])
def test_requests_of_no_group_and_new_tokens_within_a_prefix(split):
    groups = [(0, [(3, 90), (1, 5)]), (800, [(2, 5), (40, 41), (1, 1)]), (0, [(1, 300)] * 3)]
    b, bounds, prefixes = group_batch(Geometry("prenone", 1, 2, 64, 16, "float16"), LM, groups, 5)
    q = queries(b, 8, 5)
    some = bounds[1:3], prefixes[1:2]
    most = (40, 43, 300, 800)
    want = attend(b, 0, q, 0.1, bounds, prefixes, split, most)
    check_span(b, 0, q, 0.1, want)
    out = attend(b, 0, q, 0.1, *some, split, most)
    check_span(b, 0, q, 0.1, out)
    # the prefix taken to be longer than what was cached of it before: rows within it see less
    b.total[2:5] = [790, 801, 30]
    b.upload()
    check_span(b, 0, q, 0.1, attend(b, 0, q, 0.1, *some, split, most))
    b.total[2:5] = [0, -5, 800]
    b.upload()
    check_span(b, 0, q, 0.1, attend(b, 0, q, 0.1, *some, split, most))


def test_group_arrays_that_make_no_sense_touch_nothing_else():
    groups = [(600, [(1, 9)] * 9), (300, [(1, 50)] * 4)]
    b, bounds, prefixes = group_batch(Geometry("preodd", 1, 2, 64, 16, "bfloat16"), LM, groups, 6,
                                      pad=(5, 7))
    q = queries(b, 8, 6)
    most = (1, 9, 50, 600)
    for bad, lens in (([-5, 9, 100], [600, 300]), ([9, 0, 13], [600, 300]), ([0, 9, 13], [-3, 2**31 - 1]),
                      ([13, 13, 13], [600, 600]), ([2**31 - 1, -2**31, 5], [5, 5]),
                      ([0, 13, 13], [10**6, 0])):
        for split in (64, 4096):
            attend(b, 0, q, 0.1, bad, lens, split, most)
    attend(b, 0, q, 0.1, bounds, prefixes, 64, (1, 9, 3, 100))      # less than there is
    check_span(b, 0, q, 0.1, attend(b, 0, q, 0.1, bounds, prefixes, 64, most))


@pytest.mark.parametrize("split", [64, 1024, 4096])
def test_blocks_outside_the_pool_contribute_nothing(split):
    groups = [(400, [(1, 60), (2, 30), (70, 90)])]
    b, bounds, prefixes = group_batch(Geometry("prebad", 1, 2, 128, 16, "bfloat16"), LM, groups, 7)
    b.tab[:, [0, 5, 11]] = [-1, b.blocks, 2**31 - 1]
    b.tab[1, 26] = -1
    b.upload()
    q = queries(b, 8, 7)
    check_span(b, 0, q, 0.09, attend(b, 0, q, 0.09, bounds, prefixes, split))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("d,dtype,n,split", [(64, "bfloat16", 3, 64), (128, "float16", 3, 1024),
                                             (128, "bfloat16", 40, 64), (64, "float16", 40, 1024),
                                             (128, "bfloat16", 40, 4096), (64, "float16", 3, 4096)])
def test_odd_values_reach_only_the_rows_that_see_them(d, dtype, n, split, bad):
    """In the prefix: every row of the group, none of another.  Behind it: its request's.  In
    slots behind a prefix's part-filled last block, and behind the last token: none."""
    p = 333
    groups = [(p, [(2, 10 + i) for i in range(n)]), (100, [(1, 5)] * 3)]
    b, bounds, prefixes = group_batch(Geometry("preinf", 1, 1, d, 16, dtype), BM, groups, 8)
    q = queries(b, 4, 8)
    ref = attend(b, 0, q, 0.1, bounds, prefixes, split)
    check_span(b, 0, q, 0.1, ref)
    view = b.layer_view(0)
    for r in range(len(b.new)):
        T = int(b.total[r])
        if T % 16:
            view[:, int(b.tab[r, T // 16]), T % 16:] = bad
    assert torch.equal(attend(b, 0, q, 0.1, bounds, prefixes, split), ref)
    last = 2 * n                                        # rows of the first group
    for at, rows in ((0, slice(0, last)), (200, slice(0, last)), (p - 1, slice(0, last)),
                     (p, slice(0, 2)), (p + 9, slice(1, 2))):
        where = [(int(b.tab[r, at // 16]), at % 16) for r in range(n if at < p else 1)]
        keep = [view[:, x, y].clone() for x, y in where]
        for x, y in where:
            view[1, x, y, 0, 5] = bad
        out = attend(b, 0, q, 0.1, bounds, prefixes, split)
        sees = torch.zeros(b.n_tokens, dtype=torch.bool, device="cuda")
        sees[rows] = True
        hit = out[sees][:, :, 5].float()
        assert (torch.isnan(hit) if bad != bad else hit == bad).all(), at
        assert torch.equal(out[~sees], ref[~sees]), at
        rest = [i for i in range(d) if i != 5]
        assert torch.equal(out[:, :, rest], ref[:, :, rest]), at
        for (x, y), z in zip(where, keep):
            view[:, x, y] = z
            view[0, x, y] = float("nan")
        out = attend(b, 0, q, 0.1, bounds, prefixes, split)
        assert torch.isnan(out[sees].float()).all() and torch.equal(out[~sees], ref[~sees]), at
        for (x, y), z in zip(where, keep):
            view[:, x, y] = z


@pytest.mark.parametrize("split", [64, 0, 4096])
def test_large_scores_and_rising_maxima(split):
    groups = [(600, [(1, 40), (5, 30)] * 6)]
    b, bounds, prefixes = group_batch(Geometry("prebig", 1, 1, 64, 16, "float16"), BM, groups, 9)
    t = b.layer_view(0)
    for j, blk in enumerate(b.tab[0]):
        if blk >= 0:
            t[0, int(blk)] *= j / 4
    for r in range(1, 12):      # (the copies of the prefix's last block)
        t[:, int(b.tab[r, 37])][:, :8] = t[:, int(b.tab[0, 37])][:, :8]
    q = queries(b, 4, 9, gain=8.0)
    check_span(b, 0, q, 1.0, attend(b, 0, q, 1.0, bounds, prefixes, split))


def test_many_groups_and_blocks_beyond_4_gib():
    g = np.random.default_rng(15)
    for n, spare, hk in ((90, 5, 1), (700, 5, 1), (5, 140_000, 8)):
        groups = [(int(g.integers(0, 90)), [(int(g.integers(0, 3)), 3 + int(g.integers(0, 30)))
                                            for _ in range(int(g.integers(0, 5)))])
                  for _ in range(n)]
        b, bounds, prefixes = group_batch(Geometry("premany", 1, hk, 128, 16, "bfloat16"), LM, groups,
                                          15, spare=spare)
        q = queries(b, 2 * hk, 15)
        for split in (64, 0, 4096):
            check_span(b, 0, q, 0.1, attend(b, 0, q, 0.1, bounds, prefixes, split))


def test_two_calls_at_once_and_a_replayed_graph():
    groups = [(900, [(4, 9), (1, 300), (5, 5)]), (500, [(2, 30)] * 5)]
    b, bounds, prefixes = group_batch(Geometry("pregraph", 2, 2, 64, 16, "bfloat16"), BM, groups, 17)
    q = queries(b, 4, 17)
    most = (6, 12, 400, 1000)
    ref = [attend(b, l, q, 0.1, bounds, prefixes, 128, most) for l in range(2)]
    need = fk.flowkv_prefix_attention_workspace(b.n_tokens, 8, 4, 2, 64, 2, *most, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [torch.zeros_like(r) for r in ref]
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    gb, pl = i32(bounds), i32(prefixes)
    torch.cuda.synchronize()

    def call(l=1, stream=None):
        fk.flowkv_prefix_attention(b.pool, l, q, *b.args(), gb, pl, *most, 0.1, out[l], ws[l], 128,
                                   stream=stream)
    for i in range(10):
        for l in range(2):
            call(l, streams[l])
    torch.cuda.synchronize()
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for bd, pf, new, own in (([0, 3, 8], [900, 500], [4, 1, 5, 2, 2, 2, 2, 2], [9, 300, 5] + [30] * 5),
                             ([0, 3, 8], [640, 64], [0, 6, 1, 2, 0, 1, 1, 1], [70, 200, 5] + [9] * 5),
                             ([0, 0, 3], [900, 900], [1] * 8, [9, 20, 3] + [400] * 5)):
        b.new = np.asarray(new)
        b.total = np.asarray(own, np.int64)
        for g, p in enumerate(pf):
            b.total[bd[g]:bd[g + 1]] += p
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.offsets.copy_(torch.as_tensor(b.off))
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        b.max_len = int(b.total.max())
        gb.copy_(i32(bd))
        pl.copy_(i32(pf))
        out[1].fill_(float("nan"))
        ws[1].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check_span(b, 1, q, 0.1, out[1])
        assert torch.isnan(out[1][int(b.off[-1]):].float()).all()


def test_a_serving_loop():
    """A prompt's K and V appended with rotation, in two chunks with attention behind each;
    forks of the prompt; steps of the forks, each an append with rotation and attention over
    the shared prompt; and the same steps through a window.  Every output against the formula
    over the pool as it then is, which the rotated rows were checked into."""
    from tests.paged_batch import Batch
    from tests.span_batch import check_rotated, rotated_plain
    from tests.test_rotate_gpu import table
    hk, G, d, bs = 2, 4, 64, 16
    geom = Geometry("preloop", 2, hk, d, bs, "bfloat16")
    b = Batch(geom, BM, [0], [0], 18, spare=200)
    alloc = fk.Allocator(b.blocks)
    angles = table(700, d)
    gen = torch.Generator("cuda").manual_seed(18)
    prompt, forks, layer = 333, 6, 1
    lists = [alloc.alloc(-(-prompt // bs))]

    def step(new, total, prefix=None):
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.n_tokens = int(b.off[-1])
        b.tab = np.full((len(new), max(map(len, lists))), -1, np.int32)
        for r, ids in enumerate(lists):
            b.tab[r, :len(ids)] = ids
        b.upload()
        x = torch.randn((b.n_tokens, (G + 2) * hk * d), device="cuda", generator=gen).bfloat16()
        q, k, v = (y.unflatten(1, (-1, d)) for y in x.split([G * hk * d, hk * d, hk * d], 1))
        turned = torch.empty_like(q, memory_format=torch.contiguous_format)
        fk.flowkv_append_rotated(b.pool, layer, k, v, angles, *b.args(), q=q, q_out=turned)
        pos = torch.as_tensor(np.concatenate([np.arange(t - n, t) for n, t in zip(new, total)]),
                              device="cuda")
        for got, x in ((turned, q),):
            check_rotated(got, *rotated_plain(x, pos, angles, False), d)
        view = b.layer_view(layer)
        for r, i, row in b.rows():
            p = int(b.total[r] - b.new[r]) + i
            slot = view[:, int(b.tab[r, p // bs]), p % bs]
            check_rotated(slot[0][None], *rotated_plain(k[row:row + 1], pos[row:row + 1], angles,
                                                        False), d)
            assert torch.equal(slot[1], v[row])
        bounds = [0, len(new)]
        for split in (0, 64):
            out = attend(b, layer, turned, 0.1, bounds, [prefix or 0], split)
            check_span(b, layer, turned, 0.1, out)
        from tests.test_window_attention_gpu import attend as through
        for window, sinks in ((100, 4), (400, 0)):
            check_span(b, layer, turned, 0.1, through(b, layer, turned, 0.1, window, sinks), window,
                       sinks)
    step([200], [200])
    step([133], [333])
    for _ in range(forks - 1):
        ids, copy = alloc.fork(lists[0], prompt, bs)
        k = prompt // bs
        fk.flowkv_copy_blocks(b.pool, lists[0][k:k + 1], ids[k:], [copy])
        lists.append(ids)
    for t in range(1, 18):
        for r in range(forks):
            if (prompt + t - 1) // bs >= len(lists[r]):
                lists[r] = np.concatenate([lists[r], alloc.alloc(1)])
        if t in (1, 2, 17):
            step([1] * forks, [prompt + t] * forks, prompt)
    step([3] * forks, [prompt + 17] * forks, prompt)


def test_the_binding_refuses_other_types_and_shapes():
    groups = [(30, [(1, 5), (1, 6)])]
    b, bounds, prefixes = group_batch(Geometry("prerefuse", 1, 2, 64, 16, "bfloat16"), LM, groups, 9)
    q = queries(b, 4, 6)
    out, g, p = torch.empty_like(q), i32(bounds), i32(prefixes)
    for a in ((q.half(), out, g, p), (q, out.half(), g, p), (q, out, g.long(), p),
              (q, out, g[:1], p), (q, out, g, p.cpu()), (q, out, g, p[:, None]),
              (q, out[:1], g, p)):
        with pytest.raises(ValueError):
            fk.flowkv_prefix_attention(b.pool, 0, a[0], *b.args(), a[2], a[3], 1, 2, 6, 30, 0.1, a[1])
    with pytest.raises(fk.FlowKVError):
        fk.flowkv_prefix_attention(b.pool, 0, q, *b.args(), g, p, 1, 2, 6, 30, 0.1, out, None, 64)
