"""Appending to a pool's pages and copying pages within it (GPU), byte for byte over the
whole pool against plain indexing; and a run of the calls as a serving loop makes them."""

import sys

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry, make_device_pool
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch, append_plain, check_attention

pytestmark = pytest.mark.gpu
NAMES = {LM: "layer", BM: "block"}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def words(t):
    return t.view(torch.uint8 if t.element_size() == 1 else
                  {2: torch.int16, 4: torch.int32}[t.element_size()])


def same(a, b):
    return all(torch.equal(words(x), words(y)) for x, y in zip(a, b))


def new_kv(b, seed, lead=0, dtype=None):
    """K and V of the batch's tokens, as columns of one matrix behind `lead` others."""
    hk, d = b.geom.kv_heads, b.geom.head_dim
    dtype = dtype or b.pool.tensors[0].dtype
    x = torch.randn((b.n_tokens, lead + 2 * hk * d), device="cuda",
                    generator=torch.Generator("cuda").manual_seed(seed)).to(dtype)
    return (x[:, lead:lead + hk * d].unflatten(1, (hk, d)),
            x[:, lead + hk * d:].unflatten(1, (hk, d)))


SHAPES = [  # (layers, KV heads, head_dim, block size, dtype)
    (2, 2, 64, 16, "bfloat16"), (3, 8, 128, 16, "bfloat16"), (1, 1, 128, 1, "float16"),
    (2, 3, 64, 7, "float16"), (2, 1, 8, 100, "bfloat16"), (1, 5, 72, 3, "float16"),
]
BATCHES = [  # (new tokens, tokens in all)
    ([1], [1]), ([1] * 70, list(range(1, 71))), ([0, 5, 0, 1, 0], [3, 5, 0, 90, 0]),
    ([300], [300]), ([40, 1, 260], [77, 1, 1000]), ([1] * 5, [0, -3, 17, 16, 33]),
    ([6, 4], [3, 1000]),
]


@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_append_writes_the_new_tokens_and_nothing_else(layout, shape, batch):
    L, hk, d, bs, dt = SHAPES[shape]
    new, total = BATCHES[batch]
    seed = 17 * shape + batch
    b = Batch(Geometry("append", L, hk, d, bs, dt), layout, new, total, seed,
              pad=(seed % 2, seed % 3))
    say(f"append {NAMES[layout]} shape {SHAPES[shape]} new {new[:6]} of {total[:6]}")
    if batch == 4:      # blocks outside the pool
        b.tab[0, 0], b.tab[2, -1] = -1, b.blocks
        b.upload()
    if batch == 6:      # a table too short for the second request
        b.tab = np.ascontiguousarray(b.tab[:, :max(1, b.tab.shape[1] // 2)])
        b.upload()
    k, v = new_kv(b, seed, lead=(0, 8, 4 * d)[seed % 3])
    want = [t.clone() for t in b.pool.tensors]
    append_plain(b, L - 1, k, v, want)
    fk.flowkv_append(b.pool, L - 1, k, v, *b.args())
    torch.cuda.synchronize()
    assert same(b.pool.tensors, want)


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.float32, torch.int8])
def test_append_of_other_types(dtype):
    g = torch.Generator("cuda").manual_seed(4)
    size = torch.empty((), dtype=dtype).element_size()
    raw = torch.randint(0, 255, (9, 2, 2, 4, 2, 32 * size), dtype=torch.uint8, device="cuda",
                        generator=g)
    pool = fk.KVPool(BM, raw.view(dtype))
    kv = torch.randint(0, 255, (2, 5, 2, 32 * size), dtype=torch.uint8, device="cuda", generator=g)
    tab = torch.as_tensor(np.array([[7, 2, 5]], np.int32), device="cuda")
    off = torch.as_tensor(np.array([0, 5], np.int32), device="cuda")
    lens = torch.as_tensor(np.array([10], np.int32), device="cuda")
    want = raw.clone()
    for i in range(5):
        p = 5 + i
        blk = [7, 2, 5][p // 4]
        want[blk, 1, 0, p % 4], want[blk, 1, 1, p % 4] = kv[0, i], kv[1, i]
    fk.flowkv_append(pool, 1, kv[0].view(dtype), kv[1].view(dtype), off, tab, lens)
    torch.cuda.synchronize()
    assert torch.equal(raw, want)


def test_append_of_a_whole_prompt_and_far_blocks():
    """5,000 tokens at Llama-3-8B's geometry, blocks past 4 GiB of the pool's base."""
    for layout in (BM, LM):
        geom = Geometry("appendfar", 2, 8, 128, 16, "bfloat16")
        b = Batch(geom, layout, [5000, 1, 77], [5000, 9000, 300], 21, spare=90_000)
        k, v = new_kv(b, 21, lead=32 * 128)
        pre = [b.layer_view(1).clone(), b.layer_view(0).clone()]
        fk.flowkv_append(b.pool, 1, k, v, *b.args())
        torch.cuda.synchronize()
        r, pos, row = np.repeat(np.arange(3), b.new), [], np.arange(b.n_tokens)
        pos = np.concatenate([np.arange(t - m, t) for m, t in zip(b.new, b.total)])
        blk = torch.as_tensor(b.tab[r, pos // 16].astype(np.int64), device="cuda")
        slot = torch.as_tensor(pos % 16, device="cuda")
        pre[0][0, blk, slot], pre[0][1, blk, slot] = k, v
        assert torch.equal(b.layer_view(1), pre[0]) and torch.equal(b.layer_view(0), pre[1])
        del b, pre
        torch.cuda.empty_cache()


@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_a_long_append_of_many_requests_some_without_a_place(layout):
    """More pieces than one a lane takes; requests of every length, empty ones, blocks
    outside the pool, a length below its new tokens."""
    g = np.random.default_rng(31)
    new = [0, 700, 1, 0, 333, 64, 1, 1, 129, 0, 17] + [int(x) for x in g.integers(0, 40, 60)]
    total = [m + int(x) for m, x in zip(new, g.integers(0, 300, len(new)))]
    total[4] = new[4] - 100                            # the first 100 have no position
    b = Batch(Geometry("appendlong", 2, 8, 72, 13, "bfloat16"), layout, new, total, 31)
    assert b.n_tokens * 2 * 8 * 72 * 2 // 16 > 1 << 18
    b.tab[1, 3], b.tab[5, 1], b.tab[8, 0] = -7, b.blocks, 2 ** 31 - 1
    b.upload()
    k, v = new_kv(b, 31, lead=16)
    say(f"long append {NAMES[layout]} of {b.n_tokens} tokens")
    want = [t.clone() for t in b.pool.tensors]
    append_plain(b, 1, k, v, want)
    fk.flowkv_append(b.pool, 1, k, v, *b.args())
    torch.cuda.synchronize()
    assert same(b.pool.tensors, want)


def copy_plain(tensors, layout, src, dst, tokens, bs):
    for i, (s, d) in enumerate(zip(src, dst)):
        k = bs if tokens is None else int(tokens[i])
        if layout == BM:
            tensors[0][int(d), :, :, :k] = tensors[0][int(s), :, :, :k]
        else:
            for t in tensors:
                t[:, int(d), :k] = t[:, int(s), :k]


@pytest.mark.parametrize("tokens", [False, True], ids=["whole", "tokens"])
@pytest.mark.parametrize("n", [1, 7, 219, 221, 470, 1000])
@pytest.mark.parametrize("shape", [(2, 2, 64, 16), (5, 1, 128, 16), (1, 3, 64, 7), (128, 1, 8, 1),
                                   (3, 8, 128, 33)])
@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_copy_blocks(layout, shape, n, tokens):
    L, hk, d, bs = shape
    g = np.random.default_rng(n + L)
    B = 2 * n + 9
    pool = fk.KVPool(layout, make_device_pool(Geometry("copy", L, hk, d, bs, "bfloat16"), layout, B,
                                              "cuda", n))
    ids = g.permutation(B).astype(np.int32)
    dst = ids[:n]
    src = g.choice(ids[n:], n).astype(np.int32)        # a source may repeat
    tok = g.integers(0, bs + 1, n).astype(np.int32) if tokens else None
    say(f"copy {NAMES[layout]} {shape} {n} blocks tokens {tokens}")
    want = [t.clone() for t in pool.tensors]
    copy_plain(want, layout, src, dst, tok, bs)
    fk.flowkv_copy_blocks(pool, src, dst, tok)
    torch.cuda.synchronize()
    assert same(pool.tensors, want)


@pytest.mark.parametrize("tokens", [False, True], ids=["whole", "tokens"])
@pytest.mark.parametrize("shape", [(80, 3, 72, 7), (6, 8, 128, 16), (2, 1, 8, 33333)])
@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_copies_too_large_for_the_caches(layout, shape, tokens):
    """Over 256 MiB read and written, by a few hundred blocks in several launches."""
    L, hk, d, bs = shape
    block = 2 * L * hk * d * bs * 2
    n = (280 << 20) // block + 1                       # half as many bytes with token counts
    g = np.random.default_rng(n)
    B = 2 * n + 9
    pool = fk.KVPool(layout, make_device_pool(Geometry("copyall", L, hk, d, bs, "bfloat16"), layout,
                                              B, "cuda", n))
    ids = g.permutation(B).astype(np.int32)
    src, dst = g.choice(ids[n:], n).astype(np.int32), ids[:n]
    tok = g.integers(0, bs + 1, n).astype(np.int32) if tokens else None
    assert 2 * block * n // (2 if tokens else 1) > 256 << 20
    say(f"copy {NAMES[layout]} {shape} {n} blocks tokens {tokens}")
    want = [t.clone() for t in pool.tensors]
    copy_plain(want, layout, src, dst, tok, bs)
    fk.flowkv_copy_blocks(pool, src, dst, tok)
    torch.cuda.synchronize()
    assert same(pool.tensors, want)


def test_copy_blocks_by_lists_arrays_and_read_only_arrays():
    geom = Geometry("copylists", 2, 2, 64, 16, "bfloat16")
    pool = fk.KVPool(BM, make_device_pool(geom, BM, 20, "cuda", 2))
    want = [t.clone() for t in pool.tensors]
    fixed = np.array([5, 9], np.int32)
    fixed.flags.writeable = False
    for src, dst, tok in (([1, 2], [3, 4], None), (fixed, (10, 11), [4, 16]),
                          (np.array([12, 99, 13], np.int64)[::2], fixed, np.array([0, 7]))):
        copy_plain(want, BM, src, dst, tok, 16)
        fk.flowkv_copy_blocks(pool, src, dst, tok)
    torch.cuda.synchronize()
    assert same(pool.tensors, want)


def test_copy_blocks_of_2_mib_far_apart():
    geom = Geometry("copyfar", 32, 8, 128, 16, "bfloat16")
    for layout in (BM, LM):
        B = 6000
        pool = fk.KVPool(layout, make_device_pool(geom, layout, B, "cuda", 3))
        src = np.arange(B - 300, B, dtype=np.int32)
        dst = np.arange(7, 307, dtype=np.int32)
        pre = [t[src[0]:].clone() if layout == BM else t[:, src[0]:].clone() for t in pool.tensors]
        edge = [(t[[6, 307]] if layout == BM else t[:, [6, 307]]).clone() for t in pool.tensors]
        fk.flowkv_copy_blocks(pool, src, dst)
        torch.cuda.synchronize()
        for t, p, e in zip(pool.tensors, pre, edge):
            now, rim = (t[7:307], t[[6, 307]]) if layout == BM else (t[:, 7:307], t[:, [6, 307]])
            assert torch.equal(now, p) and torch.equal(rim, e)
        del pool, pre
        torch.cuda.empty_cache()


def test_refused_by_the_binding():
    geom = Geometry("pagesref", 2, 2, 64, 16, "bfloat16")
    b = Batch(geom, BM, [4, 3], [40, 30], 18)
    k, v = new_kv(b, 18)
    before = b.pool.tensors[0].clone()
    for bad in ((k.float(), v), (k, v.half()), (k[:-1], v), (k[:, :1], v), (k[..., :32], v),
                (k.cpu(), v), (k.transpose(1, 2).contiguous().transpose(1, 2), v),
                (k.flatten(1), v)):
        with pytest.raises(ValueError):
            fk.flowkv_append(b.pool, 0, *bad, *b.args())
    with pytest.raises(ValueError):
        fk.flowkv_append(b.pool, 0, k, v, b.offsets.long(), b.tables, b.lens)
    with pytest.raises(fk.FlowKVError):
        fk.flowkv_append(b.pool, 2, k, v, *b.args())
    x = torch.zeros((7, 2 * 2 * 64 + 4), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(fk.FlowKVError):       # rows that are not 16 bytes apart
        fk.flowkv_append(b.pool, 0, x[:, :128].unflatten(1, (2, 64)),
                         x[:, 128:256].unflatten(1, (2, 64)), *b.args())
    for src, dst, tok in (([0], [b.blocks], None), ([-1], [0], None), ([0, 1], [2, 2], None),
                          ([0, 1], [1, 2], None), ([3], [3], None), ([0], [1], [17]),
                          ([0], [1], [-1])):
        with pytest.raises(fk.FlowKVError):
            fk.flowkv_copy_blocks(b.pool, src, dst, tok)
    for src, dst, tok in (([0], [1, 2], None), ([0], [1], [1, 2])):
        with pytest.raises(ValueError):
            fk.flowkv_copy_blocks(b.pool, src, dst, tok)
    fk.flowkv_copy_blocks(b.pool, [], [])
    fk.flowkv_copy_blocks(b.pool, np.zeros(0, np.int32), np.zeros(0, np.int32), [])
    torch.cuda.synchronize()
    assert torch.equal(b.pool.tensors[0], before)


def test_appends_and_copies_replay_in_a_graph():
    geom = Geometry("pagesgraph", 2, 2, 64, 16, "bfloat16")
    b = Batch(geom, LM, [20, 1], [50, 33], 19)
    k, v = new_kv(b, 19)
    pre = [t.clone() for t in b.pool.tensors]
    src, dst = b.tab[0, :2], np.setdiff1d(np.arange(b.blocks), b.tab)[:2].astype(np.int32)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        fk.flowkv_append(b.pool, 1, k, v, *b.args(), stream=stream)
        fk.flowkv_copy_blocks(b.pool, src, dst, [16, 3], stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fk.flowkv_append(b.pool, 1, k, v, *b.args())
        fk.flowkv_copy_blocks(b.pool, src, dst, [16, 3])
    for i in range(3):
        b.total = np.array([50 - 5 * i, 33 + i])
        b.lens.copy_(torch.as_tensor(b.total.astype(np.int32)))
        for t, p in zip(b.pool.tensors, pre):
            t.copy_(p)
        k.normal_()
        want = [t.clone() for t in pre]
        append_plain(b, 1, k, v, want)
        copy_plain(want, LM, src, dst, [16, 3], 16)
        graph.replay()
        torch.cuda.synchronize()
        assert same(b.pool.tensors, want), f"replay {i}"


@pytest.mark.parametrize("layout", [BM, LM], ids=lambda x: NAMES[x])
def test_a_serving_loop(layout):
    """Two prompts prefilled in chunks (append, then attention), one of them forked for two
    more samples, single-token steps with decode attention on all of them, the pool
    compacted and the requests moved to another pool: every attention against the formula,
    the pool's copies byte for byte, all blocks free at the end."""
    geom = Geometry("serve", 2, 2, 64, 16, "bfloat16")
    hk, d, bs, hq, B, scale = 2, 64, 16, 8, 80, 0.125
    pool = fk.KVPool(layout, make_device_pool(geom, layout, B, "cuda", 31))
    alloc = fk.Allocator(B)
    held = alloc.alloc(9)
    lists = [list(alloc.alloc(1)) for _ in range(2)]
    alloc.free(held[::2])               # holes
    gen = torch.Generator("cuda").manual_seed(32)

    def rand(n, h):
        return torch.randn((n, h, d), device="cuda", generator=gen).to(torch.bfloat16)

    def batch_of(new, total):
        b = Batch.__new__(Batch)
        b.geom, b.layout, b.pool, b.blocks = geom, layout, pool, B
        b.new, b.total = np.asarray(new), np.asarray(total)
        b.tab = np.full((len(new), max(map(len, lists))), -1, np.int32)
        for r, x in enumerate(lists):
            b.tab[r, :len(x)] = x
        b.off = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        b.n_tokens = int(b.off[-1])
        b.upload()
        return b

    def grow(total):
        for x, t in zip(lists, total):
            need = -(-t // bs) - len(x)
            if need > 0:
                x += list(alloc.alloc(need))

    def step(new, total):
        grow(total)
        b = batch_of(new, total)
        for layer in range(2):
            k, v, q = rand(b.n_tokens, hk), rand(b.n_tokens, hk), rand(b.n_tokens, hq)
            want = [t.clone() for t in pool.tensors]
            append_plain(b, layer, k, v, want)
            fk.flowkv_append(pool, layer, k, v, *b.args())
            torch.cuda.synchronize()
            assert same(pool.tensors, want)
            need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(new), hq, hk, d, b.max_new,
                                                       b.max_len, 64)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            out = torch.empty_like(q)
            fk.flowkv_chunk_attention(pool, layer, q, *b.args(), b.max_new, b.max_len, scale, out,
                                      ws, 64)
            check_attention(b, layer, q, scale, out)
            if max(new) == 1:           # the decode step's own kernel, float32 out
                o32 = torch.empty(q.shape, dtype=torch.float32, device="cuda")
                fk.flowkv_decode_attention_noalloc(pool, layer, q, b.tables, b.lens, b.max_len,
                                                   scale, o32)
                check_attention(b, layer, q, scale, o32)
        return b

    total = [0, 0]
    for chunk in ([40, 100], [60, 30], [37, 1]):        # prompts of 137 and 131 tokens
        total = [t + c for t, c in zip(total, chunk)]
        step(chunk, total)
    for _ in range(2):                                  # two more samples of the first
        ids, tok = alloc.fork(lists[0], total[0], bs)
        k = total[0] // bs
        want = [t.clone() for t in pool.tensors]
        copy_plain(want, layout, lists[0][k:k + 1], ids[k:], [tok], bs)
        fk.flowkv_copy_blocks(pool, lists[0][k:k + 1], ids[k:], [tok])
        torch.cuda.synchronize()
        assert same(pool.tensors, want) and list(ids[:k]) == list(lists[0][:k])
        lists.append(list(ids))
        total.append(total[0])
    for _ in range(3):
        total = [t + 1 for t in total]
        last = step([1, 1, 1, 1], total)
    assert (alloc.owners(lists[0][:8]) == 3).all()
    q = rand(4, hq)
    assert fk.flowkv_chunk_attention_workspace(4, 4, hq, hk, d, 1, last.max_len) == 0
    outs = [torch.empty_like(q) for _ in range(2)]
    fk.flowkv_chunk_attention(pool, 1, q, *last.args(), 1, last.max_len, scale, outs[0])
    alloc.free(held[1::2])                              # the other holders leave, too
    src, dst = alloc.compact()
    assert len(src) and alloc.stats()["free_segments"] == 1
    fk.flowkv_copy_blocks(pool, src, dst)
    name = np.arange(B)
    name[src] = dst
    lists[:] = [[int(name[x]) for x in l] for l in lists]
    last = batch_of([1, 1, 1, 1], total)
    fk.flowkv_chunk_attention(pool, 1, q, *last.args(), 1, last.max_len, scale, outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]), "compacted pool reads differently"
    # to a decode node's pool: the first request alone
    dst_pool = fk.KVPool(BM, make_device_pool(geom, BM, B, "cuda", 33))
    there = fk.Allocator(B).alloc(len(lists[0]))
    fk.flowkv_transfer_request(pool, dst_pool, lists[0], there)
    tab = torch.as_tensor(np.asarray(there, np.int32)[None], device="cuda")
    off = torch.as_tensor(np.array([0, 1], np.int32), device="cuda")
    o = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda")
    fk.flowkv_chunk_attention(dst_pool, 1, q[:1], off, tab, last.lens[:1], 1, total[0], scale, o)
    torch.cuda.synchronize()
    assert torch.equal(o[0], outs[1][0])
    for x in lists:
        alloc.free(x)
    assert alloc.stats()["free_blocks"] == B
