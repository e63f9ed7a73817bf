"""Block owners, forks and compaction of the allocator against a plain model, and the
argument checks of append, chunk attention and block copies (CPU: every call here returns
before it touches a device)."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

from paper_2504_03775_amd import flowkv as fk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def code(f, *a):
    with pytest.raises(fk.FlowKVError) as e:
        f(*a)
    return e.value.code


class Model:
    """Owners by block, and (FIFO policies) the free list in order."""

    def __init__(self, P, policy):
        self.P, self.own, self.policy = P, np.zeros(P, np.int64), policy
        self.queue = list(range(P))

    def free(self, ids):
        for b in ids:
            self.own[b] -= 1
            if self.own[b] == 0:
                self.queue.append(b)

    def take(self, ids):
        assert (self.own[ids] == 0).all()
        self.own[ids] = 1
        if self.policy == fk.POLICY_FIFO_SORTED:
            assert list(ids) == self.queue[:len(ids)]
        self.queue = [b for b in self.queue if b not in set(int(x) for x in ids)]

    def check(self, a):
        assert (a.owners(np.arange(self.P)) == self.own).all()
        st_ = a.stats()
        free = self.own == 0
        runs = np.flatnonzero(np.diff(np.concatenate(([0], free.astype(int), [0])))).reshape(-1, 2)
        assert st_["free_blocks"] == free.sum() and st_["free_segments"] == len(runs)
        assert st_["largest_free"] == max([int(e - s) for s, e in runs], default=0)


@pytest.mark.parametrize("policy", [fk.POLICY_SEGMENT, fk.POLICY_FIFO_SORTED])
@settings(max_examples=60, deadline=None)
@given(seed=st.integers(0, 2**63 - 1))
def test_owners_forks_and_compaction_on_random_streams(policy, seed):
    g = np.random.default_rng(seed)
    P, bs = int(g.integers(1, 120)), int(g.integers(1, 9))
    a, m = fk.Allocator(P, policy), Model(P, policy)
    held = []                               # (block list, tokens)
    for _ in range(60):
        op = g.integers(0, 6)
        room = int((m.own == 0).sum())
        if op <= 1:
            tokens = int(g.integers(0, bs * (room + 1) + 2))
            n = -(-tokens // bs)
            if n > room:
                assert code(a.alloc, n) == fk.ENOSPC
            else:
                ids = a.alloc(n)
                m.take(ids)
                held.append((ids, tokens))
        elif op == 2 and held:
            ids, tokens = held.pop(int(g.integers(len(held))))
            a.free(ids)
            m.free(ids)
        elif op == 3 and held:
            ids, _ = held[int(g.integers(len(held)))]
            ids = ids[:int(g.integers(0, len(ids) + 1))]
            a.share(ids)
            m.own[ids] += 1
            held.append((ids, len(ids) * bs))
        elif op == 4 and held:
            ids, tokens = held[int(g.integers(len(held)))]
            tokens = int(g.integers(0, tokens + 1))
            full, rest = divmod(tokens, bs)
            if rest and room == 0:
                assert code(a.fork, ids, tokens, bs) == fk.ENOSPC
            else:
                new, copy = a.fork(ids, tokens, bs)
                assert copy == rest and len(new) == full + (rest > 0)
                assert (new[:full] == ids[:full]).all()
                m.own[ids[:full]] += 1
                m.take(new[full:])
                held.append((new, tokens))
        elif op == 5:
            live = int((m.own > 0).sum())
            src, dst = a.compact()
            assert (src == np.flatnonzero(m.own[live:] > 0) + live).all()
            assert (dst == np.flatnonzero(m.own[:live] == 0)).all()
            m.own[dst], m.own[src] = m.own[src], 0
            m.queue = [b for b in m.queue if b not in set(dst.tolist())] + src.tolist()
            name = np.arange(P)
            name[src] = dst
            held = [(name[ids].astype(np.int32), t) for ids, t in held]
        m.check(a)
    for ids, _ in held:
        a.free(ids)
        m.free(ids)
    m.check(a)
    assert a.stats()["free_blocks"] == P
    if policy == fk.POLICY_FIFO_SORTED:
        assert a.alloc(P).tolist() == m.queue


def test_allocator_refusals_change_nothing():
    a = fk.Allocator(10)
    ids = a.alloc(5)
    for f, args, want in (
            (a.share, ([9],), fk.EDUP), (a.share, ([0, 0],), fk.EDUP), (a.share, ([10],), fk.ERANGE),
            (a.share, ([-1],), fk.ERANGE), (a.owners, ([10],), fk.ERANGE),
            (a.fork, (ids, 21, 4), fk.EINVAL), (a.fork, (ids, -1, 4), fk.EINVAL),
            (a.fork, (ids, 3, 0), fk.EINVAL), (a.fork, ([7], 3, 4), fk.EDUP),
            (a.fork, ([1, 1], 8, 4), fk.EDUP), (a.fork, ([1, 30], 8, 4), fk.ERANGE)):
        assert code(f, *args) == want, args
        assert a.owners(np.arange(10)).tolist() == [1] * 5 + [0] * 5
    # only the blocks that the tokens lie in are looked at
    new, copy = a.fork([1, 30], 4, 4)
    assert new.tolist() == [1] and copy == 0
    assert a.owners([1, 1]).tolist() == [2, 2]
    a.free([1])
    a.free([0, 2])
    n = ctypes.c_int32(-1)
    buf = np.full(4, -9, np.int32)
    lib = fk.lib()
    assert lib.flowkv_compact(a._h, 1, buf.ctypes.data, buf.ctypes.data, ctypes.byref(n)) == fk.ECAP
    assert n.value == 2 and (buf == -9).all()
    assert lib.flowkv_compact(a._h, -1, None, None, ctypes.byref(n)) == fk.EINVAL
    assert lib.flowkv_compact(a._h, 1, None, None, ctypes.byref(n)) == fk.EINVAL
    assert lib.flowkv_compact(None, 0, None, None, ctypes.byref(n)) == fk.EINVAL
    assert lib.flowkv_compact(a._h, 0, None, None, None) == fk.EINVAL
    assert lib.flowkv_share(None, None, 0) == lib.flowkv_owners(None, None, 0, None) == fk.EINVAL
    assert lib.flowkv_share(a._h, None, 1) == lib.flowkv_owners(a._h, None, 1, None) == fk.EINVAL
    assert lib.flowkv_fork(a._h, None, 1, 3, 4, None, ctypes.byref(n)) == fk.EINVAL
    assert lib.flowkv_fork(a._h, None, 0, 0, 4, None, None) == fk.EINVAL
    src, dst = a.compact()
    assert src.tolist() == [3, 4] and dst.tolist() == [0, 2]
    assert a.owners(np.arange(10)).tolist() == [1, 1, 1] + [0] * 7
    full = fk.Allocator(3)
    full.alloc(3)
    assert code(full.fork, [0], 1, 4) == fk.ENOSPC and full.fork([0], 4, 4)[1] == 0
    assert [x.size for x in fk.Allocator(0).compact()] == [0, 0]


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_owners_forks_and_compaction_under_asan_and_ubsan(tmp_path):
    csrc, exe = os.path.join(ROOT, "paper_2504_03775_amd", "csrc"), str(tmp_path / "pages_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "native", "pages_check.cpp"),
                    os.path.join(csrc, "flowkv_alloc.cpp"), os.path.join(csrc, "flowkv_status.cpp"),
                    "-o", exe], check=True, capture_output=True, timeout=300)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0")
    r = subprocess.run([exe, "200"], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0 and "rounds ok" in r.stdout, r.stdout + r.stderr


# ---- argument checks of the device calls ----------------------------------------

def pool(layout=1, L=2, B=8, chunk=16 * 2 * 128 * 2, bases=(1 << 20,), reserved=0):
    p = fk.flowkv_pool(layout, L, B, reserved, chunk,
                       (ctypes.c_void_p * len(bases))(*bases) if bases else None)
    return p


def append(p, layer=0, k=1 << 12, ks=512, v=1 << 13, vs=512, slot=512, n=4, n_req=1, off=1 << 14,
           tables=1 << 15, max_blocks=4, lens=1 << 16):
    vp = ctypes.c_void_p
    return fk.lib().flowkv_append(ctypes.byref(p) if p else None, layer, vp(k), ks, vp(v), vs, slot,
                                  n, n_req, vp(off), vp(tables), max_blocks, vp(lens), None)


def test_append_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    assert append(p, n=0) == fk.OK and append(p, n_req=0) == fk.OK
    for c in (dict(layer=2), dict(layer=-1), dict(slot=0), dict(slot=-512), dict(slot=8),
              dict(slot=768), dict(slot=520), dict(n=-1), dict(n_req=-1), dict(max_blocks=-1),
              dict(k=0), dict(v=0), dict(off=0), dict(lens=0), dict(tables=0), dict(k=(1 << 12) + 8),
              dict(v=(1 << 12) + 2), dict(ks=520), dict(vs=513), dict(ks=256), dict(vs=0),
              dict(ks=-512), dict(n=2**31 - 1, slot=16384, ks=16384, vs=16384)):
        assert append(p, **c) == fk.EINVAL, c
    for bad in (None, pool(layout=7), pool(L=0), pool(L=129), pool(B=0), pool(chunk=0),
                pool(chunk=24), pool(bases=()), pool(bases=(8,)), pool(bases=(0,)),
                pool(reserved=1), pool(chunk=1 << 29), pool(layout=0, bases=(1 << 20, 0)),
                pool(chunk=(1 << 62) + 16)):
        assert append(bad) == fk.EINVAL


def chunk(p, layer=0, q=1 << 12, qs=1024, n=4, n_req=1, hq=8, hkv=2, dh=128, off=1 << 14,
          tables=1 << 15, max_blocks=4, lens=1 << 16, max_new=4, max_len=60, scale=0.1, split=0,
          out=1 << 17, ws=1 << 18, ws_bytes=1 << 30):
    vp = ctypes.c_void_p
    return fk.lib().flowkv_chunk_attention(
        ctypes.byref(p) if p else None, layer, vp(q), qs, n, n_req, hq, hkv, dh, vp(off),
        vp(tables), max_blocks, vp(lens), max_new, max_len, scale, split, vp(out), vp(ws), ws_bytes,
        None)


def test_chunk_attention_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    assert chunk(p, n=0) == fk.OK and chunk(p, n_req=0) == fk.OK
    for c in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(n_req=-1), dict(hq=0), dict(hkv=0),
              dict(hq=7), dict(dh=96), dict(dh=0), dict(max_blocks=-1), dict(max_blocks=1 << 27),
              dict(max_new=-1), dict(max_len=-1), dict(max_len=2**31 - 1), dict(scale=0.0),
              dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(split=-64),
              dict(split=100), dict(split=1), dict(q=0), dict(off=0), dict(tables=0), dict(lens=0),
              dict(out=0), dict(q=(1 << 12) + 8), dict(qs=1028), dict(qs=1016), dict(qs=-1024),
              dict(out=(1 << 17) + 4), dict(split=64, max_len=65, ws=0),
              dict(split=64, max_len=65, ws=(1 << 18) + 2),
              dict(n_req=2**31 - 1, hq=2, hkv=2, qs=256)):
        assert chunk(p, **c) == fk.EINVAL, c
    need = 4 * 8 * 2 * 130 * 4
    assert chunk(p, split=64, max_len=65, ws_bytes=need - 1) == fk.ECAP
    for bad in (None, pool(layout=7), pool(L=0), pool(L=129), pool(B=0), pool(chunk=0),
                pool(chunk=16 * 2 * 128 * 2 + 16), pool(bases=()), pool(bases=(8,)),
                pool(bases=(0,)), pool(L=128, chunk=1 << 24), pool(layout=0, chunk=1 << 32)):
        assert chunk(bad) == fk.EINVAL


def test_chunk_attention_workspace_is_what_the_header_says():
    ws = fk.flowkv_chunk_attention_workspace
    assert ws(100, 3, 8, 2, 128, 50, 1000, 1024) == 0
    assert ws(100, 3, 8, 2, 128, 50, 1025, 1024) == 100 * 8 * 2 * 130 * 4
    assert ws(7, 1, 4, 4, 64, 7, 640, 64) == 7 * 4 * 10 * 66 * 4
    assert ws(0, 0, 1, 1, 64, 0, 0) == 0
    for n, req, hq, hkv, d, new, top in ((1, 1, 32, 8, 128, 1, 13000), (2000, 1, 32, 8, 128, 2000,
                                         13000), (64, 32, 8, 1, 128, 2, 32000),
                                         (5, 1, 8, 8, 64, 5, 2**31 - 5000)):
        need = ws(n, req, hq, hkv, d, new, top)
        assert need % (n * hq * (d + 2) * 4) == 0
    for bad in ((-1, 1, 8, 2, 128, 1, 10), (1, -1, 8, 2, 128, 1, 10), (1, 1, 8, 3, 128, 1, 10),
                (1, 1, 8, 2, 96, 1, 10), (1, 1, 8, 2, 128, -1, 10), (1, 1, 8, 2, 128, 1, -10),
                (1, 1, 8, 2, 128, 1, 10, 63), (2**31 - 1, 1, 2**30, 1, 128, 1, 2**31 - 5000, 64)):
        with pytest.raises(fk.FlowKVError):
            ws(*bad)
    top = 2**31 - 1
    for bad in ((top - 511, 1, 1, 1, 128, 1, 10), (2**29, 1, 32, 8, 128, 1, 10, 64),
                (2**30, top, top, top, 64, 1, top, 64),
                (2**26, top, 2**20, 2**20, 64, 1, top)):       # past 2^63 bytes
        with pytest.raises(fk.FlowKVError):
            ws(*bad)
    for big in ((top - 512, top, top, top, 64, top, 0), (1, top, top, top, 128, 1, top),
                (512, 512, 1, 1, 64, 1, top)):
        assert ws(*big) >= 0
    b = ctypes.c_int64()
    assert fk.lib().flowkv_chunk_attention_workspace(1, 1, 1, 1, 64, 1, 1, 0, None) == fk.EINVAL


def copy(p, src, dst, tokens=None, n=None, slot=512):
    a = [None if x is None else np.asarray(x, np.int32) for x in (src, dst, tokens)]
    ptr = [None if x is None else x.ctypes.data for x in a]
    return fk.lib().flowkv_copy_blocks(ctypes.byref(p) if p else None, *ptr,
                                       len(a[0]) if n is None else n, slot, None)


def test_copy_blocks_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    assert copy(p, [], []) == fk.OK and copy(p, None, None, n=0) == fk.OK
    assert copy(p, [1], [2], n=-1) == fk.EINVAL
    assert copy(p, None, [2], n=1) == fk.EINVAL and copy(p, [2], None, n=1) == fk.EINVAL
    for src, dst in (([8], [1]), ([1], [8]), ([-1], [1]), ([1], [-1]), ([0, 99], [1, 2])):
        assert copy(p, src, dst) == fk.ERANGE, (src, dst)
    for src, dst in (([0, 1], [5, 5]), ([3], [3]), ([0, 1], [1, 2]), ([0, 1], [2, 0])):
        assert copy(p, src, dst) == fk.EDUP, (src, dst)
    for tok, slot in (([17], 512), ([-1], 512), ([1], 0), ([1], 24), ([1], 8), ([1], 8192 * 2 + 16)):
        assert copy(p, [1], [2], tok, slot=slot) == fk.EINVAL, (tok, slot)
    assert copy(p, [1, 2], [3, 4], [0, 0]) == fk.OK        # no token: nothing to launch
    for bad in (None, pool(layout=7), pool(L=0), pool(B=0), pool(chunk=24), pool(bases=(8,)),
                pool(chunk=1 << 29), pool(layout=0, bases=(1 << 20, 8))):
        assert copy(bad, [1], [2]) == fk.EINVAL
