"""The argument checks of rotated appends, attention through a window and attention over shared
prefixes, and the workspace they ask for (CPU: every call here returns before it touches a
device)."""

import ctypes

import numpy as np
import pytest

from paper_2504_03775_amd import flowkv as fk
from tests.test_pages_host import pool

MOST = 34_080_772       # bytes, where requests bring more than 32 rows a KV head
vp = ctypes.c_void_p


def rotated(p, layer=0, dtype=0, q=1 << 11, qs=1024, qo=1 << 19, qos=1024, k=1 << 12, ks=256,
            v=1 << 13, vs=256, hq=8, hk=2, d=128, table=1 << 18, positions=100, rot=128, inter=0,
            n=4, n_req=1, off=1 << 14, tables=1 << 15, max_blocks=4, lens=1 << 16):
    return fk.lib().flowkv_append_rotated(
        ctypes.byref(p) if p else None, layer, dtype, vp(q), qs, vp(qo), qos, vp(k), ks, vp(v), vs,
        hq, hk, d, vp(table), positions, rot, inter, n, n_req, vp(off), vp(tables), max_blocks,
        vp(lens), None)


def test_append_rotated_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    for c in (dict(n=0), dict(n_req=0), dict(positions=0),
              dict(n=0, hq=0, q=0, qo=0), dict(n=0, rot=16), dict(n=0, rot=112, inter=1)):
        assert rotated(p, **c) == fk.OK, c
    for c in (dict(layer=2), dict(layer=-1), dict(dtype=3), dict(dtype=-1), dict(hq=-1), dict(hk=0),
              dict(hk=-2), dict(d=0), dict(d=4), dict(d=100), dict(d=120), dict(rot=0),
              dict(rot=-16), dict(rot=8), dict(rot=144), dict(rot=129), dict(inter=2),
              dict(inter=-1), dict(n=-1), dict(n_req=-1), dict(max_blocks=-1), dict(positions=-1),
              dict(q=0), dict(qo=0), dict(k=0), dict(v=0), dict(table=0), dict(off=0),
              dict(tables=0), dict(lens=0), dict(q=(1 << 11) + 8), dict(qo=(1 << 19) + 8),
              dict(k=(1 << 12) + 2), dict(v=(1 << 13) + 8), dict(qs=1028), dict(qos=1020),
              dict(ks=260), dict(vs=252), dict(qs=1016), dict(qos=0), dict(ks=248), dict(vs=-256),
              dict(table=(1 << 18) + 2), dict(hq=2**31 - 1), dict(n=2**31 - 1),
              dict(hk=4, ks=512, vs=512, d=192)):
        assert rotated(p, **c) == fk.EINVAL, c
    # sizes whose products pass 64 bits
    for c in (dict(hk=2**31 - 1, d=2**31 - 16), dict(hk=2**30, d=2**30, dtype=2),
              dict(hk=1, ks=128, vs=128, n=2**31 - 1, hq=2**29, qs=2**36, qos=2**36)):
        assert rotated(p, **c) == fk.EINVAL, c
    # 4-byte elements: a slot of 2 x 128 is twice as large, rotations come in 8 elements
    big = pool(chunk=16 * 2 * 128 * 4)
    assert rotated(big, dtype=2, n=0, rot=8) == fk.OK
    assert rotated(pool(chunk=2 * 128 * 2), dtype=2, n=0) == fk.EINVAL
    assert rotated(big, dtype=2, rot=4) == fk.EINVAL
    assert rotated(big, dtype=2, qs=1026) == fk.EINVAL
    for bad in (None, pool(layout=7), pool(L=0), pool(L=129), pool(B=0), pool(chunk=0),
                pool(chunk=24), pool(bases=()), pool(bases=(8,)), pool(bases=(0,)),
                pool(reserved=1), pool(chunk=1 << 29), pool(layout=0, bases=(1 << 20, 0))):
        assert rotated(bad) == fk.EINVAL


def window(p, layer=0, dtype=0, q=1 << 12, qs=1024, n=4, n_req=1, hq=8, hkv=2, dh=128, off=1 << 14,
           tables=1 << 15, max_blocks=4, lens=1 << 16, max_new=4, max_len=60, window=20, sinks=4,
           scale=0.1, split=0, out=1 << 17, ws=1 << 18, ws_bytes=1 << 30):
    return fk.lib().flowkv_window_attention(
        ctypes.byref(p) if p else None, layer, dtype, vp(q), qs, n, n_req, hq, hkv, dh, vp(off),
        vp(tables), max_blocks, vp(lens), max_new, max_len, window, sinks, scale, split, vp(out),
        vp(ws), ws_bytes, None)


def prefix(p, layer=0, dtype=0, q=1 << 12, qs=1024, n=4, n_req=4, hq=8, hkv=2, dh=128, off=1 << 14,
           tables=1 << 15, max_blocks=4, lens=1 << 16, n_groups=1, groups=1 << 21, plens=1 << 22,
           max_new=1, max_group=4, max_own=20, max_prefix=40, scale=0.1, split=64, out=1 << 17,
           ws=1 << 18, ws_bytes=1 << 30):
    return fk.lib().flowkv_prefix_attention(
        ctypes.byref(p) if p else None, layer, dtype, vp(q), qs, n, n_req, hq, hkv, dh, vp(off),
        vp(tables), max_blocks, vp(lens), n_groups, vp(groups), vp(plens), max_new, max_group,
        max_own, max_prefix, scale, split, vp(out), vp(ws), ws_bytes, None)


COMMON = (dict(layer=2), dict(layer=-1), dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(n_req=-1),
          dict(hq=0), dict(hkv=0), dict(hq=7), dict(dh=96), dict(dh=0), dict(max_blocks=-1),
          dict(max_blocks=1 << 27), dict(max_new=-1), dict(scale=0.0), dict(scale=-1.0),
          dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=3e38), dict(split=-64),
          dict(split=100), dict(split=1), dict(q=0), dict(off=0), dict(tables=0), dict(lens=0),
          dict(out=0), dict(q=(1 << 12) + 8), dict(qs=1028), dict(qs=1016), dict(qs=-1024),
          dict(out=(1 << 17) + 4), dict(n=2**31 - 1, hq=2, qs=256))
BAD_POOLS = (None, dict(layout=7), dict(L=0), dict(L=129), dict(B=0), dict(chunk=0),
             dict(chunk=16 * 2 * 128 * 2 + 16), dict(bases=()), dict(bases=(8,)), dict(bases=(0,)),
             dict(L=128, chunk=1 << 24), dict(layout=0, chunk=1 << 32))


def test_window_attention_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    for c in (dict(n=0), dict(n_req=0), dict(n=0, window=2**31 - 1, sinks=2**31 - 1),
              dict(n=0, window=1, sinks=0, dtype=1)):
        assert window(p, **c) == fk.OK, c
    for c in COMMON + (dict(window=0), dict(window=-1), dict(sinks=-1), dict(max_len=-1),
                       dict(max_len=2**31 - 1), dict(split=64, max_len=600, window=70, ws=0),
                       dict(split=64, max_len=600, window=70, ws=(1 << 18) + 2),
                       dict(n_req=2**31 - 1, hq=2, hkv=2, qs=256)):
        assert window(p, **c) == fk.EINVAL, c
    # 4 rows a token: 16 rows lie in up to 5 of them, which see 70 + 4 + 4 tokens together
    need = 4 * 8 * 2 * 130 * 4
    assert window(p, split=64, max_len=600, window=70, ws_bytes=need - 1) == fk.ECAP
    for bad in BAD_POOLS:
        assert window(bad and pool(**bad)) == fk.EINVAL, bad


def test_prefix_attention_rejects_bad_arguments_without_touching_the_device():
    p = pool()
    for c in (dict(n=0), dict(n_req=0), dict(n=0, n_groups=0, groups=0, plens=0, split=0),
              dict(n=0, split=0), dict(n=0, dtype=1)):
        assert prefix(p, **c) == fk.OK, c
    for c in COMMON + (dict(n_groups=-1), dict(max_group=-1), dict(max_own=-1),
                       dict(max_prefix=-1), dict(max_prefix=2**31 - 1),
                       dict(max_prefix=2**31 - 4097, max_own=1), dict(groups=0), dict(plens=0),
                       dict(ws=0), dict(ws=(1 << 18) + 2),
                       dict(n_req=2**31 - 1, hq=2, hkv=2, qs=256),
                       dict(n_groups=2**31 - 1, hq=2, hkv=2, qs=256)):
        assert prefix(p, **c) == fk.EINVAL, c
    need = 4 * 8 * 2 * 130 * 4      # a record of the prefix and one of the rest
    assert prefix(p, ws_bytes=need - 1) == fk.ECAP
    for bad in BAD_POOLS:
        assert prefix(bad and pool(**bad)) == fk.EINVAL, bad


def test_window_workspace_is_what_the_header_says():
    ws = fk.flowkv_window_attention_workspace
    # within one split: none
    assert ws(100, 3, 8, 2, 128, 50, 1000, 100, 4, 1024) == 0
    # 128 rows of 4 a token lie in up to 33 tokens: they see 1,000 + 4 + 32 between them
    assert ws(100, 3, 8, 2, 128, 50, 100000, 1000, 4, 1024 + 64) == 0
    assert ws(100, 3, 8, 2, 128, 50, 100000, 1000, 4, 1024) == 100 * 8 * 2 * 130 * 4
    # never more than the whole of it
    full = fk.flowkv_chunk_attention_workspace
    for w, s in ((2**31 - 1, 0), (1, 2**31 - 1), (2**31 - 1, 2**31 - 1), (50000, 4)):
        for n, new, split in ((100, 50, 64), (3, 1, 128), (3, 1, 0), (2000, 2000, 0)):
            assert ws(n, 3, 8, 2, 128, new, 40000, w, s, split) == \
                full(n, 3, 8, 2, 128, new, 40000, split)
    for bad in ((-1, 1, 8, 2, 128, 1, 10, 5, 0), (1, 1, 8, 3, 128, 1, 10, 5, 0),
                (1, 1, 8, 2, 96, 1, 10, 5, 0), (1, 1, 8, 2, 128, 1, 10, 0, 0),
                (1, 1, 8, 2, 128, 1, 10, 5, -1), (1, 1, 8, 2, 128, 1, 10, 5, 0, 63),
                (2**31 - 1, 1, 2**30, 1, 128, 1, 2**31 - 5000, 2**30, 0, 64)):
        with pytest.raises(fk.FlowKVError):
            ws(*bad)
    b = ctypes.c_int64()
    assert fk.lib().flowkv_window_attention_workspace(1, 1, 1, 1, 64, 1, 1, 1, 0, 0, None) == \
        fk.EINVAL
    g = np.random.default_rng(61)

    def spread(most):
        return int(np.exp(g.uniform(0, np.log(most))))
    for _ in range(5000):
        hk, G, d = spread(16), spread(64), (64, 128)[int(g.integers(2))]
        new, req, top = spread(40000), spread(600), spread(1 << 30)
        n = min(spread(8) * new * req if g.integers(2) else spread(1 << 20), 1 << 24)
        if new * G > 32:
            assert ws(n, req, hk * G, hk, d, new, top, spread(1 << 20), spread(5000) - 1) <= MOST
    del b


def test_prefix_workspace_holds_every_record():
    ws = fk.flowkv_prefix_attention_workspace
    assert ws(4, 4, 8, 2, 128, 1, 1, 4, 20, 40, 64) == 4 * 8 * 2 * 130 * 4
    assert ws(4, 4, 8, 2, 128, 1, 1, 4, 65, 129, 64) == 4 * 8 * 5 * 130 * 4
    # the library's rule with the most tokens of a prefix that there can be: shared, in long splits
    # (the bytes that sharing saves, 2^24 requests' x 2^42, pass 63 bits)
    assert ws(1 << 24, 1 << 24, 8, 8, 128, 1, 1, 1 << 24, 64, 1 << 30) <= (1 << 24) * 8 * 8 * 130 * 4
    # each by itself: as attention over all of it
    full = fk.flowkv_chunk_attention_workspace
    assert ws(700, 2, 8, 2, 128, 0, 600, 0, 3000, 0) == full(700, 2, 8, 2, 128, 600, 3000)
    assert ws(5, 1, 8, 2, 64, 1, 5, 5, 300, 9000) == full(5, 1, 8, 2, 64, 5, 9300)
    for bad in ((-1, 1, 8, 2, 128, 1, 1, 1, 10, 5), (1, 1, 8, 3, 128, 1, 1, 1, 10, 5),
                (1, 1, 8, 2, 128, 1, 1, -1, 10, 5), (1, 1, 8, 2, 128, 1, 1, 1, -1, 5),
                (1, 1, 8, 2, 128, 1, 1, 1, 10, -5), (1, 1, 8, 2, 128, -1, 1, 1, 10, 5),
                (1, 1, 8, 2, 128, 1, 1, 1, 10, 5, 32),
                (1, 1, 8, 2, 128, 1, 1, 1, 2**30, 2**30),
                (2**26, 2, 2**20, 2**20, 64, 1, 1, 1, 2**30, 2**30 - 5000, 64)):
        with pytest.raises(fk.FlowKVError):
            ws(*bad)
    assert fk.lib().flowkv_prefix_attention_workspace(1, 1, 1, 1, 64, 0, 1, 1, 1, 0, 0, None) == \
        fk.EINVAL
