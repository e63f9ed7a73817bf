"""Ragged batches over a paged pool for the GPU tests, and plain forms of the calls
over them: appends by one indexed assignment per token, attention in 64 bits from the
formula.  Nothing here calls the library but KVPool."""

from __future__ import annotations

import math

import numpy as np
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import make_device_pool
from tests.gpu_helpers import BM, LM

BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2    # 2^-8, relative
U = torch.finfo(torch.float32).eps / 2                  # 2^-24


class Batch:
    """new[r] new tokens of request r, total[r] tokens with them; blocks shuffled over a
    pool with `spare` blocks more.  pad: rows of no request before and behind."""

    def __init__(self, geom, layout, new, total, seed, spare=5, pad=(0, 0), dtype=None):
        g = np.random.default_rng(seed)
        self.geom, self.layout = geom, layout
        self.new, self.total = np.asarray(new, np.int64), np.asarray(total, np.int64)
        bs = geom.block_size
        nblk = [max(0, -(-int(t) // bs)) for t in self.total]
        self.blocks = sum(nblk) + spare
        ids = g.permutation(self.blocks).astype(np.int32)
        self.tab = np.full((len(new), max(nblk + [1])), -1, np.int32)
        at = 0
        for r, k in enumerate(nblk):
            self.tab[r, :k] = ids[at:at + k]
            at += k
        self.off = (pad[0] + np.concatenate(([0], np.cumsum(self.new)))).astype(np.int32)
        self.n_tokens = int(self.off[-1]) + pad[1]
        self.pool = fk.KVPool(layout, make_device_pool(geom, layout, self.blocks, "cuda", seed))
        self.upload()

    def upload(self):
        self.offsets = torch.as_tensor(self.off, device="cuda")
        self.tables = torch.as_tensor(self.tab, device="cuda")
        self.lens = torch.as_tensor(self.total.astype(np.int32), device="cuda")
        self.max_new = int(self.new.max(initial=0))
        self.max_len = int(self.total.max(initial=0))

    def args(self):
        return self.offsets, self.tables, self.lens

    def rows(self):
        """(request, index among its new tokens, row of the batch) of every new token."""
        for r in range(len(self.new)):
            for i in range(int(self.new[r])):
                yield r, i, int(self.off[r]) + i

    def layer_view(self, layer, tensors=None):
        """(2, blocks, bs, Hkv, Dh) of one layer, a view of the pool's tensors."""
        t = tensors or self.pool.tensors
        return t[0][:, layer].movedim(1, 0) if self.layout == BM else t[layer]


def append_plain(b, layer, k, v, tensors):
    """The slots that the new tokens go to, one by one, in `tensors`."""
    view, bs = b.layer_view(layer, tensors), b.geom.block_size
    for r, i, row in b.rows():
        p = int(b.total[r] - b.new[r]) + i
        if p < 0 or p // bs >= b.tab.shape[1]:
            continue
        blk = int(b.tab[r, p // bs])
        if 0 <= blk < b.blocks:
            view[0, blk, p % bs], view[1, blk, p % bs] = k[row], v[row]


def attention_plain(b, layer, q, scale, max_seq=None):
    """(out, w1, s1, rows) in 64 bits: outputs (rows, Hq, Dh), sum_t p_t |V_t|, the largest
    scale * sum_d |q_d K_t,d| of a row, and the rows of the batch in the same order.
    Tokens whose block is outside the pool take no part."""
    geom, bs = b.geom, b.geom.block_size
    hk, d = geom.kv_heads, geom.head_dim
    G = q.shape[1] // hk
    view = b.layer_view(layer)
    outs, w1s, s1s, rows = [], [], [], []
    for r in range(len(b.new)):
        m, T = int(b.new[r]), int(b.total[r])
        if m == 0:
            continue
        readable = min(max(T, 0), b.tab.shape[1] * bs, b.max_len if max_seq is None else max_seq)
        ids = b.tab[r, :-(-readable // bs)]
        ok = torch.as_tensor(np.repeat((ids >= 0) & (ids < b.blocks), bs)[:readable],
                             device="cuda")
        idx = torch.as_tensor(np.where((ids >= 0) & (ids < b.blocks), ids, 0).astype(np.int64),
                              device="cuda")
        kv = view[:, idx].reshape(2, -1, hk, d)[:, :readable].double()
        pos = T - m + torch.arange(m, device="cuda")
        see = (torch.arange(readable, device="cuda") <= pos[:, None]) & ok     # (m, T)
        o = torch.zeros((m, q.shape[1], d), dtype=torch.float64, device="cuda")
        w1, s1 = torch.zeros_like(o), torch.zeros((m, q.shape[1]), dtype=torch.float64,
                                                  device="cuda")
        x = q[int(b.off[r]):int(b.off[r]) + m].double()
        for h in range(q.shape[1]):
            k, v = kv[0, :, h // G], kv[1, :, h // G]
            for j in range(0, m, 512):
                sl = slice(j, min(j + 512, m))
                if readable == 0:
                    continue
                s = (x[sl, h] @ k.T.contiguous()) * scale
                # what a row does not see does not exist for it
                s = torch.where(see[sl], s, -math.inf)
                top = s.amax(1, keepdim=True)
                p = torch.where(see[sl], torch.exp(s - torch.where(top == -math.inf, 0., top)), 0.)
                den = p.sum(1, keepdim=True)
                p = torch.where(den > 0, p / den, p) if not torch.isnan(den).any() else p / den
                odd = ~torch.isfinite(v)
                if odd.any():       # 0 x inf is not 0: sum over the seen tokens alone
                    for i in range(p.shape[0]):
                        c = see[sl][i]
                        o[sl.start + i, h] = (p[i, c, None] * v[c]).sum(0)
                else:
                    o[sl, h] = p @ v
                    w1[sl, h] = p @ v.abs()
                s1[sl, h] = torch.where(see[sl], (x[sl, h].abs() @ k.abs().T.contiguous()) * scale,
                                        0.).amax(1)
        outs.append(o)
        w1s.append(w1)
        s1s.append(s1)
        rows += range(int(b.off[r]), int(b.off[r]) + m)
    return torch.cat(outs), torch.cat(w1s), torch.cat(s1s), torch.as_tensor(rows, device="cuda")


def check_attention(b, layer, q, scale, out, max_seq=None):
    """`out` (all rows of the batch) against the plain form.

    Element bound, worst case: the output's own rounding, half a bf16 step of |o|; a
    weight's rounding to bf16, half a step of it, so that of sum_t p_t |V_t| = w1; and in
    float32 (u = 2^-24) the score, Dh products and some operations behind them, each off
    by u times the sum of their sizes s1, which moves a weight and the weights' sum by
    that much relatively, and the sums over T tokens.

    Over all outputs, statistically: a rounding is uniform within half a step, which is
    at most 2^-8 / sqrt(3) relative; rounded weights against V of mean 0 move o by as
    much of its size as they are off; two of them are 2^-8 sqrt(2/3) = 3.2e-3, and the
    rows hold enough values to be within 10% of it (asserted for 4096 values and more).
    """
    want, w1, s1, rows = attention_plain(b, layer, q, scale, max_seq)
    got = out[rows].double()
    assert torch.isfinite(got).all(), "non-finite output"
    T, d = max(1, b.max_len), q.shape[2]
    tol = BF16_HALF_STEP * want.abs() + w1 * (
        BF16_HALF_STEP * (1 + BF16_HALF_STEP) + U * (4 * (d + 8) * s1[:, :, None] + 2 * T + 64))
    err = (got - want).abs()
    worst = float((err / tol.clamp(min=1e-300)).max())
    assert (err <= tol).all(), f"error {worst:.3g} times its bound"
    norm = float(want.norm())
    rel = float(err.norm()) / norm if norm else 0.0
    if want.numel() >= 4096 and norm:
        assert rel <= 1.1 * BF16_HALF_STEP * math.sqrt(2 / 3), f"relative error {rel:.3g}"
    return rel, worst
