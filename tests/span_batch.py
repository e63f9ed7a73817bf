"""Plain forms, in 64 bits from the formulas, of the calls that go beyond full causal attention
over ragged batches (tests/paged_batch.py): windows with first tokens that stay visible, shared
prefixes, rotated appends; and the bounds that the tests hold the kernels to."""

from __future__ import annotations

import math

import numpy as np
import torch

from tests.paged_batch import Batch, U


def half_step(dtype) -> float:
    """A rounding's error at most, relative to the value."""
    return torch.finfo(dtype).eps / 2


def group_batch(geom, layout, groups, seed, spare=5, pad=(0, 0)):
    """A batch whose requests share prefixes: groups[g] = (prefix, [(new, own)]), own counted
    with the new tokens, behind the prefix.  The full blocks of a prefix are shared, a
    part-filled last one is a copy.  Returns the batch, group bounds and prefix lengths."""
    new = [n for _, reqs in groups for n, _ in reqs]
    total = [p + own for p, reqs in groups for _, own in reqs]
    b = Batch(geom, layout, new, total, seed, spare=spare, pad=pad)
    bs, first, bounds, prefixes = geom.block_size, 0, [0], []
    for p, reqs in groups:
        for r in range(first + 1, first + len(reqs)):
            full, rest = divmod(p, bs)
            b.tab[r, :full] = b.tab[first, :full]
            if rest:
                for layer in range(geom.num_layers):
                    v = b.layer_view(layer)
                    v[:, int(b.tab[r, full])] = v[:, int(b.tab[first, full])]
        first += len(reqs)
        bounds.append(first)
        prefixes.append(p)
    b.upload()
    return b, np.asarray(bounds, np.int32), np.asarray(prefixes, np.int32)


def visible(T, m, readable, window, sinks):
    """(m, readable): which tokens the m new ones at the end of T see."""
    pos = (T - m + torch.arange(m, device="cuda"))[:, None]
    t = torch.arange(readable, device="cuda")
    see = t <= pos
    if window:
        see &= (t > pos - window) | (t < sinks)
    return see


def span_plain(b, layer, q, scale, window=0, sinks=0, max_seq=None):
    """(out, w1, s1, vsum, rows) in 64 bits: outputs (rows, Hq, Dh), sum_t p_t |V_t|, the largest
    scale * sum_d |q_d K_t,d| that a row sees, sum_t |V_t| over what it sees, and the rows of
    the batch in the same order.  Tokens whose block is outside the pool take no part."""
    geom, bs = b.geom, b.geom.block_size
    hk, d = geom.kv_heads, geom.head_dim
    G = q.shape[1] // hk
    view = b.layer_view(layer)
    res, rows = [], []
    for r in range(len(b.new)):
        m, T = int(b.new[r]), int(b.total[r])
        if m == 0:
            continue
        readable = min(max(T, 0), b.tab.shape[1] * bs, b.max_len if max_seq is None else max_seq)
        ids = b.tab[r, :-(-readable // bs)].astype(np.int64)
        inside = (ids >= 0) & (ids < b.blocks)
        ok = torch.as_tensor(np.repeat(inside, bs)[:readable], device="cuda")
        idx = torch.as_tensor(np.where(inside, ids, 0), device="cuda")
        kv = view[:, idx].reshape(2, -1, hk, d)[:, :readable].double()
        see = visible(T, m, readable, window, sinks) & ok
        x = q[int(b.off[r]):int(b.off[r]) + m].double()
        o, w1, vs = (torch.zeros((m, q.shape[1], d), dtype=torch.float64, device="cuda")
                     for _ in range(3))
        s1 = torch.zeros((m, q.shape[1]), dtype=torch.float64, device="cuda")
        for h in range(q.shape[1] if readable else 0):
            k, v = kv[0, :, h // G], kv[1, :, h // G]
            kt = k.T.contiguous()
            for j in range(0, m, 512):
                sl = slice(j, min(j + 512, m))
                s = torch.where(see[sl], (x[sl, h] @ kt) * scale, -math.inf)
                top = s.amax(1, keepdim=True)
                p = torch.where(see[sl], torch.exp(s - torch.where(top == -math.inf, 0., top)), 0.)
                den = p.sum(1, keepdim=True)
                p = p / den if torch.isnan(den).any() else torch.where(den > 0, p / den, p)
                if torch.isfinite(v).all():
                    o[sl, h] = p @ v
                    w1[sl, h] = p @ v.abs()
                    vs[sl, h] = see[sl].double() @ v.abs()
                else:               # 0 x inf is not 0: sum over the seen tokens alone
                    for i in range(p.shape[0]):
                        c = see[sl][i]
                        o[sl.start + i, h] = (p[i, c, None] * v[c]).sum(0)
                        w1[sl.start + i, h] = (p[i, c, None] * v[c].abs()).sum(0)
                        vs[sl.start + i, h] = v[c].abs().sum(0)
                s1[sl, h] = torch.where(see[sl], (x[sl, h].abs() @ kt.abs()) * scale, 0.).amax(1)
        res.append((o, w1, s1, vs))
        rows += range(int(b.off[r]), int(b.off[r]) + m)
    out, w1, s1, vs = (torch.cat(y) for y in zip(*res))
    return out, w1, s1, vs, torch.as_tensor(rows, device="cuda")


def check_span(b, layer, q, scale, out, window=0, sinks=0, max_seq=None):
    """`out` (all rows of the batch) against the plain form.

    Element bound, worst case, with h half a step of the type: the output's own rounding, h of
    |o| (fp16 below 2^-14: 2^-25); a weight's rounding for the matrix product, h of it, so h of
    sum_t p_t |V_t| = w1 (fp16 weights, at most 2^15 and none below 2^-25 apart from it: the
    largest so far is 2^7 or more, so an error of at most 2^-25 of a weight lifted by 2^7 is
    2^-32 of the weights' sum, for each token seen); and in float32 (u = 2^-24) the score, Dh
    products and some operations behind them, each off by u times the sum of their sizes s1,
    which moves a weight and the weights' sum by that much relatively, and the sums over T
    tokens.

    Over all outputs, statistically: a rounding is uniform within half a step, which is at most
    h / sqrt(3) relative; rounded weights against V of mean 0 move o by as much of its size as
    they are off; two of them are h sqrt(2/3), and the rows hold enough values to be within 10%
    of it (asserted for 4096 values and more, where scores are small enough for float32's part
    to be below a tenth)."""
    want, w1, s1, vs, rows = span_plain(b, layer, q, scale, window, sinks, max_seq)
    got = out[rows].double()
    assert torch.isfinite(got).all(), "non-finite output"
    T, d, h = max(1, b.max_len), q.shape[2], half_step(out.dtype)
    tol = h * want.abs() + w1 * (h * (1 + h) + U * (4 * (d + 8) * s1[:, :, None] + 2 * T + 64))
    if out.dtype == torch.float16:
        tol = tol + 2.0 ** -25 + 2.0 ** -32 * vs
    err = (got - want).abs()
    worst = float((err / tol.clamp(min=1e-300)).max())
    assert (err <= tol).all(), f"error {worst:.3g} times its bound"
    norm = float(want.norm())
    rel = float(err.norm()) / norm if norm else 0.0
    if want.numel() >= 4096 and norm and float(s1.max()) * U * math.sqrt(d) < 0.1 * h:
        assert rel <= 1.1 * h * math.sqrt(2 / 3), f"relative error {rel:.3g}"
    return rel, worst


def rotated_plain(x, pos, angles, interleaved):
    """(y, size) in 64 bits: the rows of x (n, heads, dim) turned by their positions' angles, and
    |a c| + |b s| (or |a s| + |b c|) of each element, |x| behind the rotated dims."""
    half = angles.shape[1] // 2
    a = angles.double()[pos]
    c, s = a[:, None, :half], a[:, None, half:]
    y = x.double()
    size = y.abs()
    y = y.clone()
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    u, w = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = u * c - w * s, u * s + w * c
    size[..., first] = (u * c).abs() + (w * s).abs()
    size[..., second] = (u * s).abs() + (w * c).abs()
    return y, size


def check_rotated(got, want, size, rot):
    """A rotated element: two products and a sum in float32, each within u of its result, then
    one rounding to the type (fp16 below 2^-14: 2^-25).  The dims behind are the same."""
    h = half_step(got.dtype)
    tol = h * want.abs() + (1 + h) * 3 * U * size + (2.0 ** -25 if got.dtype == torch.float16
                                                    else 0)
    err = (got.double() - want).abs()
    assert (err[..., :rot] <= tol[..., :rot]).all(), float((err / tol.clamp(min=1e-300)).max())
    assert (err[..., rot:] == 0).all()
