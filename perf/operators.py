"""The operators on a paged KV cache beside the transfer and the decode step, as cases
that can be timed and checked: writing new tokens' K and V into their pages (append),
attention of a chunk of new tokens over the pages (attention), and copying pages within
a pool (copy).

A batch's new tokens lie one request after another; request r has its tokens at
q_offsets[r] .. q_offsets[r + 1], the last of them at position seq_lens[r] - 1.  Block
lists are shuffled, as a pool in use has them.  With ``own`` set a pass goes through the
library, without it through plain torch.  Inputs come from the seed alone.
"""

import math

import numpy as np
import torch

own = False

LM, BM = "layer", "block"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

# KV geometries: those of the library's workloads, and one of small heads and odd blocks.
# `group`: query heads per KV head
GEOMS = {
    "8b": dict(layers=32, kv_heads=8, head_dim=128, block=16, dtype="bf16", group=4),
    "70b-tp8": dict(layers=80, kv_heads=1, head_dim=128, block=16, dtype="bf16", group=8),
    "tiny": dict(layers=2, kv_heads=2, head_dim=64, block=16, dtype="fp16", group=2),
    "tiny-bf16": dict(layers=2, kv_heads=2, head_dim=64, block=16, dtype="bf16", group=2),
    "d64": dict(layers=8, kv_heads=4, head_dim=64, block=7, dtype="bf16", group=2),
}


def _step(name, kind, geom, layout, n_req, new, cached, singles=0, fused=False):
    """A batch of n_req requests with `new` = (least, most) new tokens behind `cached` ones;
    the last `singles` requests have one new token.  fused: q, k and v are columns of one
    matrix, as a joint projection leaves them."""
    return dict(name=name, kind=kind, geom=geom, layout=layout, n_req=n_req, new_lo=new[0],
                new_hi=new[1], cached_lo=cached[0], cached_hi=cached[1], singles=singles,
                fused=fused)


def _copy(name, how, geom, layout, n):
    """fork: n last blocks, each copied up to its tokens; compact: n whole blocks."""
    return dict(name=name, kind="copy", how=how, geom=geom, layout=layout, n=n)


def listed():
    return [
        # the smallest prefill there is: a short prompt on the two-layer test shape
        _step("attn-tiny", "attention", "tiny-bf16", LM, 1, (60, 60), (140, 140)),
        # one user, four drafted tokens and the sampled one verified over a long context
        _step("attn-verify-13k", "attention", "8b", BM, 1, (5, 5), (13000, 13000)),
        # a batch's speculative verification: a few tokens each over contexts of all lengths
        _step("attn-verify-batch", "attention", "8b", BM, 24, (2, 8), (2000, 16000)),
        # one chunk of a long prompt, the rest of it cached by the chunks before
        _step("attn-chunk", "attention", "8b", BM, 1, (2000, 2000), (11000, 11000), fused=True),
        # the 13,000-token prompt in one piece, nothing cached
        _step("attn-prefill-13k", "attention", "8b", BM, 1, (13000, 13000), (0, 0)),
        # a continuous batch on one tensor-parallel share: chunks of prompts beside decodes
        _step("attn-mixed", "attention", "70b-tp8", LM, 24, (100, 700), (500, 8000), singles=20,
              fused=True),
        # small heads, odd blocks: short prompts with a shared prefix already cached
        _step("attn-d64", "attention", "d64", LM, 12, (30, 900), (0, 1200)),
        # the step of a decoding batch: one token a request
        _step("append-decode", "append", "8b", BM, 32, (1, 1), (200, 4000), fused=True),
        # chunks of a few prompts, layer-major share, straight from the projection
        _step("append-chunks", "append", "70b-tp8", LM, 6, (300, 5000), (0, 6000), fused=True),
        # parallel sampling: the prompts' last blocks copied for their other samples
        _copy("copy-fork", "fork", "8b", BM, 24),
        # a pool's live blocks moved down into its holes, so that one free run is left
        _copy("copy-compact", "compact", "8b", BM, 1000),
        # the same on a layer-major share of 4 KiB chunks
        _copy("copy-compact-tp8", "compact", "70b-tp8", LM, 1500),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "append", "copy"])
    layout = rng.choice([BM, LM])
    if kind == "copy":
        geom = rng.choice(["8b", "70b-tp8", "tiny", "d64"])
        how = rng.choice(["fork", "compact"])
        most = {"8b": 900, "70b-tp8": 1500, "tiny": 20000, "d64": 8000}[geom]
        c = _copy("", how, geom, layout, _log(rng, 1, most // 4 if how == "fork" else most))
    else:
        geom = rng.choice(["8b", "8b", "70b-tp8", "d64", "tiny-bf16"])
        n = _log(rng, 1, 48)
        hi = _log(rng, 1, (8000 if kind == "attention" else 16000) // n + 1)
        # (at most what the prompt in one piece has of visible keys)
        ctx = _log(rng, 1, max(1, min(20000, 250000 // n, 80_000_000 // (n * hi) - hi // 2)))
        lo, low = (max(1, x // rng.choice([1, 3, 10])) for x in (hi, ctx))
        c = _step("", kind, geom, layout, n, (lo, hi), (0 if rng.random() < 0.3 else low, ctx),
                  singles=rng.choice([0, 0, n // 2]), fused=rng.random() < 0.5)
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens in all) of each request: a property of the case, whatever the seed."""
    n = case["n_req"]
    r = np.random.default_rng([n, case["new_lo"], case["new_hi"], case["cached_lo"],
                               case["cached_hi"]])
    new = r.integers(case["new_lo"], case["new_hi"] + 1, size=n)
    new[0] = case["new_hi"]
    cached = r.integers(case["cached_lo"], case["cached_hi"] + 1, size=n)
    cached[0] = case["cached_hi"]
    if case["singles"]:
        new[n - case["singles"]:] = 1
    return new.astype(np.int64), (new + cached).astype(np.int64)


def _pool_tensor(g, layout, blocks, seed):
    """One allocation per pool: (B, L, 2, bs, Hkv, Dh), or (L, 2, B, bs, Hkv, Dh) whose L
    slices are the layer tensors; N(0, 1) values."""
    slot = (g["block"], g["kv_heads"], g["head_dim"])
    shape = ((blocks, g["layers"], 2) if layout == BM else (g["layers"], 2, blocks)) + slot
    t = torch.empty(shape, dtype=DTYPES[g["dtype"]], device="cuda")
    t.normal_(generator=torch.Generator("cuda").manual_seed(seed))
    return t


def _step_inputs(case, seed):
    g = GEOMS[case["geom"]]
    new, total = _lengths(case)
    n, N = case["n_req"], int(new.sum())
    blocks = -(-total // g["block"])
    B = int(1.1 * blocks.sum()) + 16
    ids = np.random.default_rng(seed + 2).permutation(B).astype(np.int32)
    tab = np.full((n, int(blocks.max())), -1, dtype=np.int32)
    at = 0
    for r, k in enumerate(blocks):
        tab[r, :k] = ids[at:at + k]
        at += k
    hq, hk, d = g["kv_heads"] * g["group"], g["kv_heads"], g["head_dim"]
    gen = torch.Generator("cuda").manual_seed(seed + 3)
    x = torch.empty((N, (hq + 2 * hk) * d), dtype=DTYPES[g["dtype"]], device="cuda")
    x.normal_(generator=gen)
    q, k, v = (y.unflatten(1, (-1, d)) for y in x.split([hq * d, hk * d, hk * d], 1))
    if not case["fused"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q *= 2      # scores of a spread of 2: some keys stand out, as they do for a trained model
    return _pool_tensor(g, case["layout"], B, seed), tab, q, k, v


def _copy_inputs(case, seed):
    g, n = GEOMS[case["geom"]], case["n"]
    r = np.random.default_rng(seed + 4)
    if case["how"] == "fork":
        B = 4 * n + 16
        ids = r.permutation(B).astype(np.int32)
        parents = ids[:-(-n // 3)]          # up to three more samples of each
        src, dst = np.repeat(parents, 3)[:n], ids[len(parents):len(parents) + n]
        tokens = np.repeat(r.integers(1, g["block"], size=len(parents)), 3)[:n].astype(np.int32)
    else:
        # a pool half in use: the live blocks past the count of all live ones go to the holes
        B = 4 * n + 16
        live = np.zeros(B, dtype=bool)
        live[2 * n + r.permutation(B - 2 * n)[:n]] = True
        live[r.permutation(2 * n)[:n]] = True
        src = np.flatnonzero(live[2 * n:]).astype(np.int32) + 2 * n
        dst = np.flatnonzero(~live[:2 * n]).astype(np.int32)
        tokens = None
    return _pool_tensor(g, case["layout"], B, seed), src, dst, tokens


def _handle(layout, t):
    from paper_2504_03775_amd import flowkv as fk
    if layout == BM:
        return fk.KVPool(fk.LAYOUT_BLOCK_MAJOR, t)
    return fk.KVPool(fk.LAYOUT_LAYER_MAJOR, list(t.unbind(0)))


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), device="cuda").to(dtype)


def prepare(case, seed):
    g = GEOMS[case["geom"]]
    if case["kind"] == "copy":
        t, src, dst, tokens = _copy_inputs(case, seed)
        st = dict(case=case, t=t, src=src, dst=dst, tokens=tokens)
        if tokens is None:
            st["src_dev"], st["dst_dev"] = _dev(src, torch.int64), _dev(dst, torch.int64)
        else:       # a row for each token: its slot and the two blocks
            at = np.concatenate([np.arange(k) for k in tokens])
            st["slot"] = _dev(at, torch.int64)
            st["src_dev"], st["dst_dev"] = (_dev(np.repeat(x, tokens), torch.int64)
                                            for x in (src, dst))
    else:
        t, tab, q, k, v = _step_inputs(case, seed)
        new, total = _lengths(case)
        off = np.concatenate(([0], np.cumsum(new)))
        req = np.repeat(np.arange(len(new)), new)
        st = dict(case=case, t=t, q=q, k=k, v=v, tables=_dev(tab), offsets=_dev(off),
                  lens=_dev(total), max_new=int(new.max()), max_len=int(total.max()),
                  layer=g["layers"] // 2, scale=1 / math.sqrt(g["head_dim"]),
                  req=_dev(req, torch.int64), at=_dev(np.arange(off[-1]) - off[req], torch.int64),
                  out=torch.empty_like(q, memory_format=torch.contiguous_format))
    if own:
        st["pool"] = _handle(case["layout"], t)
        if case["kind"] == "attention":
            from paper_2504_03775_amd import flowkv as fk
            bytes_ = fk.flowkv_chunk_attention_workspace(
                q.shape[0], case["n_req"], q.shape[1], g["kv_heads"], g["head_dim"],
                st["max_new"], st["max_len"])
            st["ws"] = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    return st


# ---- one pass -----------------------------------------------------------------

def _plain_attention(st):
    g, lay = GEOMS[st["case"]["geom"]], st["layer"]
    hk, d, G, n = g["kv_heads"], g["head_dim"], g["group"], st["case"]["n_req"]
    ids = st["tables"].clamp(min=0).long()
    if st["case"]["layout"] == BM:
        kv = st["t"][:, lay][ids].movedim(2, 0)
    else:
        kv = st["t"][lay][:, ids]
    kv = kv.reshape(2, n, -1, hk, d).transpose(2, 3)[:, :, :, :st["max_len"]]
    k, v = kv[0].float().transpose(2, 3).contiguous(), kv[1].float().contiguous()
    # the requests' rows side by side, padded to the longest
    at = torch.arange(st["max_new"], device="cuda")
    lens, off = st["lens"].long(), st["offsets"].long()
    new = off[1:] - off[:-1]
    rows = (off[:-1, None] + at).clamp(max=len(st["q"]) - 1)
    q = st["q"].unflatten(1, (hk, G))[rows].permute(0, 2, 1, 3, 4).reshape(n * hk, -1, d).float()
    s = torch.bmm(q, k.flatten(0, 1)).mul_(st["scale"])
    s = s.view(n, hk, st["max_new"], G, -1)
    pos = (lens - new)[:, None] + at
    hidden = torch.arange(s.shape[-1], device="cuda") > pos[:, :, None]
    s.masked_fill_(hidden[:, None, :, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.bmm(s.view(n * hk, -1, s.shape[-1]), v.flatten(0, 1)).view(n, hk, -1, G, d) / total
    return o.transpose(1, 2)[st["req"], st["at"]].flatten(1, 2).to(st["q"].dtype)


def _plain_append(st):
    g, lay = GEOMS[st["case"]["geom"]], st["layer"]
    off = st["offsets"].long()
    pos = (st["lens"] - off[1:] + off[:-1])[st["req"]] + st["at"]
    blk, slot = st["tables"][st["req"], pos // g["block"]].long(), pos % g["block"]
    t = st["t"]
    if st["case"]["layout"] == BM:
        t[blk, lay, 0, slot], t[blk, lay, 1, slot] = st["k"], st["v"]
    else:
        t[lay, 0, blk, slot], t[lay, 1, blk, slot] = st["k"], st["v"]


def _plain_copy(st):
    t, src, dst = st["t"], st["src_dev"], st["dst_dev"]
    bm = st["case"]["layout"] == BM
    if st["tokens"] is None:
        if bm:
            t[dst] = t[src]
        else:
            t[:, :, dst] = t[:, :, src]
    elif bm:
        t[dst, :, :, st["slot"]] = t[src, :, :, st["slot"]]
    else:
        t[:, :, dst, st["slot"]] = t[:, :, src, st["slot"]]


def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2504_03775_amd import flowkv as fk
        if kind == "attention":
            fk.flowkv_chunk_attention(st["pool"], st["layer"], st["q"], st["offsets"],
                                      st["tables"], st["lens"], st["max_new"], st["max_len"],
                                      st["scale"], st["out"], st["ws"])
            return st["out"]
        if kind == "append":
            fk.flowkv_append(st["pool"], st["layer"], st["k"], st["v"], st["offsets"],
                             st["tables"], st["lens"])
        else:
            fk.flowkv_copy_blocks(st["pool"], st["src"], st["dst"], st["tokens"])
    elif kind == "attention":
        return _plain_attention(st)
    elif kind == "append":
        _plain_append(st)
    else:
        _plain_copy(st)
    return st["t"].view(torch.int16)    # the pool, bit for bit


# ---- what it costs and what it gives -------------------------------------------

def work(case):
    g = GEOMS[case["geom"]]
    slot = g["kv_heads"] * g["head_dim"] * 2
    if case["kind"] == "copy":
        n = case["n"]
        tokens = n * g["block"] if case["how"] == "compact" else n * g["block"] // 2
        return {"bytes": 2 * tokens * 2 * g["layers"] * slot, "flops": 0}
    new, total = _lengths(case)
    N, listed_blocks = int(new.sum()), int((-(-total // g["block"])).sum())
    if case["kind"] == "append":
        return {"bytes": N * 2 * 2 * slot + 4 * N // g["block"] + 8 * case["n_req"], "flops": 0}
    hq, d = g["kv_heads"] * g["group"], g["head_dim"]
    seen = sum(int(m) * int(T - m) + int(m) * (int(m) + 1) // 2 for m, T in zip(new, total))
    return {"bytes": int(total.sum()) * 2 * slot + N * hq * d * 2 * 2 + 4 * listed_blocks,
            "flops": 4 * seen * hq * d}


def exact(case, seed):
    if case["kind"] != "attention":
        return None     # bytes moved as they are: nothing is computed
    g = GEOMS[case["geom"]]
    t, tab, q, _, _ = _step_inputs(case, seed)
    new, total = _lengths(case)
    lay, G, d = g["layers"] // 2, g["group"], g["head_dim"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for m, T, ids in zip(new.tolist(), total.tolist(), tab):
        ids = _dev(ids[:-(-T // g["block"])], torch.int64)
        for h in range(g["kv_heads"]):
            if case["layout"] == BM:
                kv = t[:, lay, :, :, h][ids].movedim(1, 0)
            else:
                kv = t[lay, :, :, :, h][:, ids]
            k, v = kv.reshape(2, -1, d)[:, :T].double()
            k = k.T.contiguous()
            for lo in range(0, m, 2000):        # rows at a time
                hi = min(m, lo + 2000)
                x = q[first + lo:first + hi, h * G:(h + 1) * G].double()
                s = (x.reshape(-1, d) @ k / math.sqrt(d)).view(hi - lo, G, T)
                last = T - m + torch.arange(lo, hi, device="cuda")
                s = s.masked_fill(torch.arange(T, device="cuda") > last[:, None, None], -math.inf)
                p = torch.softmax(s, -1).view(-1, T)
                out[first + lo:first + hi, h * G:(h + 1) * G] = (p @ v).view(hi - lo, G, d)
        first += m
    return out
