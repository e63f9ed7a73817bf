"""What infinities and NaN in V cost attention of new tokens (GPU): nothing where no row sees
them, and no scan of all that is cached where rows do."""

import numpy as np
import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import BM, LM
from tests.paged_batch import Batch
from tests.test_chunk_attention_gpu import queries, say

pytestmark = pytest.mark.gpu


def prepared(b, q, split, max_len=None):
    """A call of layer 0 as a function, and its output."""
    max_len = b.max_len if max_len is None else max_len
    need = fk.flowkv_chunk_attention_workspace(b.n_tokens, len(b.new), q.shape[1], b.geom.kv_heads,
                                               b.geom.head_dim, b.max_new, max_len, split)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")

    def call():
        fk.flowkv_chunk_attention(b.pool, 0, q, *b.args(), b.max_new, max_len, 0.09, out, ws, split)
    return call, out


def microseconds(call, calls=5, tries=7):
    """The least of `tries` times of a call among others."""
    best = float("inf")
    for _ in range(tries):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(calls):
            call()
        end.record()
        torch.cuda.synchronize()
        best = min(best, begin.elapsed_time(end) / calls * 1e3)
    return best


def leave_block_0_unused(b):
    spare = np.setdiff1d(np.arange(1, b.blocks), b.tab)[0]
    b.tab[b.tab == 0] = spare
    b.upload()


@pytest.mark.parametrize("d,layout,new,total,split", [
    (128, BM, [300, 40], [1500, 1000], 0), (128, LM, [2100, 700], [2100, 1333], 1 << 20),
    (64, LM, [1100, 300], [1100, 1333], 1 << 20), (64, BM, [300, 40], [9000, 777], 0),
    (128, BM, [3, 1], [1500, 777], 0),
])
def test_a_bad_value_in_the_pools_first_row_costs_nothing(d, layout, new, total, split):
    """Rows that do not exist (behind a length, in a block outside the pool) are read as some
    row of the pool: what that one holds reaches no result and starts no search."""
    b = Batch(Geometry("oddfirst", 1, 8, d, 16, "bfloat16"), layout, new, total, 50)
    leave_block_0_unused(b)
    b.tab[1, 3] = b.blocks + 5
    b.upload()
    q = queries(b, 16, 50)
    call, out = prepared(b, q, split)
    view = b.layer_view(0)
    view[:, 0] = 0
    call()
    before = microseconds(call)
    want = out.clone()
    view[:, 0] = float("nan")
    out.fill_(7)
    call()
    after = microseconds(call)
    say(f"  {before:.1f} us, {after:.1f} with a NaN in block 0")
    assert torch.equal(out, want)
    assert after < 1.5 * before + 3


@pytest.mark.parametrize("d,layout,new,total,split", [
    (128, BM, 200, 20000, 1 << 20), (64, LM, 200, 20000, 1 << 20), (128, LM, 200, 20000, 0),
    (64, BM, 200, 20000, 0), (128, LM, 3, 20000, 0),
])
@pytest.mark.parametrize("at", [[40], [40, 15000], [15000, 19900]])
def test_seen_infinities_behind_a_missing_block_are_not_searched_for_token_by_token(
        d, layout, new, total, split, at):
    """A block is missing early in a long request, and tokens behind it hold infinities that
    every row sees: the call takes not much longer than without them."""
    b = Batch(Geometry("oddlong", 1, 2, d, 16, "bfloat16"), layout, [new], [total], 51)
    b.tab[0, 1] = -1                                        # tokens 16 to 31
    b.upload()
    q = queries(b, 8, 51)
    call, out = prepared(b, q, split, max_len=400_000)
    call()
    before = microseconds(call)
    ref = out.clone()
    view = b.layer_view(0)
    for i, p in enumerate(at):
        view[1, int(b.tab[0, p // 16]), p % 16, :, 3 + i] = float("inf")
    out.fill_(7)
    call()
    after = microseconds(call)
    say(f"  {before:.1f} us, {after:.1f} with infinities at {at}")
    sees = torch.as_tensor(total - new + np.arange(new)[:, None] >= np.asarray(at), device="cuda")
    for i in range(len(at)):
        got = out[:, :, 3 + i].float()
        assert (got[sees[:, i]] == float("inf")).all()
        assert torch.equal(out[:, :, 3 + i][~sees[:, i]], ref[:, :, 3 + i][~sees[:, i]])
    rest = [i for i in range(d) if not 3 <= i < 3 + len(at)]
    assert torch.equal(out[:, :, rest], ref[:, :, rest])
    assert after < 1.5 * before + 10


@pytest.mark.parametrize("d,layout,new,total,split", [
    (128, BM, 600, 4000, 0), (64, LM, 600, 4000, 0), (128, LM, 3, 8000, 0), (64, BM, 8, 8000, 2048),
    (128, LM, 2000, 2000, 0),
])
def test_a_request_of_nan_costs_little_more(d, layout, new, total, split):
    """All new tokens of one request are NaN, as a diverged layer leaves them: the others of
    the batch do not wait for it."""
    b = Batch(Geometry("oddnan", 1, 2, d, 16, "bfloat16"), layout, [new, new], [total, total], 52)
    q = queries(b, 8, 52)
    call, out = prepared(b, q, split)
    call()
    before = microseconds(call)
    ref = out.clone()
    view = b.layer_view(0)
    for p in range(total - new, total):
        view[:, int(b.tab[0, p // 16]), p % 16] = float("nan")
    out.fill_(7)
    call()
    after = microseconds(call)
    say(f"  {before:.1f} us, {after:.1f} with NaN")
    assert torch.isnan(out[:new].float()).all()
    assert torch.equal(out[new:], ref[new:])
    assert after < 1.5 * before + 10


@pytest.mark.parametrize("weight", ["-inf", "underflow"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("d,new,split,longest", [
    (128, 3, 0, False), (64, 7, 64, False), (64, 60, 0, False), (128, 200, 64, False),
    (64, 200, 1 << 20, False), (128, 200, 0, True), (64, 200, 0, True),
])
def test_bad_v_of_a_seen_token_reaches_its_rows_at_any_weight(d, new, split, longest, bad, weight):
    """A token whose score is -inf, or so low that its weight is 0, has a bad value in V: far
    before the new tokens, among them, in the last one, and beside a missing block.  Rows
    that see it have an element that is not finite; nothing else changes."""
    total, far = 700, 130
    for at in (far, total - new // 2 - 1, total - 1, 335):
        b = Batch(Geometry("oddweight", 1, 1, d, 16, "bfloat16"), LM, [new], [total], 53)
        if at == 335:
            b.tab[0, 336 // 16] = -1
            b.upload()
        q = queries(b, 4, 53)
        q[:, :, 3] = 1.0
        view = b.layer_view(0)
        slot = int(b.tab[0, at // 16]), at % 16, 0
        view[0][slot] = 0
        view[0][slot + (3,)] = float("-inf") if weight == "-inf" else -1e6
        call, out = prepared(b, q, split, 400_000 if longest else None)
        call()
        torch.cuda.synchronize()
        ref = out.clone()
        assert torch.isfinite(ref[min(1, new - 1):].float()).all()
        view[1][slot + (5,)] = bad
        out.fill_(7)
        call()
        torch.cuda.synchronize()
        sees = torch.as_tensor(total - new + np.arange(new) >= at, device="cuda")
        assert not torch.isfinite(out[sees][:, :, 5].float()).any(), at
        assert torch.equal(out[~sees], ref[~sees]), at
        rest = [i for i in range(d) if i != 5]
        assert torch.equal(out[:, :, rest], ref[:, :, rest]), at
