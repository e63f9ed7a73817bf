"""What the binding of rotated appends refuses, and leaves alone then (GPU)."""

import pytest
import torch

from paper_2504_03775_amd import flowkv as fk
from workloads import Geometry
from tests.gpu_helpers import LM
from tests.paged_batch import Batch
from tests.test_rotate_gpu import rows, table

pytestmark = pytest.mark.gpu


def test_q_and_q_out_come_together():
    b = Batch(Geometry("rotpair", 1, 2, 64, 16, "bfloat16"), LM, [3], [9], 9)
    q, k, v, t = rows(b, 4, 6), rows(b, 2, 7), rows(b, 2, 8), table(9, 64)
    out = torch.full_like(q, 7.0)
    before = [x.clone() for x in b.pool.tensors]
    for pair in (dict(q_out=out), dict(q=q)):
        with pytest.raises(ValueError, match="q_out"):
            fk.flowkv_append_rotated(b.pool, 0, k, v, t, *b.args(), **pair)
    torch.cuda.synchronize()
    assert (out == 7).all()
    assert all(torch.equal(x, y) for x, y in zip(b.pool.tensors, before))
