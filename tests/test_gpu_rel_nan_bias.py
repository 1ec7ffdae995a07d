"""A NaN in the bias of a bucket: the rows that see a key in that bucket are NaN, all others and the other heads keep their results."""
import numpy as np
import pytest

from gpu_common import from_dev
from rel_reference import check
from test_gpu_rel_attn import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bias_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("bucket", [0, 5, 20, 31])
@pytest.mark.parametrize("nq,nk", [(1, 700), (1, 3000), (150, 700), (130, 4100), (300, 300)])
def test_nan_in_a_bucket(nq, nk, bucket, dtype, bias_dtype):
    H = 4
    starts = [nk - nq, max(0, 60 - nq)]
    lengths = [nk, starts[1] + nq]
    p = Problem(2, H, 2, nq, nk, 64, dtype=dtype, bias_dtype=bias_dtype, lengths=lengths, starts=starts)
    ref = p.reference()
    p.dev[3][bucket, 1] = float("nan")
    o, lse = p.forward()
    back = p.backward(o, lse) if nq == nk else None
    o, lse = from_dev(o).astype(np.float64), from_dev(lse).astype(np.float64)
    pos = np.asarray(starts)[:, None] + np.arange(nq)
    behind = np.arange(nk) <= pos[..., None]
    seen = behind & (np.arange(nk) < np.asarray(lengths)[:, None, None])
    of = p.table[np.clip(np.arange(nk) - pos[..., None], -128, 128) + 128]
    hit = np.zeros((2, H, nq), bool)
    hit[:, 1] = (seen & (of == bucket)).any(-1)
    assert np.isnan(o[hit]).all() and np.isnan(lse[hit]).all()
    check(o[~hit], ref.o[~hit], ref.o_bound[~hit], "o of the others")
    check(lse[~hit], ref.lse[~hit], ref.lse_bound[~hit], "lse of the others")
    if back is None:
        return
    dq, dk, dv, dbias = (from_dev(t).astype(np.float64) for t in back)
    assert np.isnan(dq[hit]).all() and np.isnan(dbias[bucket, 1])
    check(dq[~hit], ref.dq[~hit], ref.dq_bound[~hit], "dq of the others")
    keep = [0, 2, 3]
    check(dbias[:, keep], ref.dbias[:, keep], ref.dbias_bound[:, keep], "dbias of the others")
    check(dk[:, 1], ref.dk[:, 1], ref.dk_bound[:, 1], "dk of the other key head")
    check(dv[:, 1], ref.dv[:, 1], ref.dv_bound[:, 1], "dv of the other key head")
