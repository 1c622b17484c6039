"""More calls of the rotary positions, the paged cache and its attention that the
header allows, against the fp64 oracle, with the tolerances of
test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from oracle import paged as OP
from paper_2503_12450_amd import binding as B
from test_gpu_paged import DEV, TDT, Case, _f64, _i32, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,m", [([3, 5], 6), ([200, 250], 310), ([4, 3, 5], 4), ([2] * 80, 101)])
def test_rows_that_the_batch_names_past_m(dtype, rows, m):
    """The matrices hold fewer rows than q_start says: those there are keep their
    tokens, the sequence's first ones of its new."""
    c = Case(101, rows, [n + 20 for n in rows], 2, 2, 32, 16, dtype)
    want = [a[:m] for a in c.oracle(True, 30, 2)]
    out = torch.full((m + 2, 64), 7.0, dtype=TDT[dtype], device=DEV)
    B.k_paged_attention(c.batch(), c.q[:m].contiguous(), out[:m], True, 30, 2)
    c.check(out[:m], want=want)
    assert torch.all(out[m:] == 7.0)
    k, v = _normal(102, (c.m, 64), dtype), _normal(103, (c.m, 64), dtype)
    pk, pv = _f64(c.k), _f64(c.v)
    before = pk.copy(), pv.copy()
    OP.store(pk, pv, _f64(k).reshape(-1, 2, 32), _f64(v).reshape(-1, 2, 32), c.table, c.q_start, c.kv)
    for s in range(len(rows)):   # what rows from m on would have stored
        for r in range(max(m, c.q_start[s]), c.q_start[s + 1]):
            t = c.kv[s] - c.q_start[s + 1] + r
            at = c.table[s, t // 16], slice(None), t % 16
            pk[at], pv[at] = before[0][at], before[1][at]
    B.k_paged_store(c.batch(), k[:m].contiguous(), v[:m].contiguous())
    assert np.array_equal(_f64(c.k), pk, equal_nan=True) and np.array_equal(_f64(c.v), pv, equal_nan=True)
