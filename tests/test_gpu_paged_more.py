"""More calls of the rotary positions, the paged cache and its attention that the
header allows, against the fp64 oracle, with the tolerances of
test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from oracle import paged as OP
from paper_2503_12450_amd import binding as B
from test_gpu_paged import DEV, TDT, Case, _check_rotation, _f64, _i32, _normal

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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("dh,sections,seqs", [(80, (20, 12, 8), 300), (64, (16,), 3), (16, (8,), 5000)])
def test_store_of_many_rows(dtype, layout, dh, sections, seqs):
    """More than 4096 rows, which go two to a workgroup: pairs of rows of one page,
    of two pages, of two sequences, and a last row alone."""
    g = np.random.Generator(np.random.Philox(seqs))
    rows = [int(n) for n in g.integers(0, 2 * 4700 // seqs + 1, seqs)]
    rows[-1] += 1 + sum(rows) % 2   # sequences of no rows among them; the sum is odd
    rows[0] += max(0, 4098 - sum(rows))
    rows[0] += 1 - sum(rows) % 2
    kv = [n + int(x) for n, x in zip(rows, g.integers(0, 40, seqs))]
    heads, Hk, page = 3, 2, 16
    c = Case(111, rows, kv, heads, Hk, dh, page, dtype, tail=2, filled=False)
    n = int(c.q_start[-1])
    assert n > 4096 and n % 2 == 1
    c.table[0, 0] = -1
    c.k.fill_(5.0)
    c.v.fill_(6.0)
    qkv = _normal(112, (c.m, (heads + 2 * Hk) * dh), dtype)
    pos = g.integers(0, 300, (c.m, len(sections))).astype(np.int32)
    freq, axis = B.rotary_sections(sections, device=DEV)
    q_out = torch.full((c.m, heads * dh), 7.0, dtype=TDT[dtype], device=DEV)
    a, b = heads * dh, (heads + Hk) * dh
    B.k_paged_store(c.batch(), qkv[:, a:b], qkv[:, b:], qkv[:, :a], q_out, B.Rotary(freq, axis, len(sections), layout),
                    _i32(pos))
    torch.cuda.synchronize()
    x, f, ax = _f64(qkv).reshape(c.m, -1, dh), _f64(freq), axis.cpu().numpy()
    _check_rotation(_f64(q_out).reshape(c.m, heads, dh)[:n], x[:n, :heads], pos[:n], f, ax, layout, dtype)
    assert torch.all(q_out[n:] == 7.0)
    # which row goes to each place
    page_of, at, row = [], [], []
    for s in range(seqs):
        t = kv[s] - rows[s] + np.arange(rows[s])
        page_of.append(c.table[s][t // page])
        at.append(t % page)
        row.append(c.q_start[s] + np.arange(rows[s]))
    page_of, at, row = (np.concatenate(i) for i in (page_of, at, row))
    page_of, at, row = (i[page_of >= 0] for i in (page_of, at, row))
    k, v = _f64(c.k), _f64(c.v)
    _check_rotation(k[page_of, :, at], x[row, heads:heads + Hk], pos[row], f, ax, layout, dtype)
    assert np.array_equal(v[page_of, :, at], x[row, heads + Hk:])
    k[page_of, :, at], v[page_of, :, at] = 5.0, 6.0
    assert np.all(k == 5.0) and np.all(v == 6.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_rotary_of_many_rows_and_heads(dtype, layout):
    m, heads, dh, sections = 4099, 5, 96, (12, 20)
    g = np.random.Generator(np.random.Philox(5))
    x = _normal(113, (m, heads * dh), dtype)
    pos = g.integers(-50, 5000, (m, 2)).astype(np.int32)
    freq, axis = B.rotary_sections(sections, device=DEV)
    out = torch.empty_like(x)
    B.k_rotary(B.Rotary(freq, axis, 2, layout), x, _i32(pos), out, dh)
    shape = (m, heads, dh)
    _check_rotation(_f64(out).reshape(shape), _f64(x).reshape(shape), pos, _f64(freq), axis.cpu().numpy(), layout,
                    dtype)
