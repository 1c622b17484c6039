"""Rotary positions, the paged cache's store and the attention over it against
the fp64 oracle (oracle/paged.py).

Tolerances, derived from the arithmetic.  One rounding to bf16 is off by at
most 2^-8 of the value, one to fp32 by 2^-24.

rotary: sine and cosine of a reduced angle carry at most 1.5e-7 (the reduced
angle rounded to fp32: 2^-26 quarter turns, 2.4e-8 rad; the functions' 2 ulp
below 1: 1.2e-7), each product and sum 2^-24 more, so an element of a pair
(a, b) is within (|a| + |b|) 2.8e-7, and then its rounding.  The oracle's own
angle is pos * freq rounded in fp64, as the kernel's: 2^-51 of the angle each.

attention: a score's fp32 sum over d_head products is off by at most d_head
2^-24 of reach = sum |q k| / sqrt(d_head), its scaling and the exponential by
another 4 x 2^-24 of it and a few ulp, so a weight by a relative
e = (d_head + 4) 2^-24 reach + 2^-21; numerator and denominator both carry it,
and their sums over L keys in fp32 L 2^-24 each, at most: 2 e + L 2^-23 of the
weights' mean of |v|.  In bf16 the weights are rounded before the second
product, 2^-8 of that mean, and the result once more.
"""
import numpy as np
import pytest
import torch

from oracle import paged as OP
from paper_2503_12450_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _f64(t):
    return t.detach().double().cpu().numpy()


def _normal(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TDT[dtype]).to(DEV)


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


# --------------------------------------------------------------------------
# Rotary positions
# --------------------------------------------------------------------------

def _check_rotation(got, x, pos, freq, axis, layout, dtype):
    """got, x [m, heads, d_head] fp64."""
    want = OP.rotary(x, pos, freq, axis, layout)
    P = len(freq)
    other = np.zeros_like(x)
    a, b = (slice(0, P), slice(P, 2 * P)) if layout == "halves" else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    other[..., a] = other[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far = np.abs(pos).max(initial=0) * np.abs(freq).max() * 2.0 ** -50
    err = (2.8e-7 + far) * other
    assert np.all(np.abs(got - want) <= err + HALF_STEP[dtype] * (np.abs(want) + err))
    rest = x[..., 2 * P:]
    assert np.array_equal(got[..., 2 * P:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("m,heads,dh,sections", [
    (1, 1, 16, (8,)), (3, 5, 64, (8, 12, 12)), (70, 3, 80, (20, 20)), (37, 2, 128, (10, 20, 30, 4)),
    (19, 7, 48, (3, 5)), (5, 40, 112, (56,)), (200, 2, 96, (16, 16, 16)),
])
def test_rotary(dtype, layout, m, heads, dh, sections):
    g = np.random.Generator(np.random.Philox(m + heads))
    x = _normal(1, (m, heads * dh), dtype)
    pos = g.integers(-50, 5000, (m, len(sections))).astype(np.int32)
    freq, axis = B.rotary_sections(sections, device=DEV)
    out = torch.empty_like(x)
    rot = B.Rotary(freq, axis, len(sections), layout)
    B.k_rotary(rot, x, _i32(pos), out, dh)
    torch.cuda.synchronize()
    shape = (m, heads, dh)
    _check_rotation(_f64(out).reshape(shape), _f64(x).reshape(shape), pos, _f64(freq), axis.cpu().numpy(), layout,
                    dtype)
    same = x.clone()
    B.k_rotary(rot, same, _i32(pos), same, dh)   # in place
    assert torch.equal(same, out)


def test_rotary_far_positions_and_strange_tables():
    """Positions at both ends of int32, a zero and a large frequency, axes that
    are none; on a column block of wider rows, whose other columns stay."""
    m, heads, dh = 6, 2, 32
    wide = _normal(2, (m, 200), "f32")
    x = wide[:, 64:64 + heads * dh]
    before = wide.clone()
    pos = np.array([[2 ** 31 - 1, -2 ** 31], [10 ** 9, 1], [-1, 0], [12345678, 87654321], [0, 0], [1, -10 ** 9]],
                   dtype=np.int32)
    freq = torch.tensor([1.0, 0.0, 1e-9, 0.7, 3.0, 1.0, 1.0, 100.0], dtype=torch.float64, device=DEV)
    axis = np.array([0, 1, 1, 1, 0, 2, -1, 0])
    out = torch.full((m, 72), 7.0, device=DEV)
    B.k_rotary(B.Rotary(freq, _i32(axis), 2), x, _i32(pos), out[:, :64], dh)
    torch.cuda.synchronize()
    got = _f64(out[:, :64].reshape(m, heads, dh))
    _check_rotation(got, _f64(x.reshape(m, heads, dh)), pos, _f64(freq), axis, "halves", "f32")
    assert torch.equal(wide, before) and torch.all(out[:, 64:] == 7.0)


def test_rotary_turns_back():
    m, heads, dh = 33, 4, 64
    x = _normal(3, (m, heads * dh), "f32")
    freq, axis = B.rotary_sections((16, 16), device=DEV)
    pos = _i32(np.arange(2 * m).reshape(m, 2) * 37)
    y, back = torch.empty_like(x), torch.empty_like(x)
    B.k_rotary(B.Rotary(freq, axis, 2), x, pos, y, dh)
    B.k_rotary(B.Rotary(-freq, axis, 2), y, pos, back, dh)
    # two rotations' errors; a pair's length bounds its elements
    r = (x.view(m, heads, 2, 32) ** 2).sum(2, keepdim=True).sqrt().expand(m, heads, 2, 32).reshape(m, -1)
    assert torch.all((back - x).abs() <= 2 * 2 ** 0.5 * 3.5e-7 * r)


def test_rotary_of_more_rows_than_one_launch():
    """2^23 rows and a few: a launch takes 2^22 workgroups of two rows."""
    m, dh = 2 ** 23 + 5, 16
    x = torch.zeros((m, dh), dtype=torch.bfloat16, device=DEV)
    x[:, 0] = 1.0
    freq, axis = B.rotary_sections((8,), device=DEV)
    pos = (torch.arange(m, dtype=torch.int32, device=DEV) % 7)[:, None].contiguous()
    B.k_rotary(B.Rotary(freq, axis, 1), x, pos, x, dh)
    angle = pos[:, 0].float()
    assert torch.all((x[:, 0].float() - angle.cos()).abs() <= 2.0 ** -8)
    assert torch.all((x[:, 8].float() - angle.sin()).abs() <= 2.0 ** -8)


# --------------------------------------------------------------------------
# A cache with batches of ragged sequences
# --------------------------------------------------------------------------

class Case:
    """rows[s] new rows and kv[s] tokens per sequence, pages in random order,
    everything that no sequence owns NaN."""

    def __init__(self, seed, rows, kv, heads, kv_heads, dh, page, dtype, tail=0, spare=2, max_kv=None, filled=True):
        g = np.random.Generator(np.random.Philox(seed))
        self.rows, self.kv, self.heads, self.kv_heads, self.dh, self.dtype = rows, kv, heads, kv_heads, dh, dtype
        self.q_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.m = int(self.q_start[-1]) + tail
        need = [-(-max(n, 0) // page) for n in kv]
        self.table = np.full((len(kv), max(1, max(need))), -1, dtype=np.int32)
        n_pages = max(1, sum(need) + spare)
        order, at = g.permutation(n_pages), 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        shape = (n_pages, kv_heads, page, dh)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=TDT[dtype], device=DEV) for _ in range(2))
        if filled:
            for s, n in enumerate(kv):
                for t0 in range(0, max(n, 0), page):
                    c, p = min(page, n - t0), int(self.table[s, t0 // page])
                    self.k[p, :, :c] = _normal(seed * 1000 + 2 * t0 + s, (kv_heads, c, dh), dtype)
                    self.v[p, :, :c] = _normal(seed * 1000 + 2 * t0 + s + 500, (kv_heads, c, dh), dtype)
        self.q = _normal(seed + 1, (self.m, heads * dh), dtype, 1.5)
        self.max_kv = max_kv

    def batch(self):
        return B.PagedBatch(B.MarPages(self.k, self.v), _i32(self.table), _i32(self.q_start), _i32(self.kv),
                            self.max_kv)

    def workspace(self, batch=None, window=0, sinks=0):
        n = B.paged_attention_workspace_bytes(batch or self.batch(), self.m, self.heads, window, sinks)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)   # NaN in every type

    def oracle(self, causal, window, sinks):
        return OP.attention(_f64(self.q).reshape(self.m, self.heads, self.dh), _f64(self.k), _f64(self.v), self.table,
                            self.q_start, self.kv, causal, window, sinks, self.max_kv)

    def check(self, out, causal=True, window=0, sinks=0, want=None, left=None):
        o, mean_abs, reach = self.oracle(causal, window, sinks) if want is None else want
        got = _f64(out).reshape(o.shape)
        L = max(max(self.kv), 1)
        e = (self.dh + 4) * 2.0 ** -24 * reach[..., None] + 2.0 ** -21
        tol = mean_abs * (2 * e + L * 2.0 ** -23 + (2.0 ** -8 if self.dtype == "bf16" else 0.0))
        tol = tol + HALF_STEP[self.dtype] * (np.abs(o) + tol)
        mine = ~np.isnan(o)
        assert np.all(np.isfinite(got[mine]))
        bad = np.abs(got - o) > tol
        assert not np.any(bad & mine), (np.argwhere(bad & mine)[:5], np.abs(got - o)[bad & mine].max())
        if left is not None:   # rows of no sequence
            assert np.all(got[~mine] == left)

    def run(self, causal=True, window=0, sinks=0, split=True, batch=None):
        batch = batch or self.batch()
        out = torch.full((self.m, self.heads * self.dh), 7.0, dtype=TDT[self.dtype], device=DEV)
        B.k_paged_attention(batch, self.q, out, causal, window, sinks,
                            self.workspace(batch, window, sinks) if split else None)
        torch.cuda.synchronize()
        return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_head_sizes(dtype, dh, causal):
    c = Case(dh, [1, 37, 5], [70, 37, 133], 2, 2, dh, 16, dtype)
    c.check(c.run(causal), causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 1), (6, 2), (7, 1), (20, 1), (64, 2), (160, 1)])
@pytest.mark.parametrize("rows", [[1, 1], [3, 9]])
def test_attention_shared_heads(dtype, heads, kv_heads, rows):
    c = Case(heads, rows, [50, 100], heads, kv_heads, 32, 32, dtype)
    c.check(c.run())


EDGE = [
    ([1], [1]), ([1], [2]), ([1], [15]), ([1], [16]), ([1], [17]), ([1], [63]), ([1], [64]), ([1], [65]),
    ([1, 1, 1], [31, 32, 33]), ([16], [16]), ([17], [17]), ([64], [64]), ([65], [65]), ([129], [129]),
    ([31, 33], [95, 97]),
    ([1, 0, 2], [0, 0, 5]),            # no tokens at all; no rows
    ([5], [2]), ([70], [3]),           # rows before the first token see nothing
    ([4, 130], [-3, 1]),               # a negative length
    ([0, 0, 0, 1], [9, 9, 9, 9]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,kv", EDGE)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_short_and_empty(dtype, rows, kv, causal):
    """Also rows behind the last sequence, left as they were."""
    c = Case(11, rows, kv, 2, 1, 32, 16, dtype, tail=3)
    c.check(c.run(causal), causal, left=7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 64), (33, 5), (64, 16), (100, 70), (128, 0),
                                          (300, 1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
def test_attention_window_and_sinks(dtype, causal, window, sinks):
    c = Case(21, [1, 150, 3], [290, 150, 70], 2, 2, 16, 32, dtype)
    c.check(c.run(causal, window, sinks), causal, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 4096])
def test_attention_page_sizes(page):
    c = Case(31, [40, 1], [300, 299], 2, 1, 32, page, "bf16")
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1, 1], [2, 90]])
def test_attention_pages_that_are_none(dtype, rows):
    """Entries below zero and past the pages: their tokens are not there.  One
    sequence has no page at all, pages shared between sequences are read."""
    c = Case(41, rows, [200, 170], 2, 2, 32, 16, dtype)
    c.table[0, 3], c.table[0, 7], c.table[1, 0] = -1, c.k.shape[0], 2 ** 31 - 1
    c.table[1, 5] = c.table[0, 4]
    c.check(c.run())
    c.check(c.run(False, 60, 20), False, 60, 20)
    c.table[0, :] = -2 ** 31
    o = c.run()
    c.check(o)
    assert torch.all(o[:rows[0]] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_attention_ignores_what_unseen_tokens_hold(dtype, bad):
    """Tokens after a causal row, before its window, on a page's unused rest:
    infinities and NaN there change no bit of rows that do not see them; rows
    that do see them are not finite."""
    c = Case(51, [70, 1, 3], [130, 77, 66], 2, 1, 64, 32, dtype)
    clean = c.run(True, 40, 5)
    c.check(clean, True, 40, 5)
    last = c.table[0, 4]
    c.k[last, 0, 1], c.v[last, 0, 1] = bad, bad          # token 129: the last row's own
    t = 75                                                # rows at 75..114 see it
    c.v[c.table[0, t // 32], 0, t % 32, 9] = bad
    got = c.run(True, 40, 5)
    p = np.arange(60, 130)
    hit = (p >= t) & (p < t + 40)
    same = _f64(got).reshape(74, 2, 64) == _f64(clean).reshape(74, 2, 64)
    assert np.all(same[:69][~hit[:69]]) and np.all(same[70:])
    assert np.all(np.delete(same[:69][hit[:69]], 9, axis=2))
    assert not np.any(np.isfinite(_f64(got).reshape(74, 2, 64)[:69][hit[:69]][:, :, 9]))
    # its own value is not finite in any column; with a key of -inf or NaN the
    # score decides
    if bad == bad and bad > 0:
        assert not np.any(np.isfinite(_f64(got)[69]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_scores_of_any_size(dtype):
    """Scores in the thousands (a softmax that is one token), equal scores, and
    zero queries (the mean of the values)."""
    c = Case(61, [60, 1], [200, 500], 2, 2, 64, 16, dtype)
    c.q[:20] *= 300.0
    c.q[20:40] = 0.0
    c.q[60] *= 1000.0
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[20, 1], [150, 1]])
def test_attention_rows_do_not_change_each_other(dtype, rows):
    """A row whose scores grow from block to block, or are not finite, leaves
    the bits of the rows that share its wave."""
    c = Case(64, rows, [400, 500], 2, 1, 64, 16, dtype)
    before = c.run()
    c.q[3] *= 400.0
    c.q[7] = float("nan")
    c.q[11] = float("inf")
    after = c.run()
    rest = [i for i in range(c.m) if i not in (3, 7, 11)]
    assert torch.equal(before[rest], after[rest])
    assert not torch.isfinite(after[7]).any() and torch.isfinite(after[3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,kv,heads,kv_heads,window", [
    ([1], [5000], 2, 1, 0), ([1], [5001], 8, 1, 0), ([4, 1], [4097, 3], 4, 2, 0), ([40], [3000], 2, 2, 0),
    ([1, 1, 1], [6000, 1, 700], 2, 1, 0), ([2], [7000], 2, 1, 3000), ([100], [2500], 1, 1, 0),
])
def test_attention_divided_among_workgroups(dtype, rows, kv, heads, kv_heads, window):
    """Few rows over long sequences; without a workspace, and with part of one,
    within the same bounds; equal calls give equal bits."""
    c = Case(71, rows, kv, heads, kv_heads, 64, 64, dtype)
    batch = c.batch()
    want = c.oracle(True, window, 4)
    out = c.run(True, window, 4, batch=batch)
    c.check(out, want=want)
    assert torch.equal(out, c.run(True, window, 4, batch=batch))
    c.check(c.run(True, window, 4, split=False, batch=batch), want=want)
    n = B.paged_attention_workspace_bytes(batch, c.m, heads, window, 4)
    for part in (n // 2 // 16 * 16, n // 5, 16, 1):
        ws = torch.full((part + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        got = torch.empty_like(out)
        B.k_paged_attention(batch, c.q, got, True, window, 4, ws[:part])
        c.check(got, want=want)
        assert torch.all(ws[part:] == 0xFF)   # nothing past the bytes that were given


def test_attention_max_kv_bounds_the_tokens():
    c = Case(81, [1, 20], [100, 90], 2, 1, 32, 16, "bf16", max_kv=60)
    c.check(c.run(False), False)
    c.check(c.run(True), True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1, 2], [60, 70]])
def test_rows_before_the_first_sequence(dtype, rows):
    """q_start need not begin at row 0."""
    c = Case(83, rows, [70, 90], 2, 2, 32, 16, dtype, tail=5)
    c.q_start = (c.q_start + 3).astype(np.int32)
    c.check(c.run(), left=7.0)
    k, v = _normal(84, (c.m, 64), dtype), _normal(85, (c.m, 64), dtype)
    pk, pv = _f64(c.k), _f64(c.v)
    OP.store(pk, pv, _f64(k).reshape(-1, 2, 32), _f64(v).reshape(-1, 2, 32), c.table, c.q_start, c.kv)
    B.k_paged_store(c.batch(), k, v)
    assert np.array_equal(_f64(c.k), pk, equal_nan=True) and np.array_equal(_f64(c.v), pv, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,m", [(5, 40), (5, 700), (90, 300)])
def test_nonsense_on_the_device_stays_inside_the_buffers(dtype, seqs, m):
    """Starts that do not ascend, lengths and tables of any value: what the
    rows hold is undefined, but nothing around the buffers changes.  (Every index
    is bounded in the kernels.)"""
    g = np.random.Generator(np.random.Philox(seqs + m))
    H, Hk, dh, page, n_pages = 4, 2, 32, 16, 11
    edge = np.array([-2 ** 31, -1, 0, 1, 5, m - 1, m, m + 1, 2 ** 30, 2 ** 31 - 1])
    q_start = np.where(g.random(seqs + 1) < 0.5, g.choice(edge, seqs + 1), g.integers(0, m, seqs + 1))
    kv_len = np.where(g.random(seqs) < 0.5, g.choice(edge, seqs), g.integers(0, 2000, seqs))
    table = np.where(g.random((seqs, 40)) < 0.3, g.choice(edge, (seqs, 40)), g.integers(0, n_pages, (seqs, 40)))

    def guarded(shape):
        n = int(np.prod(shape))
        whole = torch.full((n + 2048,), 7.0, dtype=TDT[dtype], device=DEV)
        whole[1024:-1024] = _normal(5, (n,), dtype)
        return whole, whole[1024:-1024].view(shape)

    (wk, k), (wv, v) = guarded((n_pages, Hk, page, dh)), guarded((n_pages, Hk, page, dh))
    (wo, out), (wq, q_out) = guarded((m, H * dh)), guarded((m, H * dh))
    batch = B.PagedBatch(B.MarPages(k, v), _i32(table), _i32(q_start), _i32(kv_len))
    n = B.paged_attention_workspace_bytes(batch, m, H)
    ws = torch.full((n + 4096,), 0x55, dtype=torch.uint8, device=DEV)
    q, new = _normal(6, (m, H * dh), dtype), _normal(7, (m, Hk * dh), dtype)
    freq, axis = B.rotary_sections((16,), device=DEV)
    pos = torch.zeros((m, 1), dtype=torch.int32, device=DEV)
    for window in (0, 50):
        B.k_paged_store(batch, new, new, q, q_out, B.Rotary(freq, axis, 1), pos)
        B.k_paged_attention(batch, q, out, True, window, 3, ws[:n])
        B.k_paged_attention(batch, q, out, False, window, 3)
    torch.cuda.synchronize()
    for whole in (wk, wv, wo, wq):
        assert torch.all(whole[:1024] == 7.0) and torch.all(whole[-1024:] == 7.0)
    assert torch.all(ws[n:] == 0x55)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_on_column_blocks(dtype):
    """q and out as column blocks of wider rows; the other columns stay."""
    c = Case(91, [1, 40], [60, 80], 4, 2, 48, 16, dtype)
    wide = _normal(92, (c.m, 4 * 48 + 80), dtype)
    wide[:, 64:64 + 192] = c.q
    out = torch.full((c.m, 4 * 48 + 16), 7.0, dtype=TDT[dtype], device=DEV)
    B.k_paged_attention(c.batch(), wide[:, 64:64 + 192], out[:, 8:200])
    torch.cuda.synchronize()
    c.check(out[:, 8:200].contiguous())
    assert torch.all(out[:, :8] == 7.0) and torch.all(out[:, 200:] == 7.0)


def test_cache_past_32_bit_offsets():
    """A cache of more than 2^32 bytes, the pages of the sequences at its end:
    stored to and read there."""
    Hk, page, dh = 2, 128, 128
    n_pages = (2 ** 32 // (Hk * page * dh * 2)) + 70
    k = torch.empty((n_pages, Hk, page, dh), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    small = Case(95, [3, 33], [200, 300], 2, 2, dh, page, "bf16")
    n_small = small.k.shape[0]
    k[n_pages - n_small:], v[n_pages - n_small:] = small.k, small.v
    table = np.where(small.table >= 0, small.table + n_pages - n_small, -1)
    batch = B.PagedBatch(B.MarPages(k, v), _i32(table), _i32(small.q_start), _i32(small.kv))
    out = small.run(batch=batch)
    assert torch.equal(out, small.run())
    new_k, new_v = _normal(96, (36, 256), "bf16"), _normal(97, (36, 256), "bf16")
    first_k = k[:n_small].clone()
    B.k_paged_store(batch, new_k, new_v)
    B.k_paged_store(small.batch(), new_k, new_v)
    torch.cuda.synchronize()
    assert torch.equal(k[n_pages - n_small:].view(torch.int16), small.k.view(torch.int16))
    assert torch.equal(v[n_pages - n_small:].view(torch.int16), small.v.view(torch.int16))
    assert torch.equal(k[:n_small].view(torch.int16), first_k.view(torch.int16))


def test_attention_many_sequences():
    """More sequences than a search step takes, many of them empty."""
    g = np.random.Generator(np.random.Philox(7))
    rows = [int(n) for n in g.integers(0, 3, 700)]
    kv = [int(n) for n in g.integers(0, 40, 700)]
    for dtype in ("bf16", "f32"):
        c = Case(99, rows, kv, 1, 1, 16, 16, dtype, tail=2)
        c.check(c.run(), left=7.0)
        k, v = _normal(84, (c.m, 16), dtype), _normal(85, (c.m, 16), dtype)
        pk, pv = _f64(c.k), _f64(c.v)
        OP.store(pk, pv, _f64(k).reshape(-1, 1, 16), _f64(v).reshape(-1, 1, 16), c.table, c.q_start, c.kv)
        B.k_paged_store(c.batch(), k, v)
        assert np.array_equal(_f64(c.k), pk, equal_nan=True) and np.array_equal(_f64(c.v), pv, equal_nan=True)
    rows = [int(n) for n in g.integers(90, 150, 70)]   # tiles of 128 rows
    c = Case(100, rows, [n + int(x) for n, x in zip(rows, g.integers(0, 60, 70))], 1, 1, 16, 16, "bf16", tail=2)
    c.check(c.run(), left=7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_more_tiles_than_one_launch(dtype):
    """1100 sequences of one token and 4096 heads: more than 2^22 workgroups.
    A row's only token is its answer."""
    n, H, dh = 1100, 4096, 16
    k = torch.zeros((n, H, 16, dh), dtype=TDT[dtype], device=DEV)
    v = torch.full_like(k, float("nan"))
    want = _normal(98, (n, H * dh), dtype)
    v[:, :, 0] = want.view(n, H, dh)
    q, out = _normal(99, (n, H * dh), dtype), torch.empty((n, H * dh), dtype=TDT[dtype], device=DEV)
    i = np.arange(n)
    batch = B.PagedBatch(B.MarPages(k, v), _i32(i[:, None]), _i32(np.arange(n + 1)), _i32(np.ones(n)))
    B.k_paged_attention(batch, q, out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attention_scores_near_the_end_of_the_range(dtype, sign):
    """Every score the same, +-1e30 times an order of magnitude: the mean of the
    values."""
    c = Case(63, [3, 70], [100, 90], 1, 1, 32, 16, dtype)
    c.q.zero_()
    c.q[:, 0] = 3e18
    c.k.nan_to_num_(nan=0.0)
    c.k[..., 0] = sign * 1e15
    c.check(c.run(False), False)


# --------------------------------------------------------------------------
# The store
# --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("rows,kv", [([1, 1, 1], [1, 16, 33]), ([40, 0, 7], [55, 3, 7]), ([6], [3]), ([3], [0]),
                                     ([90], [200])])
def test_store(dtype, layout, rows, kv):
    """Rotated keys and plain values on their pages, every other element of the
    pages as it was (also where the table names no page, and for tokens before
    the first), queries of the sequences' rows rotated, other rows left."""
    heads, Hk, dh = 4, 2, 32
    c = Case(5, rows, kv, heads, Hk, dh, 16, dtype, tail=2, filled=False)
    if c.table.shape[1] > 1 and kv[0] > 16:
        c.table[0, 1] = c.k.shape[0] + 3 if len(rows) > 1 else -1
    c.k.fill_(5.0)
    c.v.fill_(6.0)
    qkv = _normal(6, (c.m, (heads + 2 * Hk) * dh), dtype)
    g = np.random.Generator(np.random.Philox(8))
    pos = g.integers(0, 300, (c.m, 3)).astype(np.int32)
    freq, axis = B.rotary_sections((4, 2, 2), device=DEV)   # half of a head turns
    q_out = torch.full((c.m, heads * dh), 7.0, dtype=TDT[dtype], device=DEV)
    a, b = heads * dh, (heads + Hk) * dh
    B.k_paged_store(c.batch(), qkv[:, a:b], qkv[:, b:], qkv[:, :a], q_out, B.Rotary(freq, axis, 3, layout), _i32(pos))
    torch.cuda.synchronize()
    x = _f64(qkv).reshape(c.m, -1, dh)
    n = int(c.q_start[-1])
    _check_rotation(_f64(q_out).reshape(c.m, heads, dh)[:n], x[:n, :heads], pos[:n], _f64(freq), axis.cpu().numpy(),
                    layout, dtype)
    assert torch.all(q_out[n:] == 7.0)
    mark = np.arange(c.m, dtype=np.float64)[:, None, None] + 100 * np.ones((1, Hk, dh))
    pk, pv, row = np.full(c.k.shape, 5.0), np.full(c.v.shape, 6.0), np.full(c.k.shape, -1.0)
    OP.store(pk, pv, x[:, heads:heads + Hk], x[:, heads + Hk:], c.table, c.q_start, kv)
    OP.store(row, row.copy(), mark, mark, c.table, c.q_start, kv)
    row = row[:, 0, :, 0].astype(int) - 100   # which row went to each place
    assert np.array_equal(_f64(c.v), pv)
    got = _f64(c.k)
    assert np.all(got[np.broadcast_to((row < 0)[:, None, :, None], got.shape)] == 5.0)
    pages, at = np.nonzero(row >= 0)
    r = row[pages, at]
    if len(r):
        _check_rotation(got[pages, :, at], x[r, heads:heads + Hk], pos[r], _f64(freq), axis.cpu().numpy(), layout,
                        dtype)


def test_store_without_rotation_or_queries():
    c = Case(15, [20, 3], [30, 3], 2, 2, 64, 16, "bf16", filled=False)
    k, v = _normal(16, (c.m, 128), "bf16"), _normal(17, (c.m, 128), "bf16")
    c.k.zero_()
    c.v.zero_()
    q = _normal(18, (c.m, 192), "bf16")
    before = q.clone()
    B.k_paged_store(c.batch(), k, v)
    B.k_paged_store(c.batch(), k, v, q=q, q_out=q)   # copied onto itself
    torch.cuda.synchronize()
    pk, pv = np.zeros(c.k.shape), np.zeros(c.v.shape)
    OP.store(pk, pv, _f64(k).reshape(-1, 2, 64), _f64(v).reshape(-1, 2, 64), c.table, c.q_start, c.kv)
    assert np.array_equal(_f64(c.k), pk) and np.array_equal(_f64(c.v), pv) and torch.equal(q, before)


# --------------------------------------------------------------------------
# As they are used together
# --------------------------------------------------------------------------

def test_a_prompt_a_frame_and_single_tokens():
    """Two sequences through one attention layer, step by step: a prompt
    (causal), a frame whose rows see each other, then single tokens with a
    window; products by the framework's own kernels, the cache filled by the
    store.  Every step against the layer in fp64 from its inputs, keys and
    values kept by the test in the order they came."""
    D, H, Hk, dh, page = 256, 4, 2, 64, 16
    width = (H + 2 * Hk) * dh
    w_qkv, w_o = _normal(1, (width, D), "f32", 0.06), _normal(2, (D, H * dh), "f32", 0.06)
    b_qkv, b_o = _normal(3, (width,), "f32", 0.1), _normal(4, (D,), "f32", 0.1)
    freq, axis = B.rotary_sections((8, 12, 12), device=DEV)
    rot = B.Rotary(freq, axis, 3)
    pages = B.MarPages(torch.full((40, Hk, page, dh), float("nan"), device=DEV),
                       torch.full((40, Hk, page, dh), float("nan"), device=DEV))
    order = np.random.Generator(np.random.Philox(9)).permutation(40)
    table = order[:20].reshape(2, 10).astype(np.int32)
    hist = [[np.zeros((0, Hk, dh))] * 2 for _ in range(2)]
    length = [0, 0]
    steps = [([37, 20], True, 0, 0), ([64, 64], False, 0, 0)] + [([1, 1], True, 50, 4)] * 5
    for i, (rows, causal, window, sinks) in enumerate(steps):
        m = sum(rows)
        x, resid = _normal(100 + i, (m, D), "f32"), _normal(200 + i, (m, D), "f32")
        length = [a + n for a, n in zip(length, rows)]
        start = [0, rows[0], m]
        pos = np.concatenate([[(t // 64, t % 64 // 8, t % 8) for t in range(L - n, L)]
                              for L, n in zip(length, rows)]).astype(np.int32)
        qkv, q = torch.empty((m, width), device=DEV), torch.empty((m, H * dh), device=DEV)
        o, y = torch.empty((m, H * dh), device=DEV), torch.empty((m, D), device=DEV)
        batch = B.PagedBatch(pages, _i32(table), _i32(start), _i32(length), max_kv=160)
        B.k_linear("f32", x, w_qkv, b_qkv, qkv)
        B.k_paged_store(batch, qkv[:, H * dh:(H + Hk) * dh], qkv[:, (H + Hk) * dh:], qkv[:, :H * dh], q, rot,
                        _i32(pos))
        ws = torch.empty(B.paged_attention_workspace_bytes(batch, m, H, window, sinks), dtype=torch.uint8, device=DEV)
        B.k_paged_attention(batch, q, o, causal, window, sinks, ws)
        B.k_linear_residual("f32", o, w_o, b_o, resid, y)
        torch.cuda.synchronize()
        z = (_f64(x) @ _f64(w_qkv).T + _f64(b_qkv)).reshape(m, H + 2 * Hk, dh)
        turned = OP.rotary(z[:, :H + Hk], pos, _f64(freq), axis.cpu().numpy(), "halves")
        want = np.empty((m, H, dh))
        for s in range(2):
            r = slice(start[s], start[s + 1])
            hist[s] = [np.concatenate([hist[s][0], turned[r, H:]]), np.concatenate([hist[s][1], z[r, H + Hk:]])]
            p = length[s] - rows[s] + np.arange(rows[s])[:, None]
            j = np.arange(length[s])[None]
            seen = (j <= p) if causal else np.ones((rows[s], length[s]), bool)
            if window:
                seen = seen & ((j > p - window) | (j < sinks))
            for h in range(H):
                sc = np.where(seen, turned[r, h] @ hist[s][0][:, h // 2].T / 8.0, -np.inf)
                w = np.exp(sc - sc.max(1, keepdims=True))
                want[r, h] = (w / w.sum(1, keepdims=True)) @ hist[s][1][:, h // 2]
        want = _f64(resid) + want.reshape(m, -1) @ _f64(w_o).T + _f64(b_o)
        np.testing.assert_allclose(_f64(y), want, atol=1e-4, rtol=1e-5)   # the fp32 bar of the kernels


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_step_replays_on_changed_lengths(dtype):
    """One graph of the store and the attention, replayed as the sequences
    grow: lengths, positions and rows are read on the device.  Eager calls on
    another stream and workspace run between the replays; every replay equals
    the eager result."""
    rows, kv = [1, 1, 1], [400, 30, 2000]
    c = Case(25, rows, [n + 8 for n in kv], 4, 2, 64, 16, dtype, max_kv=2048)
    c.table = np.concatenate([c.table, np.full((3, 2048 // 16 - c.table.shape[1]), -1, np.int32)], 1)
    Hk, H, dh = 2, 4, 64
    qkv, q = _normal(26, (3, 8 * dh), dtype), torch.empty((3, H * dh), dtype=TDT[dtype], device=DEV)
    pos, lens = torch.zeros((3, 2), dtype=torch.int32, device=DEV), _i32(kv)
    freq, axis = B.rotary_sections((16, 16), device=DEV)
    rot, out = B.Rotary(freq, axis, 2), torch.empty((3, H * dh), dtype=TDT[dtype], device=DEV)
    batch = B.PagedBatch(B.MarPages(c.k, c.v), _i32(c.table), _i32(c.q_start), lens, 2048)
    ws = [torch.full((B.paged_attention_workspace_bytes(batch, 3, H),), 0xFF, dtype=torch.uint8, device=DEV)
          for _ in range(2)]

    def step(q, out, ws):
        B.k_paged_store(batch, qkv[:, H * dh:(H + Hk) * dh], qkv[:, (H + Hk) * dh:], qkv[:, :H * dh], q, rot, pos)
        B.k_paged_attention(batch, q, out, True, 0, 0, ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(q, out, ws[0])
    side = torch.cuda.Stream()
    for i in range(6):
        qkv.copy_(_normal(30 + i, qkv.shape, dtype))
        lens.copy_(_i32([n + i + 1 for n in kv]))
        pos.copy_(_i32([[n + i, i] for n in kv]))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        q2, out2 = torch.empty_like(q), torch.empty_like(out)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(q2, out2, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(q, q2), i
        if i in (0, 5):
            c.kv, c.q = [n + i + 1 for n in kv], q
            c.check(out)
