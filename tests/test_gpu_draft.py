"""Attention of trees of drafted tokens, probabilities, verification, rows moved
together and sequences continued by others against the fp64 oracle
(oracle/draft.py).

Tolerances.  The attention's are those of test_gpu_paged.py, from the same
arithmetic.  Probabilities, in fp32: with a = (max - x) log2(e) / T the exponent,
the difference, the factor's two roundings and the product leave it off by 4 x
2^-24 of itself, so 2^-a by a relative 4 x 2^-24 ln2 a, and the function's last
step by 2^-23.  A row's sum meets each term through at most V / 1024 + 30 additions
and as many factors 2^-(a - a') of moved references, whose exponents add up to
no more than the largest a: (V / 1024 + 30) 3 x 2^-24 + 4 x 2^-24 ln2 max a.  The
division and the product add 2^-23.  Results below 2^-126 may be flushed.  Tokens,
paths, tables and moved rows are equal: the random numbers of the tests do not lie
within rounding (2^-40) of a border unless both sides are exact there.
"""
import numpy as np
import pytest
import torch

from oracle import draft as OD
from paper_2503_12450_amd import binding as B
from test_gpu_paged import DEV, TDT, Case, _f64, _i32, _normal

pytestmark = pytest.mark.gpu


def _cpu(t):
    return t.cpu().numpy()


# --------------------------------------------------------------------------
# Attention of trees
# --------------------------------------------------------------------------

def _parents(g, rows, kind):
    out = []
    for n in rows:
        for i in range(n):
            if kind == "chain":
                out.append(i - 1)
            elif kind == "tree":
                out.append(-1 if i == 0 else max(0, min(i - 1, (i - 1) // 3 + int(g.integers(-1, 2)))))
            elif kind == "any":                        # forests of any shape
                out.append(int(g.integers(-1, i)) if i else -1)
            else:                                      # nonsense among them: those hang on the past
                out.append(int(g.choice([-7, -1, i, i + 1, 300, 2 ** 31 - 1, -2 ** 31, max(0, i - 1), i // 2])))
    return np.array(out, dtype=np.int64)


class Tree(Case):
    def __init__(self, seed, rows, kv, heads, kv_heads, dh, page, dtype, kind="any", tail=0, **kw):
        super().__init__(seed, rows, kv, heads, kv_heads, dh, page, dtype, tail=tail, **kw)
        g = np.random.Generator(np.random.Philox(seed + 5))
        self.parent = np.concatenate([_parents(g, rows, kind), np.zeros(tail, dtype=np.int64)])

    def workspace(self, batch=None, window=0, sinks=0):
        n = B.paged_tree_attention_workspace_bytes(batch or self.batch(), self.m, self.heads, window, sinks)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)   # NaN in every type

    def tree_oracle(self, window=0, sinks=0):
        return OD.tree_attention(_f64(self.q).reshape(self.m, self.heads, self.dh), _f64(self.k), _f64(self.v),
                                 self.table, self.q_start, self.kv, self.parent, window, sinks, self.max_kv)

    def tree(self, window=0, sinks=0, split=True, batch=None):
        batch = batch or self.batch()
        out = torch.full((self.m, self.heads * self.dh), 7.0, dtype=TDT[self.dtype], device=DEV)
        B.k_paged_tree_attention(batch, self.q, _i32(self.parent), out, window, sinks,
                                 self.workspace(batch, window, sinks) if split else None)
        torch.cuda.synchronize()
        return out

    def verify(self, window=0, sinks=0, **kw):
        out = self.tree(window, sinks, **kw)
        self.check(out, want=self.tree_oracle(window, sinks), left=7.0)
        return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("rows,kv", [([1, 20, 5], [70, 37, 133]), ([130, 60, 90], [170, 260, 91])])
def test_tree_head_sizes(dtype, dh, rows, kv):
    Tree(dh, rows, kv, 2, 2, dh, 16, dtype).verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 1), (6, 2), (7, 1), (20, 1), (64, 2), (160, 1)])
@pytest.mark.parametrize("rows", [[1, 1], [3, 9], [40, 17]])
def test_tree_shared_heads(dtype, heads, kv_heads, rows):
    Tree(heads, rows, [50, 100], heads, kv_heads, 32, 32, dtype, "tree").verify()


EDGE = [
    ([1], [1]), ([1], [2]), ([2], [2]), ([16], [16]), ([17], [40]), ([63], [64]), ([64], [64]), ([65], [65]),
    ([64], [127]), ([64], [129]), ([200], [201]), ([256], [256]), ([255, 256], [300, 290]),
    ([257], [300]), ([300, 2, 400], [310, 5, 390]),    # nodes past the 256th are left
    ([1, 0, 2], [0, 0, 5]), ([5], [2]), ([70], [3]), ([4, 130], [-3, 1]), ([0, 0, 0, 1], [9, 9, 9, 9]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,kv", EDGE)
@pytest.mark.parametrize("kind", ["chain", "any", "wrong"])
def test_tree_short_long_and_empty(dtype, rows, kv, kind):
    """Also rows behind the last sequence, left as they were."""
    Tree(11, rows, kv, 2, 1, 32, 16, dtype, kind, tail=3).verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (3, 0), (7, 3), (16, 64), (33, 5), (100, 70), (128, 0), (300, 1),
                                          (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1)])
def test_tree_window_and_sinks(dtype, kind, window, sinks):
    """Windows shorter than the trees are deep, and first tokens inside a tree."""
    Tree(21, [1, 150, 3, 40], [290, 150, 70, 42], 2, 2, 16, 32, dtype, kind).verify(window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_chain_is_causal_attention_bit_by_bit(dtype):
    """(Without a window, which the two begin at different blocks of keys: a tile's
    nodes may all hang on the past.)"""
    c = Tree(25, [100, 1, 7], [300, 250, 60], 4, 2, 64, 16, dtype, "chain")
    assert torch.equal(c.tree(), c.run(True))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 4096])
def test_tree_page_sizes(page):
    Tree(31, [70, 1], [300, 299], 2, 1, 32, page, "bf16").verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1, 1], [20, 90]])
def test_tree_pages_that_are_none(dtype, rows):
    c = Tree(41, rows, [200, 170], 2, 2, 32, 16, dtype)
    c.table[0, 3], c.table[0, 12], c.table[1, 0], c.table[1, 8] = -1, c.k.shape[0], 2 ** 31 - 1, -5
    c.table[1, 5] = c.table[0, 4]
    c.verify()
    c.verify(60, 20)
    c.table[0, :] = -2 ** 31
    assert torch.all(c.verify()[:rows[0]] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_tree_ignores_what_other_branches_hold(dtype, bad):
    """Infinities and NaN at nodes change no bit of the rows that are not below
    them; the rows that are below are not finite."""
    c = Tree(51, [70, 3, 20], [130, 66, 20], 2, 1, 64, 32, dtype, "tree")
    clean = c.verify()
    node = 9
    t = 60 + node
    c.k[c.table[0, t // 32], 0, t % 32, 1] = bad if bad != bad else 0.0
    c.v[c.table[0, t // 32], 0, t % 32, 9] = bad
    got = _f64(c.tree()).reshape(93, 2, 64)
    below = np.array([node in OD.ancestors(c.parent, 0, i) for i in range(70)])
    assert 1 < below.sum() < 70
    same = got == _f64(clean).reshape(93, 2, 64)
    assert np.all(same[:70][~below]) and np.all(same[70:])
    assert not np.any(np.isfinite(got[:70][below][:, :, 9]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_scores_of_minus_infinity_and_large(dtype):
    """A row whose scores are all -infinity is NaN, one that sees no token zeros;
    scores in the thousands."""
    c = Tree(61, [40, 1], [200, 500], 2, 2, 64, 16, dtype, "tree")
    c.q[:20] *= 300.0
    c.q[20:30] = 0.0
    c.verify()
    c = Tree(62, [6], [6], 1, 1, 32, 16, dtype, "chain")
    c.k[c.table[0, 0], 0, :6] = -float("inf")
    c.q[:] = c.q.abs() + 1
    assert torch.isnan(c.tree()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,kv,heads,kv_heads,window", [
    ([1], [5000], 2, 1, 0), ([9, 1], [4097, 3], 4, 2, 0), ([64], [3000], 2, 2, 0), ([64], [5000], 16, 2, 0),
    ([12, 30, 1], [6000, 31, 700], 2, 1, 0), ([20], [7000], 2, 1, 3000), ([200], [2500], 1, 1, 0),
])
def test_tree_divided_among_workgroups(dtype, rows, kv, heads, kv_heads, window):
    c = Tree(71, rows, kv, heads, kv_heads, 64, 64, dtype, "tree")
    batch, want = c.batch(), c.tree_oracle(window, 4)
    out = c.tree(window, 4, batch=batch)
    c.check(out, want=want)
    assert torch.equal(out, c.tree(window, 4, batch=batch))
    c.check(c.tree(window, 4, split=False, batch=batch), want=want)
    n = B.paged_tree_attention_workspace_bytes(batch, c.m, heads, window, 4)
    for part in (n // 2 // 16 * 16, n // 5, 1):
        ws = torch.full((part + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        got = torch.empty_like(out)
        B.k_paged_tree_attention(batch, c.q, _i32(c.parent), got, window, 4, ws[:part])
        c.check(got, want=want)
        assert torch.all(ws[part:] == 0xFF)


def test_tree_many_sequences_and_max_kv():
    g = np.random.Generator(np.random.Philox(7))
    rows, kv = [int(n) for n in g.integers(0, 4, 700)], [int(n) for n in g.integers(0, 40, 700)]
    for dtype in ("bf16", "f32"):
        Tree(99, rows, kv, 1, 1, 16, 16, dtype, tail=2).verify()
    rows = [int(n) for n in g.integers(90, 150, 70)]
    Tree(100, rows, [n + int(x) for n, x in zip(rows, g.integers(0, 60, 70))], 1, 1, 16, 16, "bf16", tail=2).verify()
    Tree(81, [9, 20], [100, 65], 2, 1, 32, 16, "bf16", max_kv=60).verify()
    c = Tree(83, [20, 70], [70, 90], 2, 2, 32, 16, "bf16", tail=5)
    c.q_start = (c.q_start + 3).astype(np.int32)
    c.parent = np.roll(c.parent, 3)
    c.verify()


# --------------------------------------------------------------------------
# Probabilities
# --------------------------------------------------------------------------

def _check_probabilities(got, x, T):
    want = OD.probabilities(x, T)
    t = np.ones(len(x)) if T is None else np.asarray(T, dtype=np.float64)
    for r in range(len(x)):
        if not t[r] > 2.0 ** -100:
            assert np.array_equal(got[r], want[r])
            continue
        if np.isnan(want[r]).any():
            assert np.isnan(want[r]).all() and np.isnan(got[r]).all()
            continue
        a = np.where(x[r] > -np.inf, (x[r].max() - np.maximum(x[r], -1e300)) / t[r] / np.log(2), 0.0)
        e = 2.0 ** -24 * (4 * np.log(2) * (a + a[want[r] > 2.0 ** -126].max()) + 3 * (x.shape[1] / 1024 + 30) + 6)
        assert np.all(np.abs(got[r] - want[r]) <= e * want[r] + 2.0 ** -125), r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,V", [(1, 1), (2, 2), (3, 7), (1, 8), (5, 63), (4, 1023), (3, 1025), (7, 8191), (2, 32000),
                                 (3, 100003), (1, 2 ** 20), (600, 500)])
def test_probabilities(dtype, m, V):
    g = np.random.Generator(np.random.Philox(m + V))
    x = _normal(V, (m, V), dtype, 4.0)
    T = np.where(g.random(m) < 0.3, 0.0, 0.2 + g.random(m) * 2).astype(np.float32)
    for temp in (None, T):
        out = torch.full((m, V), 7.0, device=DEV)
        B.k_probabilities(x, out, None if temp is None else torch.tensor(temp, device=DEV))
        _check_probabilities(_f64(out), _f64(x), temp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_probabilities_on_rows_of_any_stride(dtype, off):
    m, V = 5, 3001
    wide, out = _normal(3, (m, V + 10), dtype, 3.0), torch.full((m, V + 6), 7.0, device=DEV)
    B.k_probabilities(wide[:, off:off + V], out[:, 1:1 + V])
    _check_probabilities(_f64(out[:, 1:1 + V]), _f64(wide[:, off:off + V]), None)
    assert torch.all(out[:, :1] == 7.0) and torch.all(out[:, 1 + V:] == 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_probabilities_of_strange_rows(dtype):
    inf, nan, low = float("inf"), float("nan"), torch.finfo(TDT[dtype]).min
    V = 2100
    x = _normal(5, (16, V), dtype, 2.0)
    x[0] = -inf
    x[1, :V - 1] = -inf                  # one token is left
    x[2, 5] = nan
    x[3, 2000] = inf
    x[4] = low                           # masks of the type's lowest value
    x[5, :2050] = low
    x[6] = 3.0                           # ties
    x[7, 1::2] = -inf
    x[8] *= 1000.0
    x[9:16] = x[2:9]
    T = np.ones(16, dtype=np.float32)
    T[9:16] = [0.0, -1.0, nan, 1e-35, 0.0, 0.0, 0.0]
    out = torch.empty((16, V), device=DEV)
    for temp in (T, np.zeros(16, dtype=np.float32), np.full(16, 2.0 ** -99, dtype=np.float32)):
        B.k_probabilities(x, out, torch.tensor(temp, device=DEV))
        _check_probabilities(_f64(out), _f64(x), temp)


def test_probabilities_in_place():
    x = _normal(6, (9, 5000), "f32", 2.0)
    out = torch.empty_like(x)
    B.k_probabilities(x, out)
    B.k_probabilities(x, x)
    assert torch.equal(x, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_probabilities_at_an_infinite_temperature(dtype):
    """Every finite logit weighs the same, whatever its value, and -infinity nothing."""
    inf, V = float("inf"), 2100
    big = torch.finfo(TDT[dtype]).max
    x = _normal(8, (8, V), dtype, 4.0)
    x[1, 1::2] = -inf
    x[2, :V - 1] = -inf
    x[3, ::3], x[3, 1::3], x[3, 2::3] = big, -big, -inf
    x[4] = -inf
    x[5, 7] = float("nan")
    x[6, 8] = inf
    x[7, :2050] = -big
    out = torch.empty((8, V), device=DEV)
    B.k_probabilities(x, out, torch.full((8,), inf, device=DEV))
    _check_probabilities(_f64(out), _f64(x), np.full(8, inf))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_probabilities_of_logits_across_the_whole_range(dtype):
    """Logits whose difference passes the largest fp32 number, at temperatures that it
    does not outweigh."""
    V, big = 2100, torch.finfo(TDT[dtype]).max
    x = _normal(9, (6, V), dtype, 1.0)
    x *= 0.9 * big / float(x.abs().max())
    x[1, 5], x[1, 6] = big, -big
    x[2, ::2], x[2, 1::2] = big, -big
    x[3] = -big
    x[4, 3::5] = -float("inf")
    out = torch.empty((6, V), device=DEV)
    for t in (1e38, 3.4e38, 2e37, 1.0):
        temp = np.full(6, t, dtype=np.float32)
        B.k_probabilities(x, out, torch.tensor(temp, device=DEV))
        _check_probabilities(_f64(out), _f64(x), temp)


def test_probabilities_of_more_rows_than_one_launch():
    """2^22 and three rows of 2049 tokens, in place: the rows at the borders of launches
    against the oracle, the rest (all zeros before) 1 / 2049 within the division's and
    the product's rounding; the row's sum is exact."""
    V, m = 2049, 2 ** 22 + 3
    x = torch.zeros((m, V), device=DEV)
    rows = [0, 2 ** 21 - 1, 2 ** 21, 2 ** 22 - 1, 2 ** 22, m - 1]
    some = _normal(12, (len(rows), V), "f32", 3.0)
    for k, r in enumerate(rows):
        x[r] = some[k]
    B.k_probabilities(x, x)
    _check_probabilities(np.stack([_f64(x[r]) for r in rows]), _f64(some), None)
    for r in rows:
        x[r] = 1.0 / V
    for part in x.split(2 ** 19):
        low, high = torch.aminmax(part)
        assert abs(float(low) * V - 1) <= 2.0 ** -22 and abs(float(high) * V - 1) <= 2.0 ** -22


# --------------------------------------------------------------------------
# Verification
# --------------------------------------------------------------------------

def _verify(p, q_start, parent, tokens, random=None, draft=None):
    m, V, n = p.shape[0], p.shape[1], len(q_start) - 1
    path = torch.full((m,), -2, dtype=torch.int32, device=DEV)
    kept, after = (torch.full((n,), -3, dtype=torch.int32, device=DEV) for _ in range(2))
    size = B.draft_verify_workspace_bytes(m, n, V)
    ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    B.k_draft_verify(_i32(q_start), p, _i32(parent), _i32(tokens), path, kept, after,
                     None if random is None else torch.tensor(random, dtype=torch.float32, device=DEV), draft,
                     ws[:size])
    torch.cuda.synchronize()
    assert torch.all(ws[size:] == 0xFF)
    return _cpu(path), _cpu(kept), _cpu(after)


def _same(got, want):
    for a, b, name in zip(got, want, ("path", "kept", "next")):
        assert np.array_equal(a, b), (name, a, b)


def _draws(seed, rows, V, kind, drawn, hits=0.5, tail=0):
    """Tokens that the target likes, random numbers, and probabilities that are
    multiples of 2^-12 (so that sums are exact on both sides)."""
    g = np.random.Generator(np.random.Philox(seed))
    parent = np.concatenate([_parents(g, rows, kind), np.zeros(tail, dtype=np.int64)])
    m = len(parent)

    def some():
        w = g.random((m, V)) ** 8
        w = np.floor(w / w.sum(1, keepdims=True) * 4096)
        w[:, g.integers(0, V)] += 4096 - w.sum(1)
        return (w / 4096).astype(np.float32)

    p, d = some(), some()
    if drawn:
        d = ((p + d) / 2).astype(np.float32)
    tokens = np.where(g.random(m) < hits, p[np.maximum(0, np.arange(m) - 1)].argmax(1), g.integers(0, V, m))
    random = (np.floor(g.random(m) * 2 ** 20) / 2 ** 20).astype(np.float32)
    return p, d, parent, tokens, random


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["points", "drawn", "greedy"])
@pytest.mark.parametrize("rows,V,kind", [
    ([1], 1, "chain"), ([2, 3], 2, "chain"), ([1, 0, 4, 9], 7, "chain"), ([5] * 40, 64, "chain"),
    ([30, 64, 65, 3], 100, "tree"), ([300, 130], 50, "any"), ([12, 20, 7], 1023, "tree"), ([8, 9], 1025, "wrong"),
    ([6, 1, 11], 5003, "tree"), ([9] * 3, 40000, "chain"), ([4, 3], 2 ** 20, "tree"),
    ([3] * 200, 20000, "tree"), ([1, 2] * 40, 16385, "chain"),
])
def test_verification(dtype, mode, rows, V, kind):
    p, d, parent, tokens, random = _draws(len(rows) + V, rows, V, kind, mode == "drawn", tail=2)
    q_start = np.concatenate([[0], np.cumsum(rows)])
    tp, td = (torch.tensor(x).to(TDT[dtype]).to(DEV) for x in (p, d))
    draft = td if mode == "drawn" else None
    args = q_start, parent, tokens, None if mode == "greedy" else random
    got = _verify(tp, *args, draft)
    _same(got, OD.verify(_f64(tp), *args, None if draft is None else _f64(td)))
    again = _verify(tp, *args, draft)
    _same(again, got)


@pytest.mark.parametrize("mode", ["points", "drawn"])
def test_verification_of_many_children(mode):
    """Stars: up to 400 children of one node, the same token several times."""
    for seed, n, V in ((1, 400, 900), (2, 70, 20), (3, 9, 3000)):
        p, d, parent, tokens, random = _draws(seed, [n, n // 2], V, "chain", mode == "drawn", hits=0.0)
        parent = np.where(np.concatenate([np.arange(n), np.arange(n // 2)]) == 0, -1, 0)
        random = np.maximum(random, 0.5).astype(np.float32)
        tp, td = torch.tensor(p, device=DEV), torch.tensor(d, device=DEV) if mode == "drawn" else None
        q_start = [0, n, n + n // 2]
        _same(_verify(tp, q_start, parent, tokens, random, td),
              OD.verify(p, q_start, parent, tokens, random, d if mode == "drawn" else None))


def test_verification_at_the_borders():
    """Random numbers on the borders between tokens, of 0, at 1 and past it, and
    none at all; weights that are 0 around the border."""
    V = 1500
    p = np.zeros((12, V), dtype=np.float32)
    p[:, [3, 700, 1023, 1024, 1499]] = [0.25, 0.25, 0.125, 0.125, 0.25]
    p[10] = 0.0                                             # nothing
    p[11], p[11, 4] = 0.0, 1.0
    r = np.array([0, 0.25, 0.5, 0.625, 0.75, 1.0, 5.0, np.nan, -1.0, 0.9999999, 0.5, 0.5], dtype=np.float32)
    q_start = np.arange(13)
    want = [3, 700, 1023, 1024, 1499, 1499, 1499, 1499, 3, 1499, -1, 4]
    tokens, parent = np.zeros(12, dtype=np.int64), np.full(12, -1)
    got = _verify(torch.tensor(p, device=DEV), q_start, parent, tokens, r)
    assert got[2].tolist() == want and got[1].tolist() == [1] * 12
    _same(got, OD.verify(p, q_start, parent, tokens, r))
    # chains of two: r W < w at and below the border
    q_start, parent = np.array([0, 2, 4, 6, 8, 10, 12]), np.array([-1, 0] * 6)
    tokens = np.array([0, 3, 0, 3, 0, 3, 0, 4, 0, -1, 0, V])
    r = np.array([0, 0.25, 0, 0.2499999, 0, np.nan, 0, 0, 0, 0, 0, 0], dtype=np.float32)
    got = _verify(torch.tensor(p, device=DEV), q_start, parent, tokens, r)
    assert got[1].tolist() == [1, 2, 1, 1, 1, 1]
    _same(got, OD.verify(p, q_start, parent, tokens, r))


@pytest.mark.parametrize("mode", ["points", "drawn", "greedy"])
def test_verification_of_what_is_no_probability(mode):
    g = np.random.Generator(np.random.Philox(9))
    rows, V = [5, 9, 1, 6], 300
    p, d, parent, tokens, random = _draws(19, rows, V, "tree", True)
    for x in (p, d):
        x[g.random(x.shape) < 0.05] = np.nan
        x[g.random(x.shape) < 0.05] = -1.0
        if mode != "greedy":
            x[g.random(x.shape) < 0.05] = np.inf
    p[3] = np.nan
    q_start = np.concatenate([[0], np.cumsum(rows)])
    tokens[4], tokens[7], tokens[9] = -5, V, 2 ** 31 - 1
    args = q_start, parent, tokens, None if mode == "greedy" else random
    tp, td = torch.tensor(p, device=DEV), torch.tensor(d, device=DEV) if mode == "drawn" else None
    _same(_verify(tp, *args, td), OD.verify(p, *args, d if mode == "drawn" else None))


@pytest.mark.parametrize("mode", ["points", "drawn"])
@pytest.mark.parametrize("V", [400, 30000])
def test_random_numbers_that_are_none(mode, V):
    """Of 1, above it, negative, infinite or NaN: the definition as it stands, no token
    without weight."""
    g = np.random.Generator(np.random.Philox(41))
    rows = [9, 1, 20, 6]
    p, d, parent, tokens, random = _draws(43, rows, V, "tree", True)
    random[g.random(len(random)) < 0.7] = np.nan
    odd = g.random(len(random)) < 0.5
    random[odd] = g.choice([1.0, 7.0, -1.0, -np.inf, np.inf, 1e30], int(odd.sum()))
    q_start = np.concatenate([[0], np.cumsum(rows)])
    td = torch.tensor(d, device=DEV) if mode == "drawn" else None
    got = _verify(torch.tensor(p, device=DEV), q_start, parent, tokens, random, td)
    _same(got, OD.verify(p, q_start, parent, tokens, random, d if mode == "drawn" else None))
    for s, n in enumerate(rows):
        line = got[0][q_start[s]:q_start[s] + got[1][s]] + q_start[s]
        assert np.all(p[line[:-1], tokens[line[1:]]] > 0) and p[line[-1], got[2][s]] > 0


@pytest.mark.parametrize("mode", ["points", "drawn"])
@pytest.mark.parametrize("V", [2000, 30000])
def test_verification_where_the_draft_is_the_target(mode, V):
    """Drafts of a one-token target, and a draft equal to it whose token is refused
    by a random number of 1: what is left is empty, and the weights stay."""
    p = np.zeros((6, V), dtype=np.float32)
    p[:, 1111] = 1.0
    p[3:, 1111], p[3:, 7] = 0.5, 0.5
    q_start, parent = np.array([0, 3, 6]), np.array([-1, 0, 0, -1, 0, 0])
    tokens, random = np.array([0, 1111, 1111, 0, 7, 7]), np.array([0.9, 1.0, 1.0, 0.9, 1.0, 1.0], dtype=np.float32)
    d = p if mode == "drawn" else None
    got = _verify(torch.tensor(p, device=DEV), q_start, parent, tokens, random,
                  torch.tensor(p, device=DEV) if mode == "drawn" else None)
    _same(got, OD.verify(p, q_start, parent, tokens, random, d))
    assert got[2].tolist() == ([-1, 1111] if mode == "points" else [1111, 1111])


@pytest.mark.parametrize("mode", ["points", "drawn"])
def test_kept_tokens_are_distributed_as_the_target(mode):
    """60000 sequences with two children each: how often each token comes first is
    within five standard deviations of its probability."""
    n, V = 60000, 5
    p = np.array([0.4, 0.3, 0.15, 0.1, 0.05])
    d = np.array([0.1, 0.5, 0.2, 0.1, 0.1])
    g = np.random.Generator(np.random.Philox(77))
    tokens = np.zeros((n, 3), dtype=np.int64)
    tokens[:, 1:] = g.choice(V, (n, 2), p=d) if mode == "drawn" else [1, 0]
    full = torch.tensor(np.tile(p.astype(np.float32), (3 * n, 1)), device=DEV)
    draft = torch.tensor(np.tile(d.astype(np.float32), (3 * n, 1)), device=DEV) if mode == "drawn" else None
    path, kept, after = _verify(full, np.arange(n + 1) * 3, np.tile([-1, 0, 0], n), tokens.reshape(-1),
                                g.random(3 * n), draft)
    child = tokens[np.arange(n), np.maximum(path.reshape(n, 3)[:, 1], 0)]
    first = np.where(kept > 1, child, after)
    share = np.bincount(first, minlength=V) / n
    assert np.all(np.abs(share - p) < 5 * np.sqrt(p * (1 - p) / n))
    second = np.bincount(after[kept > 1], minlength=V) / (kept > 1).sum()   # after a kept one: p again
    assert np.all(np.abs(second - p) < 5 * np.sqrt(p * (1 - p) / (kept > 1).sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_greedy_takes_the_first_of_equals(dtype):
    V = 3000
    x = torch.zeros((4, V), dtype=TDT[dtype], device=DEV)
    x[0, [2999, 17, 1500]] = 5.0
    x[1, 0] = x[1, 2999] = float("inf")
    x[2] = -float("inf")
    x[3] = -2.0
    got = _verify(x, [0, 4], [-1, 0, 1, 2], [0, 17, 0, 5])
    assert [g.tolist() for g in got] == [[0, 1, 2, -1], [3], [-1]]
    got = _verify(x, [0, 4], [-1, 0, 0, 2], [0, 1500, 17, 5])
    assert [g.tolist() for g in got] == [[0, 2, -1, -1], [2], [-1]]
    got = _verify(x, [0, 1, 2, 3, 4], [-1] * 4, [0] * 4)
    assert got[2].tolist() == [17, 0, -1, 0]


def test_nothing_to_verify_or_keep():
    """No rows at all: every sequence keeps nothing and has no next token; lengths
    stay."""
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    for V in (5, 40000):
        p, ws = torch.empty((0, V), device=DEV), torch.empty(B.draft_verify_workspace_bytes(0, 3, V), dtype=torch.uint8,
                                                             device=DEV)
        for r, d in ((None, None), (torch.empty(0, device=DEV), None), (torch.empty(0, device=DEV), p)):
            kept, after = (torch.full((3,), 9, dtype=torch.int32, device=DEV) for _ in range(2))
            B.k_draft_verify(_i32([0, 0, 0, 0]), p, none, none, none.clone(), kept, after, r, d, ws)
            assert kept.tolist() == [0, 0, 0] and after.tolist() == [-1, -1, -1]
        B.k_probabilities(p, p.clone())
    c = Case(3, [0, 0], [20, 40], 1, 1, 16, 16, "bf16")
    kv = torch.zeros(2, dtype=torch.int32, device=DEV)
    B.k_paged_keep(c.batch(), none, _i32([5, 5]), kv)
    assert kv.tolist() == [20, 40]


@pytest.mark.parametrize("mode", ["points", "drawn", "greedy"])
def test_verification_on_rows_of_any_stride(mode):
    rows, V = [5, 9, 1, 6], 1501
    p, d, parent, tokens, random = _draws(29, rows, V, "tree", True)
    q_start = np.concatenate([[0], np.cumsum(rows)])
    wide = torch.full((21, V + 9), float("nan"), device=DEV)
    wide[:, 3:3 + V] = torch.tensor(p)
    other = torch.full((21, 2 * V), float("nan"), device=DEV)
    other[:, 1:1 + V] = torch.tensor(d)
    args = q_start, parent, tokens, None if mode == "greedy" else random
    drawn = mode == "drawn"
    _same(_verify(wide[:, 3:3 + V], *args, other[:, 1:1 + V] if drawn else None), OD.verify(p, *args, d if drawn else None))


# --------------------------------------------------------------------------
# Rows moved together, sequences continued by others
# --------------------------------------------------------------------------

def _bits(t):
    return t.cpu().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


def _paths(g, rows):
    path, kept = [], []
    for n in rows:
        a = int(g.integers(0, n + 1))
        path += sorted(g.permutation(n)[:a].tolist()) + [-1] * (n - a)
        kept.append(a)
    return path, kept


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dh,page,rows,kv", [
    (1, 16, 16, [1], [1]), (2, 32, 16, [5, 1, 0, 9], [40, 1, 7, 9]), (3, 48, 32, [64, 30], [100, 31]),
    (2, 80, 16, [300], [310]), (1, 128, 64, [20, 20, 20], [200, 21, 64]), (2, 112, 16, [40], [45]),
    (2, 64, 16, [9, 30], [4, 20]),       # nodes before the first token have no place
    (4096, 16, 16, [3] * 600, [5] * 600),   # more workgroups than one launch
])
def test_keeping(dtype, heads, dh, page, rows, kv):
    g = np.random.Generator(np.random.Philox(dh + len(rows)))
    big = heads > 100
    c = Case(dh, rows, kv, heads, heads, dh, page, dtype, tail=2, filled=not big)
    path, kept = _paths(g, rows)
    path += [1, 0]
    if not big:
        c.table[0, 0] = -1 if len(rows) > 1 else c.table[0, 0]
        pk, pv = _bits(c.k).copy(), _bits(c.v).copy()
        left = OD.keep([pk, pv], c.table, c.q_start, c.kv, path, kept)
    else:
        where = torch.arange(c.k.shape[0] * 16, device=DEV).view(-1, 1, 16, 1).to(c.k.dtype)
        c.k[:], c.v[:] = where, -where
        small_k, small_v = _bits(c.k[:, :1, :, :1]).copy(), _bits(c.v[:, :1, :, :1]).copy()
        left = OD.keep([small_k, small_v], c.table, c.q_start, c.kv, path, kept)
    kv_out = torch.full((len(rows),), -9, dtype=torch.int32, device=DEV)
    B.k_paged_keep(c.batch(), _i32(path), _i32(kept), kv_out)
    torch.cuda.synchronize()
    assert np.array_equal(_cpu(kv_out), left)
    if not big:
        assert np.array_equal(_bits(c.k), pk) and np.array_equal(_bits(c.v), pv)
    else:
        for t, small in ((c.k, small_k), (c.v, small_v)):
            want = torch.tensor(small).view(t.dtype).to(DEV)
            assert bool((t == want).all())


def test_keeping_with_nonsense_on_the_device():
    """Paths out of order or outside the sequence name rows that are not moved;
    nothing else changes."""
    rows, kv = [8, 8, 8], [40, 24, 60]
    c = Case(5, rows, kv, 2, 2, 32, 16, "bf16")
    path = [0, -1, 9, 2 ** 31 - 1, 1, 5, 6, 7,  -2 ** 31, 3, 1, 1, 4, 7, 2, 0,  7, 7, 7, 7, 7, 7, 7, 7]
    kept = [8, 2 ** 31 - 1, 1]
    pk, pv = _bits(c.k).copy(), _bits(c.v).copy()
    left = OD.keep([pk, pv], c.table, c.q_start, c.kv, path, kept)
    kv_out = torch.zeros(3, dtype=torch.int32, device=DEV)
    B.k_paged_keep(c.batch(), _i32(path), _i32(kept), kv_out)
    assert np.array_equal(_cpu(kv_out), left)
    assert np.array_equal(_bits(c.k), pk) and np.array_equal(_bits(c.v), pv)


def _fork(c, source, keep=None, add=None):
    n, batch = len(source), c.batch()
    table = torch.full((n, c.table.shape[1]), -7, dtype=torch.int32, device=DEV)
    kv = torch.full((n,), -7, dtype=torch.int32, device=DEV)
    missing = torch.full((1,), -7, dtype=torch.int32, device=DEV)
    size = B.paged_fork_workspace_bytes(batch, n)
    ws = torch.full((size + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    B.k_paged_fork(batch, _i32(source), table, kv, missing, *(None if x is None else _i32(x) for x in (keep, add)),
                   workspace=ws[:size])
    torch.cuda.synchronize()
    assert torch.all(ws[size:] == 0x5A)
    return _cpu(table), _cpu(kv), int(missing)


def _check_fork(c, source, keep=None, add=None):
    pk, pv = _bits(c.k).copy(), _bits(c.v).copy()
    table, kv, missing = OD.fork([pk, pv], c.table, c.kv, source, keep, add, c.max_kv)
    got = _fork(c, source, keep, add)
    assert np.array_equal(got[0], table) and np.array_equal(got[1], kv) and got[2] == missing, (got, table, kv, missing)
    assert np.array_equal(_bits(c.k), pk) and np.array_equal(_bits(c.v), pv)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seed", range(6))
def test_forking(dtype, seed):
    """Sequences continued by any number of others, cut short and lengthened,
    from a pool that suffices or not."""
    g = np.random.Generator(np.random.Philox(seed))
    S = int(g.integers(1, 9))
    kv = [int(x) for x in g.integers(-2, 90, S)]
    page, dh, heads = int(g.choice([16, 32])), int(g.choice([16, 48, 128])), int(g.choice([1, 3]))
    c = Case(seed + 200, [0] * S, kv, heads, heads, dh, page, dtype, spare=int(g.integers(0, 60)),
             max_kv=None if seed % 2 else 70)
    c.table = np.concatenate([c.table, np.full((S, 3), -1, dtype=np.int32)], 1)
    for n in (1, 2 * S, 23):
        source = g.integers(-1, S + 1, n)
        _check_fork(c, source, None, None)
        _check_fork(c, source, None, g.integers(-1, 40, n))
        _check_fork(c, source, g.integers(-5, 100, n), g.integers(0, 3, n))


def test_forking_keeps_the_page_of_the_only_writer():
    c = Case(7, [0, 0], [20, 40], 1, 1, 16, 16, "bf16", spare=6)
    t = c.table
    got, kv, missing = _check_fork(c, [0, 1], None, [5, 9])
    assert np.array_equal(got[0, :2], t[0, :2]) and np.array_equal(got[1, :3], t[1, :3]) and missing == 0
    got, _, _ = _check_fork(c, [1, 1], None, [5, 9])          # both write: the first keeps it
    assert got[0, 2] == t[1, 2] != got[1, 2]
    got, _, _ = _check_fork(c, [1, 1], None, [0, 9])          # one reads on: the writer copies
    assert got[0, 2] == t[1, 2] != got[1, 2]
    got, _, _ = _check_fork(c, [1, 1], [40, 32], [0, 9])      # a full page needs no copy
    assert got[1, 1] == t[1, 1] and got[1, 2] not in t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,n_pages", [(1, 3), (5, 6), (5, 40), (1024, 8192), (1025, 2000), (9, 8193)])
def test_forking_a_batch_without_sequences(dtype, n, n_pages):
    """The first sequences of an empty pool, in the form that plans in one workgroup and in
    the other: no table and no lengths are there to be read."""
    page, width = 16, 3
    k = torch.full((n_pages, 1, page, 16), 3.0, dtype=TDT[dtype], device=DEV)
    v = torch.full_like(k, 4.0)
    empty = torch.zeros((0, width), dtype=torch.int32, device=DEV)
    batch = B.PagedBatch(B.MarPages(k, v), empty, _i32([0]), _i32(np.zeros(0)), max_kv=width * page)
    g = np.random.Generator(np.random.Philox(n))
    source, keep, add = g.integers(-1, 3, n), g.integers(-1, 70, n), g.integers(-1, 70, n)
    for some in ((None, None), (None, add), (keep, None), (keep, add)):
        want = OD.fork([_bits(k), _bits(v)], _cpu(empty), [], source, *some, width * page)
        table = torch.full((n, width), -7, dtype=torch.int32, device=DEV)
        kv, missing = (torch.full((x,), -7, dtype=torch.int32, device=DEV) for x in (n, 1))
        ws = torch.empty(B.paged_fork_workspace_bytes(batch, n), dtype=torch.uint8, device=DEV)
        B.k_paged_fork(batch, _i32(source), table, kv, missing, *(None if x is None else _i32(x) for x in some),
                       workspace=ws)
        torch.cuda.synchronize()
        assert np.array_equal(_cpu(table), want[0]) and np.array_equal(_cpu(kv), want[1]) and int(missing) == want[2]
    assert torch.all(k == 3.0) and torch.all(v == 4.0)


def test_forking_many_and_much():
    """More rows than a step of the plan, more pages than one too, nonsense in the
    tables."""
    g = np.random.Generator(np.random.Philox(13))
    S = 1500
    kv = [int(x) for x in g.integers(0, 60, S)]
    c = Case(300, [0] * S, kv, 1, 1, 16, 16, "bf16", spare=4000, filled=False)
    c.k.normal_(), c.v.normal_()
    bad = g.random(c.table.shape) < 0.05
    c.table[bad] = g.choice([-1, -2 ** 31, 2 ** 31 - 1, c.k.shape[0]], int(bad.sum()))
    source = g.integers(0, S, 2500)
    _check_fork(c, source, None, g.integers(0, 30, 2500))
    edge = np.array([-2 ** 31, -1, 0, 1, 2 ** 30, 2 ** 31 - 1])
    _check_fork(c, g.choice(edge, 50), g.choice(edge, 50), g.choice(edge, 50))
    _check_fork(c, g.integers(0, S, 50), g.choice(edge, 50), g.choice(edge, 50))
    assert _fork(c, [])[2] == 0


def test_pages_past_32_bit_offsets():
    """A cache of more than 2^32 bytes, the pages of the sequences at its end: read,
    moved and copied there as in a small one."""
    Hk, page, dh = 2, 128, 128
    n_pages = (2 ** 32 // (Hk * page * dh * 2)) + 70
    k = torch.empty((n_pages, Hk, page, dh), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    c = Tree(95, [9, 33], [200, 300], 2, 2, dh, page, "bf16", "tree", spare=6)
    n = c.k.shape[0]
    k[n_pages - n:], v[n_pages - n:] = c.k, c.v
    big = B.PagedBatch(B.MarPages(k, v), _i32(np.where(c.table >= 0, c.table + n_pages - n, -1)), _i32(c.q_start),
                       _i32(c.kv))
    assert torch.equal(c.tree(batch=big), c.tree())
    path = [0, 3, 5, 8] + [-1] * 5 + [1, 7, 30] + [-1] * 30
    out = [torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2)]
    for b, kv in zip((big, c.batch()), out):
        B.k_paged_keep(b, _i32(path), _i32([4, 3]), kv)
    assert torch.equal(*out)
    # all the small pages but the sequences' own are the lowest free ones of both: of the
    # big cache's, the ones before them are taken by a third sequence's table
    rest = np.arange(n_pages - n, dtype=np.int32)
    wide = np.full((3, len(rest)), -1, dtype=np.int32)
    wide[:2, :c.table.shape[1]] = np.where(c.table >= 0, c.table + n_pages - n, -1)
    wide[2] = rest
    kv_len = _i32([200, 300, len(rest) * page])
    big = B.PagedBatch(B.MarPages(k, v), _i32(wide), _i32([0, 9, 42, 42]), kv_len)
    table, kv, missing = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((3, len(rest)), (3,), (1,)))
    ws = torch.empty(B.paged_fork_workspace_bytes(big, 3), dtype=torch.uint8, device=DEV)
    B.k_paged_fork(big, _i32([0, 0, 1]), table, kv, missing, add=_i32([1, 1, 1]), workspace=ws)
    got = _fork(c, [0, 0, 1], None, [1, 1, 1])
    small = _cpu(table)[:, :c.table.shape[1]]
    assert np.array_equal(np.where(small >= 0, small - (n_pages - n), -1), got[0]) and int(missing) == got[2] == 0
    assert torch.equal(k[n_pages - n:].view(torch.int16), c.k.view(torch.int16))
    assert torch.equal(v[n_pages - n:].view(torch.int16), c.v.view(torch.int16))


# --------------------------------------------------------------------------
# Together
# --------------------------------------------------------------------------

class Step:
    """A step of trees, as a serving program runs it."""

    def __init__(self, dtype="bf16", rows=(9, 20, 1), past=(30, 100, 64), V=700, H=4, Hk=2, dh=32, page=16):
        g = np.random.Generator(np.random.Philox(3))
        self.c = c = Tree(400, list(rows), [a + b for a, b in zip(rows, past)], H, Hk, dh, page, dtype, "tree", spare=20)
        c.table = np.concatenate([c.table, np.full((len(rows), 4), -1, dtype=np.int32)], 1)
        self.V, self.S = V, len(rows)
        self.qkv = _normal(5, (c.m, (H + 2 * Hk) * dh), dtype)
        self.logits = _normal(6, (c.m, V), dtype, 3.0)
        up = np.maximum(c.parent, 0) + np.repeat(c.q_start[:-1], rows)
        self.tokens = self.logits.float().argmax(1)[torch.tensor(up, device=DEV)].to(torch.int32)
        self.parent = _i32(c.parent)
        self.random = torch.tensor(g.random(c.m), dtype=torch.float32, device=DEV)
        self.temperature = torch.tensor([0.5, 0.0, 1.0] * c.m, device=DEV)[:c.m].contiguous()
        depth = [len(OD.ancestors(c.parent, int(s), i)) - 1 + p for s, n, p in zip(c.q_start, rows, past)
                 for i in range(n)]
        self.pos = _i32(depth)[:, None].contiguous()
        self.rot = B.Rotary(*B.rotary_sections((dh // 2,), device=DEV), 1)
        self.batch = c.batch()
        n = lambda *shape, t=torch.int32: torch.zeros(shape, dtype=t, device=DEV)
        self.q, self.out = n(c.m, H * dh, t=TDT[dtype]), n(c.m, H * dh, t=TDT[dtype])
        self.p = n(c.m, V, t=torch.float32)
        self.path, self.kept, self.next, self.kv = n(c.m), n(self.S), n(self.S), n(self.S)
        self.ws = c.workspace(self.batch)
        self.scratch = n(B.draft_verify_workspace_bytes(c.m, self.S, V), t=torch.uint8)
        self.source, self.add = _i32(range(self.S)), _i32([len(r) if hasattr(r, "__len__") else r for r in rows])
        self.table2, self.kv2, self.missing = n(*c.table.shape), n(self.S), n(1)
        # the lengths that the fork goes by are those that the rows moved together leave
        self.batch2 = B.PagedBatch(self.batch.pages, self.batch.table, self.batch.q_start, self.kv)
        self.fork_ws = n(B.paged_fork_workspace_bytes(self.batch2, self.S), t=torch.uint8)

    def run(self, stream=None):
        c, kw = self.c, dict(stream=stream)
        H, Hk, dh = c.heads, c.kv_heads, c.dh
        x = self.qkv
        B.k_paged_store(self.batch, x[:, H * dh:(H + Hk) * dh], x[:, (H + Hk) * dh:], q=x[:, :H * dh], q_out=self.q,
                        rotary=self.rot, pos=self.pos, **kw)
        B.k_paged_tree_attention(self.batch, self.q, self.parent, self.out, workspace=self.ws, **kw)
        B.k_probabilities(self.logits, self.p, self.temperature, **kw)
        B.k_draft_verify(self.batch.q_start, self.p, self.parent, self.tokens, self.path, self.kept, self.next,
                         random=self.random, workspace=self.scratch, **kw)
        B.k_paged_keep(self.batch, self.path, self.kept, self.kv, **kw)
        B.k_paged_fork(self.batch2, self.source, self.table2, self.kv2, self.missing, add=self.add,
                       workspace=self.fork_ws, **kw)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.out, self.p, self.path, self.kept, self.next, self.kv, self.table2, self.kv2,
                                    self.missing, self.c.k, self.c.v)]

    def same(self, a, b):
        for x, y in zip(a, b):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_of_all_of_them(dtype):
    """Each call reads what the one before left; against the oracle of each, and
    the next step's attention sees the kept tokens alone."""
    st = Step(dtype)
    c = st.c
    st.run()
    out, p, path, kept, after, kv, table2, kv2, missing, k, v = st.results()
    _check_probabilities(_f64(p), _f64(st.logits), _cpu(st.temperature))
    want = OD.verify(_f64(p), c.q_start, c.parent, _cpu(st.tokens), _cpu(st.random))
    _same((_cpu(path), _cpu(kept), _cpu(after)), want)
    assert int(kept.max()) > 2
    # once more up to the attention, which leaves the pages as the store does
    x = st.qkv
    H, Hk, dh = c.heads, c.kv_heads, c.dh
    B.k_paged_store(st.batch, x[:, H * dh:(H + Hk) * dh], x[:, (H + Hk) * dh:], q=x[:, :H * dh], q_out=st.q,
                    rotary=st.rot, pos=st.pos)
    c.q = st.q
    c.check(out, want=c.tree_oracle())
    pk, pv = _bits(c.k).copy(), _bits(c.v).copy()
    assert np.array_equal(_cpu(kv), OD.keep([pk, pv], c.table, c.q_start, c.kv, want[0], want[1]))
    t2, l2, miss = OD.fork([pk, pv], c.table, _cpu(kv), range(st.S), None, _cpu(st.add))
    assert np.array_equal(_cpu(table2), t2) and np.array_equal(_cpu(kv2), l2) and int(missing) == miss == 0
    assert np.array_equal(_bits(k), pk) and np.array_equal(_bits(v), pv)


def test_a_step_captured_and_replayed():
    """Twice the same graph's work on buffers of their own, replayed in turn with
    the program's own work between; every replay as the eager call."""
    a, b = Step("bf16"), Step("bf16", rows=(30, 5), past=(400, 70))
    wants = []
    for st in (a, b):
        st.run()
        wants.append(st.results())
    graphs = []
    for st in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    for _ in range(3):
        for st, g, want in zip((a, b), graphs, wants):
            for t in (st.out, st.p, st.path, st.kept, st.next, st.kv, st.table2, st.kv2, st.missing):
                t.fill_(1)
            st.ws.fill_(0x33), st.scratch.fill_(0x44), st.fork_ws.fill_(0x55)
            g.replay()
            st.same(st.results(), want)
        torch.randn(1000, device=DEV).sum().item()
    a.run()
    a.same(a.results(), wants[0])


def test_a_step_on_another_stream():
    st = Step("bf16")
    st.run()
    want = st.results()
    for t in (st.out, st.p, st.path, st.kept, st.next, st.kv, st.table2):
        t.zero_()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    st.run(stream=other)
    torch.cuda.current_stream().wait_stream(other)
    st.same(st.results(), want)


def test_nonsense_on_the_device_stays_inside_the_buffers():
    """Starts that do not ascend, parents, tokens, lengths, tables and paths of any
    value: nothing around the buffers changes.  (Every index is bounded in the
    kernels.)"""
    for dtype, seqs, m in (("bf16", 5, 40), ("f32", 5, 700), ("bf16", 90, 300)):
        g = np.random.Generator(np.random.Philox(seqs + m))
        H, Hk, dh, page, n_pages, V = 4, 2, 32, 16, 11, 130
        edge = np.array([-2 ** 31, -1, 0, 1, 5, m - 1, m, m + 1, 2 ** 30, 2 ** 31 - 1])
        mix = lambda shape, most, share=0.5: _i32(np.where(g.random(shape) < share, g.choice(edge, shape),
                                                           g.integers(0, most, shape)))
        q_start, kv_len, table = mix(seqs + 1, m), mix(seqs, 2000), mix((seqs, 40), n_pages, 0.3)
        parent, tokens, path_in, kept_in = mix(m, 20), mix(m, V), mix(m, 20), mix(seqs, 20)

        def guarded(shape, t):
            n = int(np.prod(shape))
            whole = torch.full((n + 2048,), 7, dtype=t, device=DEV)
            return whole, whole[1024:-1024].view(shape)

        t, i32 = TDT[dtype], torch.int32
        made = [guarded((n_pages, Hk, page, dh), t), guarded((n_pages, Hk, page, dh), t), guarded((m, H * dh), t),
                guarded((m,), i32), guarded((seqs,), i32), guarded((seqs,), i32), guarded((seqs,), i32),
                guarded((seqs, 40), i32), guarded((1,), i32)]
        k, v, out, path, kept, after, kv, table2, missing = (x for _, x in made)
        k.normal_(), v.normal_()
        batch = B.PagedBatch(B.MarPages(k, v), table, q_start, kv_len)
        sizes = (B.paged_tree_attention_workspace_bytes(batch, m, H), B.draft_verify_workspace_bytes(m, seqs, V),
                 B.paged_fork_workspace_bytes(batch, seqs))
        rooms = [torch.full((n + 4096,), 0x55, dtype=torch.uint8, device=DEV) for n in sizes]
        q, p = _normal(6, (m, H * dh), dtype), torch.softmax(_normal(7, (m, V), "f32"), 1)
        random = torch.rand(m, device=DEV)
        for window in (0, 50):
            B.k_paged_tree_attention(batch, q, parent, out, window, 3, rooms[0][:sizes[0]])
            B.k_paged_tree_attention(batch, q, parent, out, window, 3)
        for r, d in ((random, None), (random, p), (None, None)):
            B.k_draft_verify(q_start, p, parent, tokens, path, kept, after, r, d, rooms[1][:sizes[1]])
            assert bool(((after >= -1) & (after < V)).all())
        B.k_paged_keep(batch, path, kept, kv)
        B.k_paged_keep(batch, path_in, kept_in, kv)
        B.k_paged_fork(batch, mix(seqs, seqs), table2, kv, missing, mix(seqs, 600), mix(seqs, 600),
                       rooms[2][:sizes[2]])
        torch.cuda.synchronize()
        for whole, _ in made:
            assert torch.all(whole[:1024] == 7) and torch.all(whole[-1024:] == 7)
        for n, ws in zip(sizes, rooms):
            assert torch.all(ws[n:] == 0x55)
