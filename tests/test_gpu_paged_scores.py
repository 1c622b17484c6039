"""Attention over the paged cache where scores are large: a softmax depends on
differences of scores alone, whatever their size, and equal scores have equal
weights in every block of keys, wave and part.

The scores here are exact: one or two columns of q and k are not zero, their
products and sums have at most 24 bits.  So what `test_gpu_paged.py` allows for
the rounding of a score (relative to its size) does not apply, and tolerances
are relative to differences of scores.  A difference of d (log2 units) carries
a rounded scale, product and difference, 3 x 2^-24 of itself, and its exponential
2^-22; weights below 2^-25 do not show in bf16, those above have d <= 25: a weight
is off by e = 25 x 3 x 2^-24 + 2^-22 < 2^-17 of itself, in the first block and in
any other.  Numerator and denominator carry it, their sums over L keys
L 2^-23, the weights' rounding in bf16 2^-8 (equal weights none: they are rounded
alike), the result half a step.  fp32 rounds the scaled score itself; its weights
are tested where all of them are equal or zero.
"""
import numpy as np
import pytest
import torch

from test_gpu_paged import DEV, HALF_STEP, TDT, Case, _f64

pytestmark = pytest.mark.gpu

# few rows, several blocks to each wave; many rows; keys divided among workgroups
FORMS = {"few": ([3, 5], [700, 650]), "many": ([250, 300], [700, 650]), "parts": ([1], [5000])}
PAGE, TOKENS = 128, 5120


def _case(form, dh, dtype):
    return Case(63, *FORMS[form], 2, 1, dh, PAGE, dtype)


def _scores(c, q, k):
    """Scores q . k of the leading columns, for every row: q a list, k [TOKENS,
    columns]."""
    c.q.zero_()
    c.q.view(c.m, 2, c.dh)[:, :, :len(q)] = torch.tensor(q, dtype=torch.float64).to(TDT[c.dtype]).to(DEV)
    rows = torch.zeros((TOKENS // PAGE, PAGE, c.dh), dtype=TDT[c.dtype])
    rows[..., :len(q)] = torch.tensor(k).to(TDT[c.dtype]).view(-1, PAGE, len(q))
    for s, n in enumerate(c.kv):
        pages = -(-n // PAGE)
        c.k[torch.tensor(c.table[s, :pages].astype(np.int64), device=DEV), 0] = rows[:pages].to(DEV)


def _want(c, k_score):
    """Mean of the values weighted by exp(k_score), and of their sizes."""
    v = _f64(c.v)
    out, size = np.zeros((c.m, 2, c.dh)), np.zeros((c.m, 2, c.dh))
    for s, n in enumerate(c.kv):
        w = np.exp(k_score[:n] - k_score[:n].max())
        w /= w.sum()
        t = np.arange(n)
        vs = v[c.table[s][t // PAGE], 0, t % PAGE]
        r = slice(c.q_start[s], c.q_start[s + 1])
        out[r], size[r] = w @ vs, w @ np.abs(vs)
    return out, size


def _check(c, k_score, weights=0.0):
    want, size = _want(c, k_score)
    got = _f64(c.run(False)).reshape(want.shape)
    tol = size * (2 * 2.0 ** -17 + max(c.kv) * 2.0 ** -23 + weights)
    assert np.all(np.abs(got - want) <= tol + HALF_STEP[c.dtype] * (np.abs(want) + tol))


# products of the two, from 2^12 to near the end of fp32; scaled, in log2 units, most
# are past 2^24
PAIRS = [(14528.0, 15232.0), (57600.0, 46848.0), (413696.0, 272384.0), (28288.0, 28544.0), (30080.0, 29952.0),
         (2.0 ** 10, 2.0 ** 10), (130.0, 150.0), (2.0 ** 61 * 1.25, 2.0 ** 50 * 1.75), (2.0 ** 64, 2.0 ** 62)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_scores_of_any_size(dtype, form, dh, sign):
    """The mean of the values, to the last bit that its rounding leaves."""
    c = _case(form, dh, dtype)
    for q, k in PAIRS:
        _scores(c, [q], np.full((TOKENS, 1), sign * k))
        _check(c, np.zeros(TOKENS))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("q", [2.0, 2.0 ** 9, 2.0 ** 16, 2.0 ** 18, -2.0 ** 18, 2.0 ** 60])
def test_scores_that_change_from_block_to_block(dtype, form, q):
    """Groups of 100 keys whose scores rise, fall and repeat, 22 and more apart:
    the largest groups share the weight."""
    level = np.array([129, 137, 131, 145, 129, 145, 133])[np.arange(TOKENS) // 100 % 7].astype(np.float64)
    c = _case(form, 32, dtype)
    _scores(c, [8.0 * q], level[:, None])
    _check(c, 8.0 * q * level / 32 ** 0.5)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("q,k,unit", [(2 ** 5, 2 ** 5, 1), (2 ** 10, 2 ** 10, 1), (2 ** 13, 2 ** 14, 16),
                                      (181 * 64, 181 * 128, 16)])
def test_small_differences_of_large_scores(form, sign, q, k, unit):
    """q k + unit j with j of 0 to 6, exact: of the size 2^10, 2^20 and past 2^27,
    where a step of fp32 is 16; weights exp(unit j / 8)."""
    j = np.random.Generator(np.random.Philox(1)).integers(0, 7, TOKENS).astype(np.float64)
    c = _case(form, 64, "bf16")
    _scores(c, [sign * q, unit], np.stack([np.full(TOKENS, float(k)), j], 1))
    _check(c, unit * j / 8, weights=2.0 ** -8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_scores_of_minus_infinity(dtype, form):
    """Keys of -infinity have no weight; rows whose keys all are, and those alone,
    are 0 / 0; rows that see no token stay zeros."""
    c = _case(form, 64, dtype)
    inf = np.full((TOKENS, 1), -np.inf)
    _scores(c, [1.0], inf)
    assert torch.isnan(c.run(False)).all() and torch.isnan(c.run(True, 40, 3)).all()
    for at in ([0], [33], [600], [5, 333, 600]):
        k = inf.copy()
        k[at] = 2.0
        _scores(c, [1.0], k)
        _check(c, k[:, 0])
    # causal, with a window: rows before token 400 and from 440 on see keys of
    # -infinity alone
    k = inf.copy()
    k[400:410] = 1.0
    _scores(c, [1.0], k)
    out = c.run(True, 31, 0)
    for s, n in enumerate(c.kv):
        rows = slice(c.q_start[s], c.q_start[s + 1])
        p = torch.arange(n - c.rows[s], n, device=DEV)
        assert torch.equal(~torch.isnan(out[rows]).any(1), (p >= 400) & (p < 440))
    c.table[:] = -1
    assert torch.all(c.run(False) == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_values_up_to_the_bound(dtype, form):
    """Equal values of the largest size that the header names, 2^118 / (kv_len +
    32), under weights that grow by 2^7.7 behind the first blocks: they are their
    own mean."""
    c = _case(form, 64, dtype)
    k = np.where(np.arange(TOKENS) < 100, 0.0, 43.0)[:, None]
    _scores(c, [1.0], k)
    size = 2.0 ** np.floor(np.log2(2.0 ** 118 / (max(c.kv) + 32)))
    c.v.copy_(torch.where(torch.isnan(c.v), c.v, size))
    _check(c, k[:, 0] / 8)
    c.v.neg_()
    _check(c, k[:, 0] / 8)
