"""Each kernel of the attention over the paged cache at sizes far from where the
choice between them changes: every head size, order, window and sinks, tokens
that are not finite where no row sees them, divided keys.

The reference is one softmax in fp64 over a mask of every pair of row and token,
pinned here on oracle/paged.py; tolerances are those of test_gpu_paged.py.
"""
import ctypes
import re

import numpy as np
import pytest
import torch

from paper_2503_12450_amd import binding as B
from test_gpu_paged import DEV, Case, _f64

pytestmark = pytest.mark.gpu

# (rows, kv) per sequence.  More than 200 packed rows a sequence: 128 of them to a
# tile; with 16 heads the fp32 tiles have 32 rows, and last ones of 1, 17, 15 and 32
MANY = ([300, 1, 257, 0, 530], [700, 50, 257, 9, 900])
WIDE = ([385, 401, 399, 416], [450, 401, 600, 420])

ORDERS = [(True, 0, 0), (False, 0, 0), (True, 100, 0), (True, 100, 70), (False, 150, 64), (True, 64, 1), (True, 1, 200),
          (False, 33, 0)]


def _dense(c, causal, window, sinks):
    """What `Case.oracle` returns, by one mask of all pairs."""
    group = c.heads // c.kv_heads
    page = c.k.shape[2]
    o = torch.full((c.m, c.heads, c.dh), float("nan"), dtype=torch.float64, device=DEV)
    mean_abs, reach = torch.zeros_like(o), torch.zeros((c.m, c.heads), dtype=torch.float64, device=DEV)
    q = c.q.double().view(c.m, c.heads, c.dh)
    for s, (n, L) in enumerate(zip(c.rows, c.kv)):
        r = slice(int(c.q_start[s]), int(c.q_start[s]) + n)
        p = torch.arange(L - n, L, device=DEV)[:, None]
        j = torch.arange(L, device=DEV)[None]
        seen = (j <= p) if causal else torch.ones((n, L), dtype=torch.bool, device=DEV)
        if window:
            seen = seen & ((j > p - window) | (j < sinks))
        table = torch.tensor(c.table[s].astype(np.int64), device=DEV)
        at = table[torch.arange(L, device=DEV) // page], torch.arange(L, device=DEV) % page
        used = seen.any(0)[:, None]
        for h in range(c.heads):
            k, v = (torch.where(used, x[at[0], h // group, at[1]].double(), 0.0) for x in (c.k, c.v))
            score = (q[r, h] @ k.T.contiguous()) / c.dh ** 0.5
            w = torch.exp(score.masked_fill(~seen, -torch.inf) - score.masked_fill(~seen, -torch.inf).amax(1, True))
            w = torch.where(seen, w, 0.0)   # rows that see nothing: 0 / 0 above
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
            o[r, h], mean_abs[r, h] = w @ v, w @ v.abs()
            size = (q[r, h].abs() @ k.abs().T.contiguous()) / c.dh ** 0.5
            if n and L:
                reach[r, h] = size.masked_fill(~seen, 0.0).amax(1)
    return o.cpu().numpy(), mean_abs.cpu().numpy(), reach.cpu().numpy()


@pytest.mark.parametrize("causal,window,sinks", ORDERS)
def test_the_reference_is_the_oracle(causal, window, sinks):
    c = Case(7, [5, 40, 0], [30, 40, 3], 4, 2, 16, 16, "f32", tail=1)
    for mine, theirs in zip(_dense(c, causal, window, sinks), c.oracle(causal, window, sinks)):
        assert np.allclose(mine, theirs, rtol=1e-12, atol=1e-13, equal_nan=True)


def _launches(c, path, *order):
    """The kernels that one call launches: the nodes of a graph that it is captured
    into (and that never runs)."""
    batch, out = c.batch(), torch.empty_like(c.q)
    ws = c.workspace(batch, *order[1:])
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.k_paged_attention(batch, c.q, out, *order, ws)
    with open("/proc/self/maps") as f:
        hip = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    assert hip.hipGraphDebugDotPrint(ctypes.c_void_p(graph.raw_cuda_graph()), str(path).encode(), ctypes.c_uint(1)) == 0
    return re.findall(r"_1\d(attn_[a-z0-9]+)I(\S+?)E+vNS", path.read_text())


def _spoil(c, causal, window, sinks, bad):
    """Keys and values that no row of their sequence sees, and the rest of its last
    page, become `bad`."""
    page = c.k.shape[2]
    for s, (n, L) in enumerate(zip(c.rows, c.kv)):
        p = L - n + np.arange(n)[:, None]
        j = np.arange(c.table.shape[1] * page)[None]
        seen = (j < L) & ((j <= p) if causal else True) & ((j > p - window) | (j < sinks) if window else True)
        for t in np.nonzero(~seen.any(0))[0]:
            at = c.table[s, t // page]
            if at >= 0:
                c.k[at, :, t % page], c.v[at, :, t % page] = bad, bad


def _run_and_check(c, path, kernel, order):
    """Against the reference; the rest of the last pages holds NaN (`Case`)."""
    assert _launches(c, path, *order)[0] == kernel
    out = c.run(*order)
    c.check(out, want=_dense(c, *order))
    return out


@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("order", ORDERS)
def test_tiles_of_many_rows(dh, order, tmp_path):
    ring = 3 if dh <= 96 else 2
    c = Case(dh, *MANY, 4, 2, dh, 16 if dh % 32 else 64, "bf16", tail=1)
    _run_and_check(c, tmp_path / "g", ("attn_many", f"Li{dh}ELi{ring}"), order)


@pytest.mark.parametrize("dh", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("order", [(True, 0, 0), (False, 0, 0), (True, 100, 70), (False, 150, 64)])
def test_fp32_tiles_of_32_rows(dh, order, tmp_path):
    c = Case(dh, *WIDE, 16, 16, dh, 32, "f32", tail=1)
    _run_and_check(c, tmp_path / "g", ("attn_f32", f"Li{dh}ELi2"), order)


@pytest.mark.parametrize("dtype,dh,heads,batch,kernel", [
    ("bf16", 64, 2, MANY, ("attn_many", "Li64ELi3")), ("bf16", 80, 2, MANY, ("attn_many", "Li80ELi3")),
    ("bf16", 128, 2, MANY, ("attn_many", "Li128ELi2")), ("f32", 64, 16, WIDE, ("attn_f32", "Li64ELi2")),
])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_tokens_that_no_row_or_few_rows_see(dtype, dh, heads, batch, kernel, bad, tmp_path):
    """Infinities and NaN in tokens that no row sees change no bit; in one value
    inside the window they reach the rows that see it, in that column alone."""
    order = (True, 40, 5)
    c = Case(51, *batch, heads, heads, dh, 32, dtype)
    clean = _run_and_check(c, tmp_path / "g", kernel, order)
    _spoil(c, *order, bad)
    assert torch.equal(c.run(*order), clean)
    t, head = c.kv[0] - 60, heads - 1   # rows at t .. t + 39 of the first sequence see it
    c.v[c.table[0, t // 32], head, t % 32, 9] = bad
    got, was = (_f64(x).reshape(c.m, heads, dh) for x in (c.run(*order), clean))
    p = c.kv[0] - c.rows[0] + np.arange(c.rows[0])
    hit = np.zeros(got.shape, dtype=bool)
    hit[:c.rows[0], head, 9] = (p >= t) & (p < t + 40)
    assert not np.any(np.isfinite(got[hit])) and np.all(got[~hit] == was[~hit])


@pytest.mark.parametrize("rows,kv,order,kernel", [
    ([300], [4000], (True, 3000, 5), ("attn_many", "Li128ELi2")), ([260], [5000], (False, 0, 0), ("attn_many", "Li128ELi2")),
    ([3], [9000], (True, 0, 0), ("attn_few", "Li128")), ([20, 1], [3000, 9000], (True, 2000, 70), ("attn_few", "Li128")),
])
def test_divided_keys_of_wide_heads(rows, kv, order, kernel, tmp_path):
    c = Case(61, rows, kv, 2, 1, 128, 64, "bf16")
    _run_and_check(c, tmp_path / "g", kernel, order)
    assert [name for name, _ in _launches(c, tmp_path / "h", *order)] == [kernel[0], "attn_join"]
