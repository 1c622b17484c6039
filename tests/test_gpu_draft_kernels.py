"""Each kernel of the attention of trees at every head size, window and sinks, the
launched one asserted, with keys that are divided and keys that are not, and tokens
that are not finite where no row sees them.

The reference is one softmax in fp64 over a mask of every pair of row and token,
pinned here on oracle/draft.py; tolerances are those of test_gpu_paged.py.
"""
import ctypes
import re

import numpy as np
import pytest
import torch

from oracle import draft as OD
from paper_2503_12450_amd import binding as B
from test_gpu_draft import Tree
from test_gpu_paged import DEV, _f64, _i32

pytestmark = pytest.mark.gpu

# (rows, kv) per sequence: nodes past the 256th, none, one; last tiles of 128 rows with
# 2 to 88 of them; more than 2560 keys, which are divided
BATCH = ([64, 1, 130, 0, 256, 300], [700, 50, 260, 9, 5900, 310])
SHORTER = (BATCH[0], [700, 50, 260, 9, 4100, 310])   # tiles of 32 rows at every head size
ORDERS = [(0, 0), (100, 0), (100, 70), (3, 1), (64, 1), (1, 200)]
FAR = 1 << 17   # a bound of the lengths that asks for tiles of 128 rows


def _tree(seed, heads, kv_heads, dh, page, dtype, batch=BATCH, max_kv=None, kind="any"):
    c = Tree(seed, *batch, heads, kv_heads, dh, page, dtype, kind, tail=1, max_kv=max_kv)
    if max_kv:
        more = max_kv // page - c.table.shape[1]
        c.table = np.concatenate([c.table, np.full((len(batch[0]), more), -1, dtype=np.int32)], 1)
    return c


def _seen(c, window, sinks):
    """Of every sequence: the rows that are nodes, and which tokens each sees."""
    for s, (n, L) in enumerate(zip(c.rows, c.kv)):
        start, first = int(c.q_start[s]), L - n
        nodes = min(n, OD.MOST_NODES)
        seen = np.zeros((nodes, max(L, 0)), dtype=bool)
        j = np.arange(max(L, 0))
        for i in range(nodes):
            line = OD.ancestors(c.parent, start, i)
            pos = first + len(line) - 1
            seen[i] = (j < first) & ((j > pos - window) | (j < sinks) if window else True)
            for up, a in enumerate(line):
                if 0 <= first + a < L and (not window or up < window or pos - up < sinks):
                    seen[i, first + a] = True
        yield s, slice(start, start + nodes), seen


def _dense(c, window, sinks):
    group, page = c.heads // c.kv_heads, c.k.shape[2]
    o = torch.full((c.m, c.heads, c.dh), float("nan"), dtype=torch.float64, device=DEV)
    mean_abs, reach = torch.zeros_like(o), torch.zeros((c.m, c.heads), dtype=torch.float64, device=DEV)
    q = c.q.double().view(c.m, c.heads, c.dh)
    for s, r, seen in _seen(c, window, sinks):
        if not seen.size:
            o[r] = 0.0
            continue
        seen = torch.tensor(seen, device=DEV)
        token = torch.arange(seen.shape[1], device=DEV)
        at = torch.tensor(c.table[s].astype(np.int64), device=DEV)[token // page], token % page
        used = seen.any(0)[:, None]
        for h in range(c.heads):
            k, v = (torch.where(used, x[at[0], h // group, at[1]].double(), 0.0) for x in (c.k, c.v))
            score = ((q[r, h] @ k.T.contiguous()) / c.dh ** 0.5).masked_fill(~seen, -torch.inf)
            w = torch.where(seen, torch.exp(score - score.amax(1, True)), 0.0)   # rows that see nothing: 0 / 0
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
            o[r, h], mean_abs[r, h] = w @ v, w @ v.abs()
            size = (q[r, h].abs() @ k.abs().T.contiguous()) / c.dh ** 0.5
            reach[r, h] = size.masked_fill(~seen, 0.0).amax(1)
    return o.cpu().numpy(), mean_abs.cpu().numpy(), reach.cpu().numpy()


@pytest.mark.parametrize("window,sinks", ORDERS)
def test_the_reference_is_the_oracle(window, sinks):
    c = _tree(7, 4, 2, 16, 16, "f32", ([5, 40, 0], [30, 40, 3]))
    for mine, theirs in zip(_dense(c, window, sinks), c.tree_oracle(window, sinks)):
        assert np.allclose(mine, theirs, rtol=1e-12, atol=1e-13, equal_nan=True)


def _launches(c, path, *order):
    """The kernels that one call launches: the nodes of a graph that it is captured
    into (and that never runs)."""
    batch, out, parent = c.batch(), torch.empty_like(c.q), _i32(c.parent)
    ws = c.workspace(batch, *order)
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.k_paged_tree_attention(batch, c.q, parent, out, *order, ws)
    with open("/proc/self/maps") as f:
        hip = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    assert hip.hipGraphDebugDotPrint(ctypes.c_void_p(graph.raw_cuda_graph()), str(path).encode(), ctypes.c_uint(1)) == 0
    return re.findall(r"4tree.{0,16}_1\d(attn_[a-z0-9]+)I(\S+?)E+vNS", path.read_text())


def _check(c, path, kernel, order):
    assert _launches(c, path, *order)[0] == kernel
    out = c.tree(*order)
    c.check(out, want=_dense(c, *order), left=7.0)
    assert torch.equal(out, c.tree(*order))
    return out


@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("order", ORDERS)
def test_tiles_of_128_rows(dh, order, tmp_path):
    c = _tree(dh, 4, 2, dh, 16 if dh % 32 else 64, "bf16", max_kv=FAR)
    _check(c, tmp_path / "g", ("attn_many", f"Li{dh}ELi{3 if dh <= 96 else 2}"), order)


@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("order", [(0, 0), (100, 70)])
def test_tiles_of_32_rows(dh, order, tmp_path):
    c = _tree(dh, 4, 2, dh, 16 if dh % 32 else 64, "bf16", SHORTER)
    _check(c, tmp_path / "g", ("attn_few", f"Li{dh}"), order)


@pytest.mark.parametrize("dh", [16, 64, 80, 128])
@pytest.mark.parametrize("order", [(0, 0), (100, 70), (3, 1)])
def test_fp32_tiles_of_32_rows(dh, order, tmp_path):
    c = _tree(dh, 32, 32, dh, 32, "f32")
    _check(c, tmp_path / "g", ("attn_f32", f"Li{dh}ELi2"), order)


@pytest.mark.parametrize("dh,kernel", [(64, ("attn_many", "Li64ELi3")), (128, ("attn_many", "Li128ELi2"))])
@pytest.mark.parametrize("rows,kv", [([64], [9000]), ([64, 20, 90], [9000, 300, 2600]), ([250], [2561])])
def test_divided_keys(dh, kernel, rows, kv, tmp_path):
    """Tiles whose keys are in several parts beside such as write out themselves, the
    workspace of NaN; without one, and with half of it."""
    c = _tree(61, 8, 1, dh, 64, "bf16", (rows, kv), max_kv=FAR, kind="tree")
    out = _check(c, tmp_path / "g", kernel, (0, 0))
    assert [name for name, _ in _launches(c, tmp_path / "h", 0, 0)] == ["attn_many", "attn_join"]
    want = _dense(c, 0, 0)
    c.check(c.tree(split=False), want=want, left=7.0)
    batch, got = c.batch(), torch.full_like(out, 7.0)
    ws = c.workspace(batch)
    B.k_paged_tree_attention(batch, c.q, _i32(c.parent), got, workspace=ws[:ws.numel() // 2])
    c.check(got, want=want, left=7.0)


@pytest.mark.parametrize("dtype,heads,max_kv,kernel", [
    ("bf16", 2, FAR, ("attn_many", "Li64ELi3")), ("bf16", 2, None, ("attn_few", "Li64")),
    ("f32", 32, None, ("attn_f32", "Li64ELi2")),
])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_tokens_that_no_row_or_few_rows_see(dtype, heads, max_kv, kernel, bad, tmp_path):
    """Infinities and NaN in tokens that no row sees change no bit; in one value of a
    node they reach the rows below it, in that column alone."""
    order = (40, 5)
    c = _tree(51, heads, heads, 64, 32, dtype, max_kv=max_kv, kind="tree")
    clean = _check(c, tmp_path / "g", kernel, order)
    page = c.k.shape[2]
    for s, r, seen in _seen(c, *order):
        for t in range(c.kv[s]):
            if not seen[:, t].any():
                c.k[c.table[s, t // page], :, t % page] = c.v[c.table[s, t // page], :, t % page] = bad
    assert torch.equal(c.tree(*order), clean)
    node, head = 7, heads - 1   # of the third sequence
    t = c.kv[2] - c.rows[2] + node
    c.v[c.table[2, t // page], head, t % page, 9] = bad
    got, was = (_f64(x).reshape(c.m, heads, 64) for x in (c.tree(*order), clean))
    hit = np.zeros(got.shape, dtype=bool)
    first = int(c.q_start[2])
    below = [i for i in range(c.rows[2]) if node in OD.ancestors(c.parent, first, i)]
    assert len(below) > 1
    hit[[first + i for i in below], head, 9] = True
    assert not np.any(np.isfinite(got[hit])) and np.all(got[~hit] == was[~hit])


@pytest.mark.parametrize("dtype,n", [("bf16", 1100), ("bf16", 950), ("f32", 1100)])
def test_more_tiles_than_one_launch(dtype, n):
    """Sequences of two nodes that both hang on nothing, 4096 heads: either side of 2^22
    workgroups.  A row's own token is its answer, or its parent's too: the mean of
    both, as all scores are 0."""
    H, dh = 4096, 16
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    k = torch.zeros((n, H, 16, dh), dtype=t, device=DEV)
    v = torch.full_like(k, float("nan"))
    g = torch.Generator(device=DEV).manual_seed(98)
    want = torch.randn((2 * n, H, dh), generator=g, device=DEV).to(t)
    v[:, :, 0], v[:, :, 1] = want[0::2], want[1::2]
    q = torch.randn((2 * n, H * dh), generator=g, device=DEV).to(t)
    out, i = torch.empty_like(q), np.arange(n)
    batch = B.PagedBatch(B.MarPages(k, v), _i32(i[:, None]), _i32(2 * np.arange(n + 1)), _i32(np.full(n, 2)))
    B.k_paged_tree_attention(batch, q, torch.full((2 * n,), -1, dtype=torch.int32, device=DEV), out)
    assert torch.equal(out, want.view(2 * n, -1))
    B.k_paged_tree_attention(batch, q, _i32(np.tile([-1, 0], n)), out)
    assert torch.equal(out[0::2], want[0::2].reshape(n, -1))
    mean = (want[0::2].float() + want[1::2].float()) / 2
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23   # the output's rounding (f32: two sums'); the 1% holds those of 32 bits
    assert torch.all((out[1::2].float() - mean.view(n, -1)).abs() <= half * mean.view(n, -1).abs() * 1.01 + 1e-38)
