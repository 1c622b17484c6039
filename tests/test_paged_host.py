"""The paged cache's oracle against plain dense forms, and the refusals of the
entry points, all on the CPU: every check is made on the host before anything
is enqueued, so the pointers here are never followed."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged as OP
from oracle.mar_oracle import attention as dense_attention
from paper_2503_12450_amd import binding as B


def test_oracle_over_pages_is_dense_attention():
    """One sequence in pages in a shuffled order, every key seen: the slot
    attention's oracle on the keys laid out densely."""
    g = np.random.Generator(np.random.Philox(3))
    H, dh, page, L = 3, 16, 16, 53
    q, k, v = (g.standard_normal((L, H, dh)) for _ in range(3))
    table = g.permutation(6)[:4][None].astype(np.int32)
    pk, pv = np.zeros((6, H, page, dh)), np.zeros((6, H, page, dh))
    OP.store(pk, pv, k, v, table, np.array([0, L]), np.array([L]))
    o, _, _ = OP.attention(q, pk, pv, table, np.array([0, L]), np.array([L]), causal=False)
    for h in range(H):
        np.testing.assert_allclose(o[:, h], dense_attention(q[:, h], k[:, h], v[:, h]), atol=1e-12)


def test_oracle_masks_are_the_definitions():
    """Causal with a window and sinks, shared heads: against one softmax over a
    mask of every pair."""
    g = np.random.Generator(np.random.Philox(4))
    H, Hk, dh, L, n, W, sinks = 4, 2, 16, 40, 25, 7, 3
    q, k, v = g.standard_normal((n, H, dh)), g.standard_normal((L, Hk, dh)), g.standard_normal((L, Hk, dh))
    table = np.arange(3, dtype=np.int32)[None]
    pk, pv = np.zeros((3, Hk, 16, dh)), np.zeros((3, Hk, 16, dh))
    OP.store(pk, pv, k, v, table, np.array([0, L]), np.array([L]))
    o, _, _ = OP.attention(q, pk, pv, table, np.array([0, n]), np.array([L]), True, W, sinks)
    p = L - n + np.arange(n)[:, None]
    j = np.arange(L)[None]
    seen = (j <= p) & ((j > p - W) | (j < sinks))
    for h in range(H):
        s = np.where(seen, q[:, h] @ k[:, h // 2].T / 4.0, -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        np.testing.assert_allclose(o[:, h], (w / w.sum(1, keepdims=True)) @ v[:, h // 2], atol=1e-12)


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_oracle_rotation_keeps_relative_positions(layout):
    """A rotation is orthogonal and its scores depend on position differences
    alone, axis by axis; negated frequencies undo it."""
    g = np.random.Generator(np.random.Philox(5))
    q, k = g.standard_normal((1, 1, 32)), g.standard_normal((1, 1, 32))
    freq, axis = (t.numpy() for t in B.rotary_sections((5, 11), device="cpu"))
    at = lambda x, *p: OP.rotary(x, np.array([p]), freq, axis, layout)
    a = (at(q, 7, 100) * at(k, 3, 90)).sum()
    b = (at(q, 7 + 20, 100 - 40) * at(k, 3 + 20, 90 - 40)).sum()
    assert abs(a - b) < 1e-12 and abs(a - (q * k).sum()) > 1e-3
    back = OP.rotary(at(q, 7, 100), np.array([(7, 100)]), -freq, axis, layout)
    np.testing.assert_allclose(back, q, atol=1e-13)


def test_sections():
    freq, axis = B.rotary_sections((2, 4), base=100.0, device="cpu")
    assert axis.tolist() == [0, 0, 1, 1, 1, 1]
    np.testing.assert_allclose(freq, [1, 0.1, 1, 100 ** -0.25, 0.1, 100 ** -0.75])
    freq, axis = B.rotary_sections((2, 2), base=16.0, shared=True, device="cpu")
    assert axis.tolist() == [0, 0, 1, 1]
    np.testing.assert_allclose(freq, [1, 0.5, 0.25, 0.125])


# --------------------------------------------------------------------------
# Refusals through the C entry points
# --------------------------------------------------------------------------

PTR = 4096  # a non-NULL, aligned address that no check may follow


def _rot(**kw):
    f = dict(freq=PTR, axis=PTR, n_pairs=32, n_axes=2, layout=0)
    f.update(kw)
    return B.MarRotaryC(**f)


def _batch(**kw):
    f = dict(k=PTR, v=PTR, table=PTR, q_start=PTR, kv_len=PTR, n_pages=10, n_heads=2, page=16, d_head=64, n_seqs=3,
             max_pages=4, max_kv=64)
    f.update(kw)
    return B.MarPagedBatchC(**f)


def _rotary_call(rot=None, **kw):
    a = dict(dtype=1, x=PTR, ld_x=128, pos=PTR, m=5, n_heads=2, d_head=64, out=2 * PTR, ld_out=128)
    a.update(kw)
    rot = _rot() if rot is None else rot
    return B.load().mar_k_rotary(a["dtype"], ctypes.byref(rot) if rot else None, a["x"], a["ld_x"], a["pos"], a["m"],
                                 a["n_heads"], a["d_head"], a["out"], a["ld_out"], None)


def _store_call(batch=None, rot=None, **kw):
    a = dict(dtype=1, pos=PTR, m=5, k=PTR, ld_k=128, v=PTR, ld_v=128, hq=4, q=PTR, ld_q=256, q_out=2 * PTR, ld_o=256)
    a.update(kw)
    batch, rot = _batch() if batch is None else batch, _rot() if rot is None else rot
    return B.load().mar_k_paged_store(a["dtype"], ctypes.byref(batch) if batch else None, ctypes.byref(rot) if rot else None, a["pos"],
                                      a["m"], a["k"], a["ld_k"], a["v"], a["ld_v"], a["hq"], a["q"], a["ld_q"],
                                      a["q_out"], a["ld_o"], None)


def _attention_call(batch=None, **kw):
    a = dict(dtype=1, m=5, hq=4, q=PTR, ld_q=256, causal=1, window=0, sinks=0, ws=None, ws_bytes=0, out=2 * PTR,
             ld_o=256)
    a.update(kw)
    batch = _batch() if batch is None else batch
    return B.load().mar_k_paged_attention(a["dtype"], ctypes.byref(batch) if batch else None, a["m"], a["hq"], a["q"],
                                          a["ld_q"], a["causal"], a["window"], a["sinks"], a["ws"], a["ws_bytes"],
                                          a["out"], a["ld_o"], None)


ARG, SHAPE, WS = B.MAR_E_ARG, B.MAR_E_SHAPE, B.MAR_E_WORKSPACE

BAD_ROWS = [dict(ld=127), dict(ld=120), dict(ld=0), dict(ld=-128), dict(ld=1 << 31)]


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=2)), (ARG, dict(x=None)), (ARG, dict(out=None)), (ARG, dict(pos=None)), (ARG, dict(x=PTR + 8)),
    (ARG, dict(out=PTR + 2)), (SHAPE, dict(m=-1)), (SHAPE, dict(n_heads=0)), (SHAPE, dict(d_head=24)),
    (SHAPE, dict(d_head=144)), (SHAPE, dict(d_head=0)), (SHAPE, dict(m=1 << 29)),
    (ARG, dict(out=PTR, ld_out=256)), (ARG, dict(rot=False)),
    (ARG, dict(rot=_rot(freq=None))), (ARG, dict(rot=_rot(axis=None))), (SHAPE, dict(rot=_rot(n_pairs=40))),
    (SHAPE, dict(rot=_rot(n_pairs=12))), (SHAPE, dict(rot=_rot(n_pairs=0))), (SHAPE, dict(rot=_rot(n_pairs=-8))),
    (SHAPE, dict(rot=_rot(n_axes=0))), (SHAPE, dict(rot=_rot(n_axes=5))), (ARG, dict(rot=_rot(layout=2))),
] + [(SHAPE, dict(ld_x=b["ld"])) for b in BAD_ROWS] + [(SHAPE, dict(ld_out=b["ld"])) for b in BAD_ROWS])
def test_rotary_refuses(status, kw):
    assert _rotary_call(**kw) == status
    assert B.load().mar_last_error()


BAD_BATCH = [
    (SHAPE, dict(d_head=72)), (SHAPE, dict(n_heads=0)), (SHAPE, dict(n_heads=4097)), (SHAPE, dict(n_seqs=-1)), (SHAPE, dict(n_seqs=65537)),
    (SHAPE, dict(page=24)), (SHAPE, dict(page=8)), (SHAPE, dict(page=8192)), (SHAPE, dict(page=0)),
    (SHAPE, dict(page=-16)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(max_pages=0)), (SHAPE, dict(max_kv=65)),
    (SHAPE, dict(max_kv=0)), (SHAPE, dict(max_pages=1 << 27)), (ARG, dict(k=None)), (ARG, dict(v=None)),
    (ARG, dict(table=None)), (ARG, dict(q_start=None)), (ARG, dict(kv_len=None)), (ARG, dict(k=PTR + 4)),
    (ARG, dict(v=PTR + 8)),
]


@pytest.mark.parametrize("status,kw", BAD_BATCH)
def test_store_and_attention_refuse_a_batch(status, kw):
    assert _store_call(batch=_batch(**kw)) == status
    assert _attention_call(batch=_batch(**kw)) == status
    lib = B.load()
    assert lib.mar_k_paged_attention_workspace_bytes(1, ctypes.byref(_batch(**kw)), 5, 4, 0, 0) == 0
    assert lib.mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=-1)), (ARG, dict(batch=False)), (ARG, dict(k=None)), (ARG, dict(v=None)),
    (ARG, dict(q_out=None)), (SHAPE, dict(hq=0)), (SHAPE, dict(ld_k=64)), (SHAPE, dict(ld_v=132)),
    (SHAPE, dict(ld_q=128)), (SHAPE, dict(ld_o=250)), (SHAPE, dict(m=-3)), (ARG, dict(k=PTR + 8)),
    (ARG, dict(q_out=PTR, ld_o=264)), (ARG, dict(pos=None)), (SHAPE, dict(rot=_rot(n_pairs=48))),
])
def test_store_refuses(status, kw):
    assert _store_call(**kw) == status
    assert B.load().mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=7)), (ARG, dict(batch=False)), (SHAPE, dict(hq=3)), (SHAPE, dict(hq=0)), (SHAPE, dict(hq=1)),
    (SHAPE, dict(m=-1)), (ARG, dict(q=None)), (ARG, dict(out=None)), (ARG, dict(out=PTR)), (SHAPE, dict(ld_q=255)),
    (SHAPE, dict(ld_o=248)), (ARG, dict(window=-1)), (ARG, dict(sinks=-1)), (WS, dict(ws=None, ws_bytes=64)),
    (WS, dict(ws=PTR + 4, ws_bytes=64)), (SHAPE, dict(m=1 << 28)),
])
def test_attention_refuses(status, kw):
    assert _attention_call(**kw) == status
    assert B.load().mar_last_error()


def test_nothing_to_do_is_not_an_error():
    """No rows, or no sequences: nothing is enqueued and no pointer is followed."""
    assert _rotary_call(m=0, x=None, out=None, pos=None) == B.MAR_OK
    assert _store_call(m=0, k=None, v=None, q=None, q_out=None, pos=None) == B.MAR_OK
    assert _store_call(batch=_batch(n_seqs=0, table=None, kv_len=None)) == B.MAR_OK
    assert _attention_call(m=0, q=None, out=None) == B.MAR_OK
    assert _attention_call(batch=_batch(n_seqs=0, table=None, kv_len=None)) == B.MAR_OK


# --------------------------------------------------------------------------
# Refusals of the binding
# --------------------------------------------------------------------------

def test_binding_refuses_what_the_library_cannot_see():
    pages = B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 32))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    table = torch.zeros((2, 2), dtype=torch.int32)
    batch = B.PagedBatch(pages, table, i32(0, 1, 2), i32(3, 4))
    assert batch.c.max_kv == 32
    rot = B.Rotary(*B.rotary_sections((8, 8), device="cpu"), 2)
    x, pos = torch.zeros(2, 64), torch.zeros((2, 2), dtype=torch.int32)
    bad = [
        lambda: B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 16)),
        lambda: B.MarPages(torch.zeros(4, 2, 16, 32).half(), torch.zeros(4, 2, 16, 32).half()),
        lambda: B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 32).bfloat16()),
        lambda: B.MarPages(torch.zeros(4, 2, 16, 64)[..., :32], torch.zeros(4, 2, 16, 32)),
        lambda: B.PagedBatch(pages, table.long(), i32(0, 1, 2), i32(3, 4)),
        lambda: B.PagedBatch(pages, table, i32(0, 2), i32(3, 4)),
        lambda: B.PagedBatch(pages, table, i32(0, 1, 2), i32(3)),
        lambda: B.PagedBatch(pages, table[:, ::2], i32(0, 1, 2), i32(3, 4)),
        lambda: B.Rotary(rot.freq.float(), rot.axis, 2),
        lambda: B.Rotary(rot.freq, rot.axis[:8], 2),
        lambda: B.Rotary(rot.freq, rot.axis.long(), 2),
        lambda: B.Rotary(rot.freq, rot.axis, 2, "thirds"),
        lambda: B.k_rotary(rot, x, pos, x[:, :32], 32),             # widths differ
        lambda: B.k_rotary(rot, x, pos, x.bfloat16(), 32),          # types differ
        lambda: B.k_rotary(rot, x, pos[:, :1], x, 32),              # axes differ
        lambda: B.k_rotary(rot, x, pos[:1], x, 32),                 # rows differ
        lambda: B.k_rotary(rot, x.t(), pos, x.t(), 2),              # columns not dense
        lambda: B.k_rotary(rot, x, pos, x, 48),                     # no whole heads
        lambda: B.k_rotary(rot, x, pos, x, 0),
        lambda: B.k_rotary(rot, x, pos, x, 32),                     # not on a GPU
        lambda: B.k_paged_store(batch, x, x[:, :32]),               # value heads
        lambda: B.k_paged_store(batch, x.bfloat16(), x.bfloat16()), # not the pages' type
        lambda: B.k_paged_store(batch, x, x, q=x),                  # no q_out
        lambda: B.k_paged_store(batch, x, x, rotary=rot),           # no pos
        lambda: B.k_paged_store(batch, x, x),                       # not on a GPU
        lambda: B.k_paged_attention(batch, x, x[:1]),               # rows differ
        lambda: B.k_paged_attention(batch, x.double(), x.double()),
        lambda: B.k_paged_attention(batch, x, torch.zeros(2, 64), workspace=torch.zeros(8, 2)[:, :1]),
        lambda: B.k_paged_attention(batch, x, torch.zeros(2, 64)),  # not on a GPU
        lambda: B.paged_attention_workspace_bytes(batch, 2, 3),
    ]
    for call in bad:
        with pytest.raises(B.MarError):
            call()


def test_binding_refuses_what_32_bits_do_not_hold():
    """ctypes keeps the lower 32 bits of an int: a window of 2^32 + 5 would be one
    of 5."""
    pages = B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 32))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    table = torch.zeros((2, 2), dtype=torch.int32)
    batch = B.PagedBatch(pages, table, i32(0, 1, 2), i32(3, 4))
    rows, far = torch.zeros(2, 64), 2 ** 32
    one = torch.zeros(1, 64).expand(far + 2, 64)   # rows without memory of their own
    bad = [
        lambda: B.PagedBatch(pages, table, i32(0, 1, 2), i32(3, 4), max_kv=far + 5),
        lambda: B.Rotary(*B.rotary_sections((8, 8), device="cpu"), far + 2),
        lambda: B.paged_attention_workspace_bytes(batch, far + 2, 2),
        lambda: B.paged_attention_workspace_bytes(batch, 2, far + 2),
        lambda: B.paged_attention_workspace_bytes(batch, 2, 2, window=far + 5),
        lambda: B.paged_attention_workspace_bytes(batch, 2, 2, window=5, sinks=-far),
        lambda: B.k_paged_attention(batch, rows, rows.clone(), window=far + 5),
        lambda: B.k_paged_attention(batch, rows, rows.clone(), window=5, sinks=far),
        lambda: B.k_paged_attention(batch, one, one),
        lambda: B.k_paged_store(batch, one, one),
    ]
    for call in bad:
        with pytest.raises(B.MarError, match="32 bits"):
            call()


def test_the_current_stream_without_the_private_call(monkeypatch):
    """Where torch has no raw handle to give, its Stream object's is taken."""
    class Stream:
        cuda_stream = 1234
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    assert B._stream() == 1234 and B._stream_here(torch.device("cuda", 0), None) == 1234
    other = Stream()
    other.cuda_stream = 99
    assert B._stream(other) == 99 and B._stream_here(torch.device("cuda", 0), other) == 99
