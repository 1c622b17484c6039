"""The oracle of decoding with drafted tokens pinned on other forms, and the
refusals of the entry points, all on the CPU: every check is made on the host
before anything is enqueued, so the pointers here are never followed."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from oracle import draft as OD
from oracle import paged as OP
from paper_2503_12450_amd import binding as B
from test_paged_host import ARG, BAD_BATCH, PTR, SHAPE, WS, _batch


def _paged(seed, Hk, dh, L, page=16):
    g = np.random.Generator(np.random.Philox(seed))
    n = -(-L // page)
    return g, g.standard_normal((n, Hk, page, dh)), g.standard_normal((n, Hk, page, dh)), np.arange(n)[None]


@pytest.mark.parametrize("window,sinks", [(0, 0), (7, 0), (7, 3), (1, 0)])
def test_a_chain_is_causal_attention(window, sinks):
    g, pk, pv, table = _paged(3, 2, 16, 40)
    q = g.standard_normal((9, 4, 16))
    args = q, pk, pv, table, np.array([0, 9]), np.array([33])
    a, ma, ra = OD.tree_attention(*args, np.arange(-1, 8), window, sinks)
    b, mb, rb = OP.attention(*args, True, window, sinks)
    for x, y in ((a, b), (ma, mb), (ra, rb)):
        np.testing.assert_allclose(x, y, atol=1e-13)


def test_a_branch_is_the_sequence_that_it_spells():
    """Each node's output is that of the last row of a chain of its ancestors."""
    g, pk, pv, table = _paged(4, 1, 16, 60)
    parent = np.array([-1, 0, 0, 1, 2, 2, -1, 6, 4])
    n, L = len(parent), 41
    q = g.standard_normal((n, 1, 16))
    o, _, _ = OD.tree_attention(q, pk, pv, table, np.array([0, n]), np.array([L]), parent, 20, 2)
    flat = lambda p: np.concatenate(list(p[:, 0]))
    for i in range(n):
        line = OD.ancestors(parent, 0, i)[::-1]
        tokens = list(range(L - n)) + [L - n + a for a in line]
        pad = np.zeros((64 - len(tokens), 16))
        k, v = (np.concatenate([flat(p)[tokens], pad]).reshape(4, 16, 1, 16).transpose(0, 2, 1, 3) for p in (pk, pv))
        want, _, _ = OP.attention(q[i:i + 1], k, v, np.arange(4)[None], np.array([0, 1]), np.array([len(tokens)]),
                                  True, 20, 2)
        np.testing.assert_allclose(o[i], want[0], atol=1e-13)


@pytest.mark.parametrize("drawn", [False, True])
def test_kept_tokens_are_distributed_as_the_target(drawn):
    """The law of the first token after node 0, summed over every draw of the draft
    and integrated over the random numbers in cells of 1/64, on which nothing
    changes (all probabilities are multiples of it, where they decide)."""
    V = 3
    p = np.array([0.5, 0.125, 0.375])
    d = np.array([0.25, 0.5, 0.25])
    law, cells = np.zeros(V), 64
    drafts = itertools.product(range(V), repeat=2) if drawn else [(1, 0)]
    for x, y in drafts:
        chance = d[x] * d[y] if drawn else 1.0
        tokens, parent = np.array([0, x, y]), np.array([-1, 0, 0])
        full = np.stack([p, p, p])
        draft = np.stack([d, d, d]) if drawn else None
        mids = (np.arange(cells) + 0.5) / cells
        for r1, r2 in itertools.product(mids[::4] if drawn else mids, repeat=2):
            for r0 in mids[::8]:
                path, kept, after = OD.verify(full, [0, 3], parent, tokens, np.array([r0, r1, r2]), draft)
                first = tokens[path[1]] if kept[0] > 1 else after[0]
                law[first] += chance / ((cells // 4 if drawn else cells) ** 2 * (cells // 8))
    # cells that a border cuts: at most one of each number's
    np.testing.assert_allclose(law, p, atol=0.07 if drawn else 0.02)
    assert abs(law.sum() - 1) < 1e-12


def test_verification_by_hand():
    p = np.array([[0.5, 0.25, 0.25, 0.0], [0.0, 1.0, 0.0, 0.0], [0.25, 0.25, 0.25, 0.25]])
    run = lambda parent, tokens, r, d=None: [list(map(int, x)) for x in
                                             OD.verify(p, [0, 3], np.array(parent), np.array(tokens), r, d)]
    # both children of node 0: 0.5 < 0.5 fails, then 0.4 * 0.5 < 0.25
    assert run([-1, 0, 0], [9, 0, 2], np.array([0.0, 0.5, 0.4])) == [[0, 2, -1], [2], [0]]
    # neither: what is left is token 1 alone
    assert run([-1, 0, 0], [9, 0, 2], np.array([0.99, 0.5, 0.5])) == [[0, -1, -1], [1], [1]]
    # the same token twice: nothing is left of it
    assert run([-1, 0, 0], [9, 1, 1], np.array([0.0, 0.25, 0.0])) == [[0, -1, -1], [1], [0]]
    # a chain, its last token not kept
    assert run([-1, 0, 1], [9, 0, 0], np.array([0.5, 0.0, 0.0])) == [[0, 1, -1], [2], [1]]
    # greedy: the first largest
    assert run([-1, 0, 1], [9, 0, 1], None) == [[0, 1, 2], [3], [0]]
    # drawn from the target itself: always kept; from elsewhere: what the draft has too much of goes
    assert run([-1, 0, 1], [9, 2, 1], np.array([0.3, 0.99, 0.99]), p) == [[0, 1, 2], [3], [1]]
    # (0.25 0 0.25 0 after the first, 0.25 0 0.5 0 after the second: 0.4 of 0.75 lies in the third)
    d = np.array([[0.25, 0.75, 0.0, 0.0]] * 3)
    assert run([-1, 0, 0], [9, 1, 1], np.array([0.4, 0.5, 0.5]), d) == [[0, -1, -1], [1], [2]]


def test_keeping_and_forking_by_hand():
    k = np.arange(6 * 16, dtype=np.float64).reshape(6, 1, 16, 1)
    before = k.copy()
    table = np.array([[4, 1, -1]])
    left = OD.keep([k], table, [0, 5], [18], [0, 2, 4, -1, -1], [3])
    assert left.tolist() == [16] and k[4, 0, 13:, 0].tolist() == [77, 79, 17]
    k = before.copy()
    out, length, missing = OD.fork([k], table, [18], [0, 0, 0, -1], [18, 18, 3, 0], [1, 20, 0, 16])
    # two rows write to page 1, nobody else names it: the lower one keeps it
    assert out.tolist() == [[4, 1, -1], [4, 0, 2], [4, -1, -1], [3, -1, -1]]
    assert length.tolist() == [19, 38, 3, 16] and missing == 0
    assert k[0, 0, :2, 0].tolist() == [16, 17] and np.array_equal(k[0, 0, 2:], before[0, 0, 2:])
    out, _, missing = OD.fork([k], np.array([[0, 1, 2], [3, 4, 5]]), [40, 48], [0, 0], None, [1, 1])
    assert missing == 1 and out.tolist() == [[0, 1, 2], [0, 1, -1]]


def test_probabilities_by_hand():
    got = OD.probabilities(np.array([[0.0, np.log(3.0)], [1.0, 1.0], [-np.inf, 5.0], [-np.inf, np.nan]]),
                           [1.0, 0.0, 2.0, 0.0])
    np.testing.assert_allclose(got, [[0.25, 0.75], [1, 0], [0, 1], [0, 0]])


def test_probabilities_by_hand_at_an_infinite_temperature():
    inf = np.inf
    got = OD.probabilities(np.array([[0.0, 9.0, -inf], [-3e38, 3e38, -inf], [-inf, -inf, -inf], [1.0, inf, -inf]]),
                           [inf] * 4)
    np.testing.assert_array_equal(got, [[0.5, 0.5, 0], [0.5, 0.5, 0], [np.nan] * 3, [np.nan] * 3])


# --------------------------------------------------------------------------
# Refusals through the C entry points
# --------------------------------------------------------------------------

def _tree_call(batch=None, **kw):
    a = dict(dtype=1, m=5, hq=4, q=PTR, ld_q=256, parent=PTR, window=0, sinks=0, ws=None, ws_bytes=0, out=2 * PTR,
             ld_o=256)
    a.update(kw)
    batch = _batch() if batch is None else batch
    return B.load().mar_k_paged_tree_attention(a["dtype"], ctypes.byref(batch) if batch else None, a["m"], a["hq"],
                                               a["q"], a["ld_q"], a["parent"], a["window"], a["sinks"], a["ws"],
                                               a["ws_bytes"], a["out"], a["ld_o"], None)


def _probs_call(**kw):
    a = dict(dtype=1, x=PTR, ld=100, T=PTR, m=5, vocab=100, out=2 * PTR, ld_o=100)
    a.update(kw)
    return B.load().mar_k_probabilities(a["dtype"], a["x"], a["ld"], a["T"], a["m"], a["vocab"], a["out"], a["ld_o"],
                                        None)


def _verify_call(**kw):
    a = dict(dtype=1, n=3, q_start=PTR, m=5, vocab=100, p=PTR, ld_p=100, draft=None, ld_d=100, parent=PTR, tokens=PTR,
             random=PTR, path=2 * PTR, kept=PTR, next=2 * PTR, ws=PTR, ws_bytes=1 << 30)
    a.update(kw)
    return B.load().mar_k_draft_verify(a["dtype"], a["n"], a["q_start"], a["m"], a["vocab"], a["p"], a["ld_p"],
                                       a["draft"], a["ld_d"], a["parent"], a["tokens"], a["random"], a["path"],
                                       a["kept"], a["next"], a["ws"], a["ws_bytes"], None)


def _keep_call(batch=None, **kw):
    a = dict(dtype=1, m=5, path=PTR, kept=PTR, out=2 * PTR)
    a.update(kw)
    batch = _batch() if batch is None else batch
    return B.load().mar_k_paged_keep(a["dtype"], ctypes.byref(batch) if batch else None, a["m"], a["path"], a["kept"],
                                     a["out"], None)


def _fork_call(batch=None, **kw):
    a = dict(dtype=1, n=5, source=PTR, keep=None, add=None, table=2 * PTR, kv=2 * PTR, missing=PTR, ws=PTR,
             ws_bytes=1 << 30)
    a.update(kw)
    batch = _batch() if batch is None else batch
    return B.load().mar_k_paged_fork(a["dtype"], ctypes.byref(batch) if batch else None, a["n"], a["source"],
                                     a["keep"], a["add"], a["table"], a["kv"], a["missing"], a["ws"], a["ws_bytes"],
                                     None)


@pytest.mark.parametrize("status,kw", BAD_BATCH)
def test_calls_refuse_a_batch(status, kw):
    bad = _batch(**kw)
    assert _tree_call(batch=bad) == status
    assert _keep_call(batch=bad) == status
    assert _fork_call(batch=bad) == status
    lib = B.load()
    assert lib.mar_k_paged_tree_attention_workspace_bytes(1, ctypes.byref(bad), 5, 4, 0, 0) == 0
    assert lib.mar_last_error()
    assert lib.mar_k_paged_fork_workspace_bytes(ctypes.byref(bad), 5) == 0 and lib.mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=7)), (ARG, dict(batch=False)), (SHAPE, dict(hq=3)), (SHAPE, dict(hq=0)), (SHAPE, dict(m=-1)),
    (ARG, dict(q=None)), (ARG, dict(out=None)), (ARG, dict(out=PTR)), (ARG, dict(parent=None)), (SHAPE, dict(ld_q=255)),
    (SHAPE, dict(ld_o=248)), (ARG, dict(window=-1)), (ARG, dict(sinks=-1)), (WS, dict(ws=None, ws_bytes=64)),
    (WS, dict(ws=PTR + 4, ws_bytes=64)), (SHAPE, dict(m=1 << 28)),
])
def test_tree_attention_refuses(status, kw):
    assert _tree_call(**kw) == status
    assert B.load().mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=2)), (SHAPE, dict(m=-1)), (SHAPE, dict(m=1 << 30)), (SHAPE, dict(vocab=0)),
    (SHAPE, dict(vocab=(1 << 20) + 1, ld=1 << 21, ld_o=1 << 21)), (SHAPE, dict(ld=99)), (SHAPE, dict(ld_o=99)),
    (SHAPE, dict(ld=1 << 31)), (ARG, dict(x=None)), (ARG, dict(out=None)), (ARG, dict(x=PTR + 1)),
    (ARG, dict(out=PTR + 2)), (ARG, dict(out=PTR)), (ARG, dict(dtype=0, out=PTR, ld_o=101)),
])
def test_probabilities_refuse(status, kw):
    assert _probs_call(**kw) == status
    assert B.load().mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=2)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=65537)), (SHAPE, dict(m=-1)), (SHAPE, dict(m=1 << 30)),
    (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=1 << 21, ld_p=1 << 21)), (SHAPE, dict(ld_p=99)),
    (SHAPE, dict(draft=PTR, ld_d=98)), (ARG, dict(draft=PTR, random=None)), (ARG, dict(draft=PTR + 1)),
    (ARG, dict(p=PTR + 1)), (ARG, dict(p=None)), (ARG, dict(q_start=None)), (ARG, dict(parent=None)),
    (ARG, dict(tokens=None)), (ARG, dict(path=None)), (ARG, dict(kept=None)), (ARG, dict(next=None)),
    (WS, dict(ws=PTR + 8)), (WS, dict(ws=None, ws_bytes=1 << 30)), (WS, dict(ws_bytes=4)),
    (ARG, dict(path=2 * PTR, parent=2 * PTR)), (ARG, dict(path=2 * PTR, tokens=2 * PTR)),
    (ARG, dict(kept=2 * PTR, next=2 * PTR)),
])
def test_verification_refuses(status, kw):
    assert _verify_call(**kw) == status
    assert B.load().mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=2)), (ARG, dict(batch=False)), (SHAPE, dict(m=-1)), (SHAPE, dict(m=1 << 30)),
    (ARG, dict(path=None)), (ARG, dict(kept=None)), (ARG, dict(out=None)), (ARG, dict(out=PTR)),
])
def test_keeping_refuses(status, kw):
    assert _keep_call(**kw) == status
    assert B.load().mar_last_error()


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(dtype=2)), (ARG, dict(batch=False)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=65537)),
    (ARG, dict(source=None)), (ARG, dict(table=None)), (ARG, dict(kv=None)), (ARG, dict(missing=None)),
    (ARG, dict(table=PTR)), (ARG, dict(kv=PTR)), (ARG, dict(source=2 * PTR)), (ARG, dict(keep=2 * PTR)),
    (ARG, dict(add=2 * PTR)), (WS, dict(ws=PTR + 8)), (WS, dict(ws=None)), (WS, dict(ws_bytes=16)),
])
def test_forking_refuses(status, kw):
    assert _fork_call(**kw) == status
    assert B.load().mar_last_error()


def _refused_overlap(status, *names):
    said = B.load().mar_last_error().decode()
    assert status == ARG and all(n in said for n in names) and "overlap" in said, (status, said)


def _apart(**sizes):
    """Addresses of ranges of these sizes, 64 bytes between them."""
    at, out = 1 << 20, {}
    for name, n in sizes.items():
        out[name] = at
        at += -(-n // 64) * 64 + 64
    return out


V = dict(n=3, m=5, vocab=20, ld_p=20, ld_d=20, dtype=0)
V_ARGS = dict(path=20, kept=12, next=12, ws=4096, q_start=16, parent=20, tokens=20, random=20, p=400, draft=400)


@pytest.mark.parametrize("out", ["path", "kept", "next", "ws"])
@pytest.mark.parametrize("other", list(V_ARGS))
def test_verification_refuses_outputs_that_overlap(out, other):
    """The last word of one in the first of the other, and the reverse; of a workspace,
    what the call needs of it."""
    if out == other:
        return
    at = _apart(**V_ARGS)
    need = B.draft_verify_workspace_bytes(V["m"], V["n"], V["vocab"])
    size = dict(V_ARGS, ws=need)
    if out == "ws":  # aligned, it stays
        moved = [{other: at["ws"] + need - 4}]
    else:
        moved = [{out: at[other] - size[out] + 4}, {out: at[other] + size[other] - 4}]
    for places in moved:
        status = _verify_call(**V, **dict(at, **places), ws_bytes=4096)
        _refused_overlap(status, *("workspace" if x == "ws" else x for x in (out, other)))


def test_verification_may_leave_outputs_between_rows():
    """What lies between the rows of p is not p's: the call goes on to the next refusal
    (the overlap of kept and next)."""
    at = _apart(**dict(V_ARGS, p=4000))
    status = _verify_call(**dict(V, ld_p=200), **dict(at, path=at["p"] + 80, next=at["kept"]), ws_bytes=4096)
    _refused_overlap(status, "kept", "next")


@pytest.mark.parametrize("other,size", [("kv_len", 12), ("q_start", 16), ("table", 48), ("path", 20), ("kept", 12),
                                        ("k", 10 * 2 * 16 * 64 * 2), ("v", 10 * 2 * 16 * 64 * 2)])
def test_keeping_refuses_lengths_that_overlap(other, size):
    sizes = dict(kv_len=12, q_start=16, table=48, path=20, kept=12, k=40960, v=40960, out=12)
    at = _apart(**sizes)
    for where in (at[other] - 8, at[other] + size - 4):
        batch = _batch(**{n: at[n] for n in ("k", "v", "table", "q_start", "kv_len")})
        _refused_overlap(_keep_call(batch=batch, path=at["path"], kept=at["kept"], out=where), "kv_len_out", other)


@pytest.mark.parametrize("out,name", [("table_out", "table"), ("kv_len_out", "kv"), ("missing", "missing")])
@pytest.mark.parametrize("other", ["table", "kv_len", "source", "keep", "add", "k", "v", "ws"])
def test_forking_refuses_outputs_that_overlap(out, name, other):
    sizes = dict(table_out=80, kv_len_out=20, missing=4, table=48, kv_len=12, source=20, keep=20, add=20, k=40960,
                 v=40960, ws=4096)
    at = _apart(**sizes)
    batch = _batch(**{n: at[n] for n in ("k", "v", "table", "kv_len")})
    need = B.load().mar_k_paged_fork_workspace_bytes(ctypes.byref(batch), 5)
    last = dict(sizes, ws=need)[other]
    for where in (at[other], at[other] + last - 4):
        where = {"table_out": at["table_out"], "kv_len_out": at["kv_len_out"], "missing": at["missing"], out: where}
        status = _fork_call(batch=batch, table=where["table_out"], kv=where["kv_len_out"], missing=where["missing"],
                            source=at["source"], keep=at["keep"], add=at["add"], ws=at["ws"], ws_bytes=4096)
        _refused_overlap(status, out, "workspace" if other == "ws" else other)


def test_rows_that_overlap_are_refused():
    """Probabilities and outputs of attention over their inputs: dense ones anywhere,
    strided ones where columns meet."""
    x = 1 << 20
    for off in (-5 * 400 + 4, -400, 4, 5 * 400 - 4):                     # dense, fp32
        _refused_overlap(_probs_call(dtype=0, x=x, out=x + off), "out", "logits")
    _refused_overlap(_probs_call(dtype=1, x=x, out=x + 996), "out", "logits")
    for off in (-396, 396, 800 + 396, -800 - 396, 3200 + 396, 800):      # rows 800 bytes apart, 400 wide
        _refused_overlap(_probs_call(dtype=0, x=x, out=x + off, ld=200, ld_o=200), "out", "logits")
    _refused_overlap(_probs_call(x=x, out=x + 4096, T=x + 4096 + 5 * 400 - 4), "out", "temperature")
    for off in (4 * 512 + 496, -16, 512, 16):
        _refused_overlap(_tree_call(q=x, out=x + off, ld_q=256, ld_o=256), "out", "q")
    for off in (1008, 2 * 1024 + 496, -496):                             # rows 1024 bytes apart, 512 wide
        _refused_overlap(_tree_call(q=x, out=x + off, ld_q=512, ld_o=512), "out", "q")
    _refused_overlap(_tree_call(q=x, out=2 * x, parent=2 * x + 512 * 5 - 4), "out", "parent")
    # columns of one matrix are apart, also first and last rows: the next refusal speaks
    for off in (400, -400, 3200 + 400, -4000 - 400, 4000):
        status = _probs_call(dtype=0, x=x, out=x + off, ld=200, ld_o=200, T=x + off, m=1)
        _refused_overlap(status, "out", "temperature")


def test_nothing_to_do_is_not_an_error():
    """No rows, or no sequences: nothing is enqueued and no pointer is followed."""
    none = dict(n_seqs=0, table=None, kv_len=None)
    assert _tree_call(m=0, q=None, out=None, parent=None) == B.MAR_OK
    assert _tree_call(batch=_batch(**none)) == B.MAR_OK
    assert _probs_call(m=0, x=None, out=None) == B.MAR_OK
    assert _verify_call(n=0, q_start=None, kept=None, next=None) == B.MAR_OK
    assert _probs_call(m=0, x=None, out=None, T=None) == B.MAR_OK
    assert _keep_call(batch=_batch(**none), kept=None, out=None) == B.MAR_OK


def test_the_workspaces_are_sized():
    lib = B.load()
    assert B.draft_verify_workspace_bytes(100, 10, 1000) > 0
    for bad in ((-1, 1, 10), (1, -1, 10), (1, 1, 0), (1, 1, 1 << 21)):
        assert lib.mar_k_draft_verify_workspace_bytes(*bad) == 0 and lib.mar_last_error()
        with pytest.raises(B.MarError):
            B.draft_verify_workspace_bytes(*bad)


@pytest.mark.parametrize("m", [0, 1, 100, 2 ** 30 - 1])
@pytest.mark.parametrize("n,vocab", [(1, 16384), (65536, 5), (3, 100)])
def test_verification_of_few_tokens_asks_for_the_maxima_alone(m, n, vocab):
    need = -(-4 * m // 16) * 16
    assert B.draft_verify_workspace_bytes(m, n, vocab) == need
    if m:
        assert _verify_call(m=m, n=n, vocab=vocab, ld_p=vocab, ws_bytes=need - 1) == WS


def test_verification_of_more_asks_for_its_sums():
    """A header of 256 sums and a sum for every 1024 tokens, to a sequence: of up to 191
    of them, as more are taken in one launch.  Never less for more."""
    for n, vocab in ((191, 2 ** 20), (1, 16385), (10, 65536), (65536, 2 ** 20)):
        some = min(n, 191)
        least = some * (8 * 256 + 8 * -(-vocab // 1024))
        assert least <= B.draft_verify_workspace_bytes(5, n, vocab) <= least + 16 * some + 32
        assert B.draft_verify_workspace_bytes(2 ** 28, n, vocab) == 2 ** 30
    sizes = [[B.draft_verify_workspace_bytes(5, n, vocab) for n in (1, 100, 191, 192, 65536)]
             for vocab in (100, 16384, 16385, 50000, 2 ** 20)]
    assert np.all(np.diff(sizes, axis=0) >= 0) and np.all(np.diff(sizes, axis=1) >= 0)


# --------------------------------------------------------------------------
# Refusals of the binding
# --------------------------------------------------------------------------

def test_binding_refuses_what_the_library_cannot_see():
    pages = B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 32))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    table = torch.zeros((2, 2), dtype=torch.int32)
    batch = B.PagedBatch(pages, table, i32(0, 1, 2), i32(3, 4))
    x, p, f = torch.zeros(2, 64), torch.zeros(2, 50), torch.zeros(2)
    two, one = i32(0, 0), i32(0)
    ok = lambda **kw: dict(dict(q_start=i32(0, 1, 2), p=p, parent=two, tokens=two, path=two, kept=two, next_token=two,
                                random=f, draft=None), **kw)
    bad = [
        lambda: B.k_paged_tree_attention(batch, x, two.long(), x.clone()),
        lambda: B.k_paged_tree_attention(batch, x, one, x.clone()),
        lambda: B.k_paged_tree_attention(batch, x, two, x[:, :32]),
        lambda: B.k_paged_tree_attention(batch, x.bfloat16(), two, x.bfloat16()),
        lambda: B.k_paged_tree_attention(batch, x, two, x.clone(), workspace=torch.zeros(8, 2)[:, :1]),
        lambda: B.k_paged_tree_attention(batch, x, two, x.clone()),                     # not on a GPU
        lambda: B.paged_tree_attention_workspace_bytes(batch, 2, 3),
        lambda: B.k_probabilities(p, p.bfloat16()),
        lambda: B.k_probabilities(p.half(), p),
        lambda: B.k_probabilities(p[0], p[0]),
        lambda: B.k_probabilities(p, p[:, :40]),
        lambda: B.k_probabilities(p.t(), torch.zeros(50, 2)),
        lambda: B.k_probabilities(p, p.clone(), temperature=f.double()),
        lambda: B.k_probabilities(p, p.clone(), temperature=torch.zeros(3)),
        lambda: B.k_probabilities(p, p.clone()),                                        # not on a GPU
        lambda: B.k_draft_verify(**ok(q_start=i32())),
        lambda: B.k_draft_verify(**ok(q_start=i32(0, 2))),
        lambda: B.k_draft_verify(**ok(p=p.double())),
        lambda: B.k_draft_verify(**ok(draft=p.bfloat16())),
        lambda: B.k_draft_verify(**ok(draft=p[:, :49])),
        lambda: B.k_draft_verify(**ok(parent=one)),
        lambda: B.k_draft_verify(**ok(tokens=two.long())),
        lambda: B.k_draft_verify(**ok(path=i32(0, 0, 0)[::2])),
        lambda: B.k_draft_verify(**ok(kept=one)),
        lambda: B.k_draft_verify(**ok(next_token=f)),
        lambda: B.k_draft_verify(**ok(random=f.double())),
        lambda: B.k_draft_verify(**ok()),                                               # not on a GPU
        lambda: B.k_paged_keep(batch, two.float(), two, two.clone()),
        lambda: B.k_paged_keep(batch, two, one, two.clone()),
        lambda: B.k_paged_keep(batch, two, two, one),
        lambda: B.k_paged_keep(batch, table, two, two),
        lambda: B.k_paged_keep(batch, two, two, two.clone()),                           # not on a GPU
        lambda: B.k_paged_fork(batch, two, table, two, two),
        lambda: B.k_paged_fork(batch, two, table[:, :1], two, one),
        lambda: B.k_paged_fork(batch, two, table, one, one),
        lambda: B.k_paged_fork(batch, two, table, two, one, keep=one),
        lambda: B.k_paged_fork(batch, two, table, two, one, add=f),
        lambda: B.k_paged_fork(batch, two.long(), table, two, one),
        lambda: B.k_paged_fork(batch, two, table.clone(), two, one),                    # not on a GPU
        lambda: B.paged_fork_workspace_bytes(batch, -1),
    ]
    for call in bad:
        with pytest.raises(B.MarError):
            call()
    far, wide = 2 ** 32, torch.zeros(1, 64).expand(2 ** 32 + 2, 64)
    for call in [lambda: B.paged_tree_attention_workspace_bytes(batch, far + 2, 2),
                 lambda: B.k_paged_tree_attention(batch, x, two, x.clone(), window=far + 5),
                 lambda: B.draft_verify_workspace_bytes(far + 1, 1, 5),
                 lambda: B.paged_fork_workspace_bytes(batch, far + 1),
                 lambda: B.k_probabilities(wide, wide)]:
        with pytest.raises(B.MarError, match="32 bits"):
            call()


def test_binding_refuses_tensors_that_are_missing():
    pages = B.MarPages(torch.zeros(4, 2, 16, 32), torch.zeros(4, 2, 16, 32))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    table = torch.zeros((2, 2), dtype=torch.int32)
    batch = B.PagedBatch(pages, table, i32(0, 1, 2), i32(3, 4))
    x, p, two = torch.zeros(2, 64), torch.zeros(2, 50), i32(0, 0)
    calls = [
        (B.k_paged_tree_attention, dict(batch=batch, q=x, parent=two, out=x.clone()), ("q", "parent", "out")),
        (B.k_probabilities, dict(logits=p, out=p.clone()), ("logits", "out")),
        (B.k_draft_verify, dict(q_start=i32(0, 1, 2), p=p, parent=two, tokens=two, path=two.clone(), kept=two.clone(),
                                next_token=two.clone()),
         ("q_start", "p", "parent", "tokens", "path", "kept", "next_token")),
        (B.k_paged_keep, dict(batch=batch, path=two, kept=two, kv_len_out=two.clone()), ("path", "kept", "kv_len_out")),
        (B.k_paged_fork, dict(batch=batch, source=two, table_out=table.clone(), kv_len_out=two.clone(), missing=i32(0)),
         ("source", "table_out", "kv_len_out", "missing")),
    ]
    for call, args, needed in calls:
        for name in needed:
            with pytest.raises(B.MarError, match=f"{name} is missing"):
                call(**dict(args, **{name: None}))
        with pytest.raises(B.MarError, match="current GPU"):   # all there: the next refusal
            call(**args)
