"""Decoding with drafted tokens over the paged key/value cache, as cases to be
timed.

Six kinds:

tree    attention of trees of drafted tokens over the cache: a row sees what is
        cached before the tree, itself and its ancestors
probs   probabilities of logits, each row with a temperature of its own
verify  which drafted tokens the target's probabilities accept, and the token
        after them, from given random numbers; the drafts are points, drawn
        from probabilities of their own, or checked greedily
keep    the accepted rows of the trees moved together in the cache
fork    sequences continued by several others: shared pages, copies of the
        part-filled ones, fresh pages, freed ones
step    all of it for one new tree per sequence: the tree's keys and values into
        the cache, its attention, the head's probabilities, the verification,
        and what was accepted moved together

With `own` false `run` computes the plain form in elementary torch operations
(32 bits; 64 for sums that decide between tokens), with `own` true it makes the
calls of the binding.

Inputs are drawn on the GPU from the seed.  Lengths and trees follow from the
case alone: `lengths` starts their generator.  Sequences own pages in a random
order, as after many allocations and releases.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
TDT = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0
MOST_NODES = 256


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _tree(name, seqs, nodes, branch, past, heads, kv_heads, d_head, page, dtype, window=0, sinks=0, lengths=1,
          kind="tree"):
    return {"name": name, "kind": kind, "seqs": seqs, "nodes_lo": nodes[0], "nodes_hi": nodes[1], "branch": branch,
            "past_lo": past[0], "past_hi": past[1], "heads": heads, "kv_heads": kv_heads, "d_head": d_head,
            "page": page, "dtype": dtype, "window": window, "sinks": sinks, "lengths": lengths}


def _probs(name, rows, vocab, dtype, cold):
    return {"name": name, "kind": "probs", "rows": rows, "vocab": vocab, "dtype": dtype, "cold": cold}


def _verify(name, seqs, nodes, branch, vocab, dtype, draft, spread=2.0, noise=0.7, lengths=1):
    return {"name": name, "kind": "verify", "seqs": seqs, "nodes_lo": nodes[0], "nodes_hi": nodes[1], "branch": branch,
            "vocab": vocab, "dtype": dtype, "draft": draft, "spread": spread, "noise": noise, "lengths": lengths}


def _keep(name, seqs, nodes, past, kv_heads, d_head, page, dtype, lengths=1):
    return {"name": name, "kind": "keep", "seqs": seqs, "nodes_lo": nodes[0], "nodes_hi": nodes[1],
            "past_lo": past[0], "past_hi": past[1], "kv_heads": kv_heads, "d_head": d_head, "page": page,
            "dtype": dtype, "lengths": lengths}


def _fork(name, seqs, copies, past, add, kv_heads, d_head, page, dtype, lengths=1):
    return {"name": name, "kind": "fork", "seqs": seqs, "copies": copies, "past_lo": past[0], "past_hi": past[1],
            "add": add, "kv_heads": kv_heads, "d_head": d_head, "page": page, "dtype": dtype, "lengths": lengths}


def listed():
    return [
        # a serving batch: trees of 16 to 64 drafted tokens on contexts of very
        # different lengths, shared key/value heads
        _tree("tree_batch", 32, (16, 64), 3, (500, 8000), 32, 4, 128, 64, "bf16"),
        # one tree on one very long context: its keys have to be split
        _tree("tree_long", 1, (64, 64), 4, (131000, 131000), 16, 2, 128, 64, "bf16", lengths=2),
        # the fp32 path on chains and small trees, with a window and first tokens
        _tree("tree_f32", 6, (3, 21), 2, (100, 1500), 12, 12, 64, 16, "f32", window=512, sinks=64, lengths=3),
        # the head's logits of one small tree
        _probs("probs_tree", 7, 32000, "bf16", False),
        # the same of a serving batch, some of its rows greedy (temperature 0)
        _probs("probs_batch", 600, 65536, "bf16", True),
        # chains drawn from a draft model's own probabilities
        _verify("verify_chains", 48, (5, 9), 1, 65536, "f32", "drawn", lengths=4),
        # trees of likely tokens, an odd vocabulary
        _verify("verify_trees", 32, (16, 64), 3, 100003, "f32", "points", lengths=5),
        # greedy decoding straight from the logits
        _verify("verify_greedy", 64, (6, 8), 1, 32768, "bf16", "greedy", lengths=6),
        # accepted rows of wide trees
        _keep("keep_trees", 48, (24, 64), (10, 4000), 4, 128, 64, "bf16", lengths=7),
        # one prompt continued by four samples: the smallest fork
        _fork("fork_samples", 1, 4, (325, 325), 1, 12, 64, 16, "bf16", lengths=8),
        # prompts continued by eight samples each, 16 new tokens of room
        _fork("fork_batch", 16, 8, (1000, 8000), 16, 8, 128, 64, "bf16", lengths=9),
        # a whole step of one sequence: the smallest calls after each other
        {**_tree("step_tree", 1, (8, 8), 2, (320, 320), 12, 12, 64, 16, "bf16", lengths=10, kind="step"),
         "vocab": 16384, "spread": 2.0, "noise": 0.7},
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _some(rng):
    kind = rng.choice(("tree", "tree", "probs", "verify", "verify", "keep", "fork", "step"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    lengths = rng.randint(20, 10**6)
    if kind == "probs":
        vocab = _log(rng, 1000, 150000)
        return _probs("", _log(rng, 1, max(1, min(1000, 30000000 // vocab))), vocab, dtype, rng.random() < 0.3)
    if kind == "verify":
        draft = rng.choice(("points", "drawn", "greedy"))
        vocab = _log(rng, 1000, 120000)
        if draft == "drawn":
            nodes, branch = _log(rng, 2, 12), rng.choice((1, 1, 2))
        else:
            nodes, branch = _log(rng, 2, 80), rng.choice((1, 2, 3, 4))
        seqs = _log(rng, 1, max(1, min(96, 25000000 // (vocab * nodes))))
        return _verify("", seqs, (max(1, nodes // 2), nodes), branch, vocab, dtype if draft == "greedy" else "f32",
                       draft, rng.choice((1.0, 2.0, 3.0)), rng.choice((0.3, 0.7, 1.5)), lengths)
    group = rng.choice((1, 1, 2, 4, 7, 8))
    kv_heads = rng.choice((1, 2, 4, 8)) if group > 1 else rng.choice((4, 12, 16))
    d_head = rng.choice((32, 64, 64, 80, 112, 128, 128))
    page = rng.choice((16, 16, 32, 64, 128))
    if kind == "keep":
        nodes = _log(rng, 6, MOST_NODES)
        return _keep("", _log(rng, 1, 96), (max(4, nodes // 3), nodes), (1, _log(rng, 16, 4000)), kv_heads, d_head,
                     page, dtype, lengths)
    if kind == "fork":
        seqs = _log(rng, 1, 32)
        return _fork("", seqs, _log(rng, 1, 128 // seqs), (1, _log(rng, 16, 6000)), rng.choice((1, 1, 5, 16, 70)),
                     kv_heads, d_head, page, dtype, lengths)
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 4, 3000), rng.choice((0, 1, 4, 64, 100)))
    nodes, branch = _log(rng, 1, 150), rng.choice((1, 2, 3, 4))
    seqs, past = _log(rng, 1, 48), _log(rng, 16, 20000)
    if kind == "step":
        nodes, seqs, past = min(nodes, 40), min(seqs, 4), min(past, 4000)
    c = _tree("", seqs, (max(1, nodes // 3), nodes), branch, (1, past), group * kv_heads, kv_heads, d_head, page,
              dtype, window, sinks, lengths, kind)
    if kind == "step":
        c.update(vocab=_log(rng, 1000, 16384), spread=2.0, noise=0.7)
    return c


def draw(rng):
    while True:
        c = _some(rng)
        del c["name"]
        if c["kind"] != "tree":
            return c
        # what the plain form keeps of every pair, and the products' cost
        pairs = c["seqs"] * c["nodes_hi"] * (c["past_hi"] + c["nodes_hi"]) * c["heads"]
        if pairs <= (20e6 if c["dtype"] == "f32" else 250e6):
            return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 6151 + 17)


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _lengths(case):
    """Nodes of every tree, and tokens before it."""
    r = random.Random(case["lengths"])
    nodes = [_log(r, case["nodes_lo"], case["nodes_hi"]) if "nodes_lo" in case else 0 for _ in range(case["seqs"])]
    past = [_log(r, case["past_lo"], case["past_hi"]) if "past_lo" in case else 0 for _ in range(case["seqs"])]
    return nodes, past


def _parents(case):
    """Each tree's parents, level by level: about `branch` children to a node."""
    r, b = random.Random(case["lengths"] + 1), case["branch"]
    return [[-1] + [(i - 1) // b if b == 1 else max(0, min(i - 1, (i - 1) // b + r.randint(-1, 1)))
                    for i in range(1, n)] for n in _lengths(case)[0]]


def _starts(nodes):
    start = [0]
    for n in nodes:
        start.append(start[-1] + n)
    return start


def _cache(case, g, kv, spare, room=0):
    """Pages in a random order, `spare` of them nobody's; `room` for more pages
    in a sequence's row."""
    t, page, shape = TDT[case["dtype"]], case["page"], (case["kv_heads"], case["page"], case["d_head"])
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(kv), max(need) + room), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return {"table": table, "k_pages": _normal(g, (n_pages, *shape), 1.0, t),
            "v_pages": _normal(g, (n_pages, *shape), 1.0, t)}


def _frequencies(d_head):
    pairs = d_head // 2
    return (torch.tensor([BASE ** (-j / pairs) for j in range(pairs)], dtype=torch.float64, device=DEV),
            torch.zeros(pairs, dtype=torch.int32, device=DEV))


def _tree_inputs(case, seed):
    g, t = _gen(seed), TDT[case["dtype"]]
    nodes, past = _lengths(case)
    parents = _parents(case)
    kv = [a + b for a, b in zip(nodes, past)]
    H, Hk, dh, m = case["heads"], case["kv_heads"], case["d_head"], sum(nodes)
    st = {"nodes": nodes, "kv": kv, "q_start": _i32(_starts(nodes)), "kv_len": _i32(kv),
          "parent": _i32([p for tree in parents for p in tree]), **_cache(case, g, kv, 3)}
    if case["kind"] == "tree":
        st["q"] = _normal(g, (m, H * dh), 1.5, t)
        return st
    st["qkv"] = _normal(g, (m, (H + 2 * Hk) * dh), 1.0, t)
    st["freq"], st["axis"] = _frequencies(dh)
    pos = []
    for tree, before in zip(parents, past):
        depth = []
        for p in tree:
            depth.append(0 if p < 0 else depth[p] + 1)
        pos += [before + d for d in depth]
    st["pos"] = _i32(pos)[:, None].contiguous()
    st.update(_drafts(case, g, parents))
    st["temperature"] = torch.ones(m, device=DEV)
    return st


def _drafts(case, g, parents):
    """Target logits, drafted tokens and random numbers of trees.  The draft's
    logits are the target's with noise; a node's children are its likeliest
    tokens, or drawn from the draft's probabilities."""
    m, V, drawn = sum(len(t) for t in parents), case["vocab"], case.get("draft") == "drawn"
    start = _starts([len(t) for t in parents])
    above, rank = [], []
    for s, tree in enumerate(parents):
        seen = {}
        for p in tree:
            above.append(start[s] + max(p, 0))
            rank.append(seen.get(p, 0))
            seen[p] = rank[-1] + 1
    above, rank = torch.tensor(above, device=DEV), torch.tensor(rank, device=DEV)
    logits = _normal(g, (m, V), case["spread"])
    near = logits + _normal(g, (m, V), case["noise"])
    st = {"logits": logits.to(TDT[case["dtype"]]), "random": torch.rand(m, generator=g, device=DEV)}
    if drawn:
        st["draft"] = torch.softmax(near, 1)
        race = st["draft"][above] / torch.empty((m, V), device=DEV).exponential_(generator=g)
        st["tokens"] = race.argmax(1).to(torch.int32)
    else:
        best = near.topk(min(V, int(rank.max()) + 1), 1).indices
        st["tokens"] = best[above, rank].to(torch.int32)
    return st


def _inputs(case, seed):
    kind = case["kind"]
    if kind in ("tree", "step"):
        return _tree_inputs(case, seed)
    g = _gen(seed)
    if kind == "probs":
        rows = case["rows"]
        T = 0.6 + 0.8 * torch.rand(rows, generator=g, device=DEV)
        if case["cold"]:
            T[torch.rand(rows, generator=g, device=DEV) < 0.2] = 0.0
        return {"logits": _normal(g, (rows, case["vocab"]), 3.0, TDT[case["dtype"]]), "temperature": T}
    nodes, past = _lengths(case)
    if kind == "verify":
        parents = _parents(case)
        st = {"nodes": nodes, "q_start": _i32(_starts(nodes)), "parent": _i32([p for t in parents for p in t]),
              **_drafts(case, g, parents)}
        if case["draft"] != "greedy":
            st["logits"] = torch.softmax(st["logits"], 1)
        return st
    if kind == "keep":
        # accepted rows of trees whose first level alone is longer than a path:
        # no row that moves lies where another one goes
        r = random.Random(case["lengths"] + seed)
        kept = [r.randint(1, max(1, min(9, n // 2))) for n in nodes]
        path = []
        for n, a in zip(nodes, kept):
            rows = [0] + sorted(r.sample(range(a, n), a - 1))
            path += rows + [-1] * (n - a)
        kv = [a + b for a, b in zip(nodes, past)]
        return {"nodes": nodes, "kv": kv, "q_start": _i32(_starts(nodes)), "kv_len": _i32(kv), "path": _i32(path),
                "kept": _i32(kept), **_cache(case, g, kv, 3)}
    # fork: the first rows go on as they are (prompts that more samples may
    # start from), the others continue one of them each, in a random order
    S, n, page = case["seqs"], case["seqs"] * (1 + case["copies"]), case["page"]
    order = torch.randperm(n - S, generator=g, device=DEV)
    source = torch.cat([torch.arange(S, device=DEV), (order % S)]).to(torch.int32)
    add = torch.full((n,), case["add"], dtype=torch.int32, device=DEV)
    add[:S] = 0
    more = (n - S) * (2 + case["add"] // page)
    c = _cache(case, g, past, more, 2 + case["add"] // page)
    return {"kv": past, "source": source, "add": add, "q_start": _i32([0] * (S + 1)), "kv_len": _i32(past), **c}


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    kind = case["kind"]
    if not own:
        return st
    from paper_2503_12450_amd import binding as B
    empty = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device=DEV)
    room = lambda n: empty(n, dtype=torch.uint8)
    if "table" in st:
        st["pages"] = B.MarPages(st["k_pages"], st["v_pages"])
        st["batch"] = B.PagedBatch(st["pages"], st["table"], st["q_start"], st["kv_len"], max_kv=max(st["kv"]))
    if kind in ("tree", "step"):
        m, H, t = sum(st["nodes"]), case["heads"], TDT[case["dtype"]]
        st["out"] = empty(m, H * case["d_head"], dtype=t)
        st["workspace"] = room(B.paged_tree_attention_workspace_bytes(st["batch"], m, H, window=case["window"],
                                                                      sinks=case["sinks"]))
    if kind == "step":
        st["rotary"] = B.Rotary(st["freq"], st["axis"], 1)
        st["q"] = empty(m, H * case["d_head"], dtype=t)
    if kind in ("probs", "step"):
        st["p"] = empty(*st["logits"].shape, dtype=torch.float32)
    if kind in ("verify", "step"):
        m, V = st["logits"].shape
        st["path"], st["kept"], st["next"] = empty(m), empty(case["seqs"]), empty(case["seqs"])
        st["scratch"] = room(B.draft_verify_workspace_bytes(m, case["seqs"], V))
    if kind in ("keep", "step"):
        st["kv_out"] = empty(case["seqs"])
    if kind == "fork":
        n = st["source"].shape[0]
        st["table_out"], st["kv_out"], st["missing"] = empty(n, st["table"].shape[1]), empty(n), empty(1)
        st["workspace"] = room(B.paged_fork_workspace_bytes(st["batch"], n))
    return st


# ---------------------------------------------------------------------------
# One pass: the plain form
# ---------------------------------------------------------------------------

def _per_seq(st):
    """Index of row i of every sequence [seqs, most rows] and whether it is one."""
    start = st["q_start"].long()
    i = torch.arange(max(st["nodes"]), device=DEV)
    there = i < (start[1:] - start[:-1])[:, None]
    return torch.where(there, start[:-1, None] + i, 0), there


def _plain_tree(st, case, q):
    H, Hk, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    G, W, sinks, L = H // Hk, case["window"], case["sinks"], max(st["kv"])
    row, there = _per_seq(st)
    S, n = row.shape
    # ancestors [S, n, n]: the parents' matrix and one, squared until all are in
    step = torch.eye(n, device=DEV) + (st["parent"].long()[row][:, :, None] == torch.arange(n, device=DEV)).float()
    for _ in range(max(1, n - 1).bit_length()):
        step = (torch.matmul(step, step) > 0).float()
    depth = step.sum(2) - 1
    kv = st["kv_len"].long()
    first = (kv - there.sum(1))[:, None]
    token = torch.arange(L, device=DEV)
    ids = st["table"][:, token // page].long().clamp(min=0), token % page
    k, v = (p[ids[0], :, ids[1]].float().permute(0, 2, 1, 3) for p in (st["k_pages"], st["v_pages"]))
    # what a key is: a token of the past at its own position, or drafted token a
    a = (token - first).clamp(0, n - 1)                                     # [S, L]
    past = token < first
    at = torch.where(past, token, first + depth.long().gather(1, a))        # its position
    p = first + depth.long()                                                # the rows' positions
    seen = past[:, None] | (step.bool().gather(2, a[:, None].expand(S, n, L)) & (token < kv[:, None])[:, None])
    if W:
        seen &= (at[:, None] > p[:, :, None] - W) | (at[:, None] < sinks)
    seen |= ~there[:, :, None]  # rows that are none
    qs = q[row].float().view(S, n, Hk, G, dh).permute(0, 2, 3, 1, 4).reshape(S, Hk, G * n, dh)
    score = torch.matmul(qs, k.transpose(2, 3).contiguous()).view(S, Hk, G, n, L) * dh ** -0.5
    score.masked_fill_(~seen[:, None, None], -math.inf)
    weight = score.sub_(score.amax(-1, keepdim=True)).exp_()
    v = torch.where((token < kv[:, None])[:, None, :, None], v, 0.0).contiguous()
    o = torch.matmul(weight.view(S, Hk, G * n, L), v).view(S, Hk, G, n, dh) / weight.sum(-1, keepdim=True)
    o = o.permute(0, 3, 1, 2, 4).reshape(S * n, H * dh)
    out = torch.empty((q.shape[0] + 1, H * dh), dtype=q.dtype, device=DEV)
    out[torch.where(there, row, q.shape[0]).view(-1)] = o.to(q.dtype)
    return out[:-1]


def _plain_probs(logits, T):
    x = logits.float()
    top = x.amax(1, keepdim=True)
    e = torch.exp((x - top) / torch.where(T > 0, T, 1.0)[:, None])
    p = e / e.sum(1, keepdim=True)
    i = torch.arange(x.shape[1], device=DEV)
    best = torch.where(x == top, i, x.shape[1]).amin(1)
    return torch.where((T > 0)[:, None], p, (i == best[:, None]).float())


def _plain_verify(st, p, draft, points):
    row, there = _per_seq(st)
    S, n = row.shape
    V, base, seq = p.shape[1], row[:, 0], torch.arange(S, device=DEV)
    cur, kept = torch.zeros_like(base), torch.ones_like(base)
    path = torch.full((p.shape[0] + 1,), -1, dtype=torch.int64, device=DEV)
    path[base] = 0
    r = st["random"].double()
    if not points and draft is None:
        i = torch.arange(V, device=DEV)
        best = torch.where(p == p.amax(1, keepdim=True), i, V).amin(1)
    else:
        w, W = p[base].double(), torch.ones(S, dtype=torch.float64, device=DEV)
    for i in range(1, n):
        at = row[:, i]
        child = there[:, i] & (st["parent"][at] == cur)
        x = st["tokens"][at].long()
        if not points and draft is None:
            yes = child & (x == best[base + cur])
        elif points:
            a = w[seq, x]
            yes = child & (r[at] * W < a)
            no = child & ~yes
            W = torch.where(no, W - a, W)
            w[seq, x] = torch.where(no, 0.0, a)
        else:
            d = draft[base + cur].double()
            yes = child & (r[at] * d[seq, x] * W < w[seq, x])
            rest = (w / W[:, None] - d).clamp(min=0)
            total = rest.sum(1)
            no = child & ~yes & (total > 0)
            w, W = torch.where(no[:, None], rest, w), torch.where(no, total, W)
        path[torch.where(yes, base + kept, p.shape[0])] = i
        kept += yes
        cur = torch.where(yes, i, cur)
        if points or draft is not None:
            w, W = torch.where(yes[:, None], p[at].double(), w), torch.where(yes, 1.0, W)
    if points or draft is not None:
        c = w.cumsum(1)
        token = (c <= (r[base] * c[:, -1])[:, None]).sum(1).clamp(max=V - 1)
    else:
        token = best[base + cur]
    return {"path": path[:-1].to(torch.int32), "kept": kept.to(torch.int32), "next": token.to(torch.int32)}


def _plain_keep(st, case, path, kept):
    page = case["page"]
    row, there = _per_seq(st)
    first = (st["kv_len"].long() - there.sum(1))[:, None]
    i = torch.arange(row.shape[1], device=DEV)
    to = (first + i)[there]
    of = (first + torch.where(path[row] >= 0, path[row].long(), i))[there]
    seq = torch.arange(row.shape[0], device=DEV)[:, None].expand_as(row)[there]
    for p in (st["k_pages"], st["v_pages"]):
        rows = p[st["table"][seq, of // page].long(), :, of % page]
        p[st["table"][seq, to // page].long(), :, to % page] = rows
    return (first[:, 0] + kept).to(torch.int32)


def _plain_fork(st, case):
    page, table, kv = case["page"], st["table"], st["kv_len"].long()
    n_pages, (_, width) = st["k_pages"].shape[0], table.shape
    slot, source, add = torch.arange(width, device=DEV), st["source"].long(), st["add"].long()
    count = lambda where, ids: torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV).scatter_add_(
        0, torch.where(where, ids.long(), n_pages).view(-1), torch.ones(ids.numel(), dtype=torch.int64, device=DEV))
    used = count(slot < (-(-kv // page))[:, None], table)[:-1]
    keep = kv[source]
    length = keep + add
    held, old, new = -(-keep // page), table[source].long(), -(-length // page)
    last = old.gather(1, (held - 1)[:, None])[:, 0]       # the page of the last token kept
    writes = (add > 0) & (keep % page > 0)
    names, writers = count(slot < held[:, None], old), count(writes, last)
    i = torch.arange(source.numel(), device=DEV)
    low = torch.full((n_pages + 1,), source.numel(), dtype=torch.int64, device=DEV).scatter_reduce_(
        0, torch.where(writes, last, n_pages), i, "amin")
    copy = writes & (names[last] > 1) & ~((names[last] == writers[last]) & (low[last] == i))
    need = new - held + copy.long()
    rank = torch.cumsum((used == 0).long(), 0)
    fresh = torch.full((n_pages + need.numel() * width + 1,), -1, dtype=torch.int64, device=DEV)
    fresh[torch.where(used == 0, rank - 1, fresh.numel() - 1)] = torch.where(
        used == 0, torch.arange(n_pages, device=DEV), -1)
    begin = (torch.cumsum(need, 0) - need)[:, None]
    own_from = (held - copy.long())[:, None]
    given = fresh[(begin + slot - own_from).clamp(0, fresh.numel() - 1)]
    out = torch.where(slot < own_from, old, torch.where(slot < new[:, None], given, -1))
    to = torch.where(copy, out.gather(1, (held - 1)[:, None])[:, 0], last)
    part = (torch.arange(page, device=DEV) < (keep % page)[:, None])[:, None, :, None]
    for p in (st["k_pages"], st["v_pages"]):
        p[to] = torch.where(part, p[last], p[to])
    missing = (need.sum() - rank[-1]).clamp(min=0).view(1)
    return {"table": out.to(torch.int32), "kv_len": length.to(torch.int32), "missing": missing.to(torch.int32),
            "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_store(st, case):
    H, Hk, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    t = TDT[case["dtype"]]
    x = st["qkv"].view(-1, H + 2 * Hk, dh)
    angle = st["pos"].double() * st["freq"]
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[:, :H + Hk].float().chunk(2, -1)
    qk = torch.cat([a * c - b * s, b * c + a * s], -1).to(t)
    row = torch.arange(x.shape[0], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["q_start"][1:].contiguous(), row, right=True)
    token = st["kv_len"][seq] - st["q_start"][seq + 1] + row
    where = st["table"][seq, token // page].long(), slice(None), (token % page).long()
    st["k_pages"][where] = qk[:, H:]
    st["v_pages"][where] = x[:, H + Hk:]
    return qk[:, :H].reshape(-1, H * dh)


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "tree":
        return _plain_tree(st, case, st["q"])
    if kind == "probs":
        return _plain_probs(st["logits"], st["temperature"])
    if kind == "verify":
        return _plain_verify(st, st["logits"], st.get("draft"), case["draft"] == "points")
    if kind == "keep":
        kv = _plain_keep(st, case, st["path"], st["kept"])
        return {"kv_len": kv, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if kind == "fork":
        return _plain_fork(st, case)
    q = _plain_store(st, case)
    out = _plain_tree(st, case, q)
    p = _plain_probs(st["logits"], st["temperature"])
    got = _plain_verify(st, p, None, True)
    kv = _plain_keep(st, case, got["path"], got["kept"])
    return {"out": out, "p": p, **got, "kv_len": kv, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    if not own:
        return _plain(st)
    from paper_2503_12450_amd import binding as B
    case = st["case"]
    kind = case["kind"]
    if kind == "step":
        H, Hk, dh, x = case["heads"], case["kv_heads"], case["d_head"], st["qkv"]
        B.k_paged_store(st["batch"], x[:, H * dh:(H + Hk) * dh], x[:, (H + Hk) * dh:], q=x[:, :H * dh], q_out=st["q"],
                        rotary=st["rotary"], pos=st["pos"])
    if kind in ("tree", "step"):
        B.k_paged_tree_attention(st["batch"], st["q"], st["parent"], st["out"], window=case["window"],
                                 sinks=case["sinks"], workspace=st["workspace"])
    if kind == "tree":
        return st["out"]
    if kind in ("probs", "step"):
        B.k_probabilities(st["logits"], st["p"], temperature=st["temperature"])
    if kind == "probs":
        return st["p"]
    if kind in ("verify", "step"):
        greedy = kind == "verify" and case["draft"] == "greedy"
        B.k_draft_verify(st["q_start"], st["p"] if kind == "step" else st["logits"], st["parent"], st["tokens"],
                         st["path"], st["kept"], st["next"], random=None if greedy else st["random"],
                         draft=st.get("draft"), workspace=st["scratch"])
    got = {k: st[k] for k in ("path", "kept", "next")} if kind in ("verify", "step") else {}
    if kind == "verify":
        return got
    pages = {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if kind in ("keep", "step"):
        B.k_paged_keep(st["batch"], st["path"], st["kept"], st["kv_out"])
        pages["kv_len"] = st["kv_out"]
    if kind == "keep":
        return pages
    if kind == "step":
        return {"out": st["out"], "p": st["p"], **got, **pages}
    B.k_paged_fork(st["batch"], st["source"], st["table_out"], st["kv_out"], st["missing"], add=st["add"],
                   workspace=st["workspace"])
    return {"table": st["table_out"], "kv_len": st["kv_out"], "missing": st["missing"], **pages}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------

def _lineage(tree):
    """Every node's ancestors from itself upwards."""
    lines = []
    for i, p in enumerate(tree):
        lines.append([i] + (lines[p] if p >= 0 else []))
    return lines


def _tree64(case, st, q, k_pages, v_pages):
    H, Hk, dh, page, W = case["heads"], case["kv_heads"], case["d_head"], case["page"], case["window"]
    out = torch.zeros((q.shape[0], H, dh), dtype=torch.float64, device=DEV)
    q, first_row = q.view(-1, H, dh), 0
    for s, tree in enumerate(_parents(case)):
        n, L = len(tree), st["kv"][s]
        before, lines = L - n, _lineage(tree)
        hidden = torch.ones((n, L), dtype=torch.bool)
        for i, line in enumerate(lines):
            mine = before + len(line) - 1
            hidden[i, :before] = False
            if W:
                hidden[i, min(before, case["sinks"]):max(0, min(before, mine - W + 1))] = True
            for up, a in enumerate(line):
                hidden[i, before + a] = bool(W) and up >= W and mine - up >= case["sinks"]
        hidden = hidden.to(DEV)
        token = torch.arange(L, device=DEV)
        ids = st["table"][s].long()[token // page]
        for h in range(H):
            kh = k_pages[ids, h * Hk // H, token % page].to(torch.float64)
            vh = v_pages[ids, h * Hk // H, token % page].to(torch.float64)
            logit = (q[first_row:first_row + n, h].to(torch.float64) @ kh.T.contiguous()) / math.sqrt(dh)
            logit[hidden] = -math.inf
            out[first_row:first_row + n, h] = torch.exp(logit - torch.logsumexp(logit, 1, keepdim=True)) @ vh
        first_row += n
    return out.view(-1, H * dh)


def _probs64(logits, T):
    x, rows = logits.to(torch.float64), []
    for r, t in enumerate(T.tolist()):
        if t > 0:
            rows.append(torch.exp(x[r] / t - torch.logsumexp(x[r] / t, 0)))
        else:
            first = int((x[r] == x[r].max()).nonzero()[0])
            rows.append(torch.zeros_like(x[r]).index_fill_(0, torch.tensor([first], device=DEV), 1.0))
    return torch.stack(rows)


def _verify64(case, st, p, draft, greedy):
    path, kept, after, first = [], [], [], 0
    tokens, chance = st["tokens"].tolist(), st["random"].tolist()
    for tree in _parents(case):
        node, line, done = 0, [0], False
        while not done:
            weight, whole, done = p[first + node].to(torch.float64).clone(), 1.0, True
            for i in [i for i, up in enumerate(tree) if up == node and i > 0]:
                x, r = tokens[first + i], chance[first + i]
                if greedy:
                    take = x == int((weight == weight.max()).nonzero()[0])
                elif draft is None:
                    take = r * whole < float(weight[x])
                else:
                    q = draft[first + node].to(torch.float64)
                    take = r * float(q[x]) * whole < float(weight[x])
                if take:
                    node, done = i, False
                    line.append(i)
                    break
                if greedy:
                    continue
                if draft is None:
                    whole -= float(weight[x])
                    weight[x] = 0.0
                else:
                    rest = torch.relu(weight / whole - q)
                    if float(rest.sum()) > 0:
                        weight, whole = rest, float(rest.sum())
        if greedy:
            after.append(int((weight == weight.max()).nonzero()[0]))
        else:
            run_sum = torch.cumsum(weight, 0)
            after.append(int((run_sum > chance[first] * run_sum[-1]).nonzero()[0]))
        path += line + [-1] * (len(tree) - len(line))
        kept.append(len(line))
        first += len(tree)
    return {"path": _i32(path), "kept": _i32(kept), "next": _i32(after)}


def _keep64(case, st, k_pages, v_pages, path, kept):
    page, first, left = case["page"], 0, []
    for s, (n, a) in enumerate(zip(st["nodes"], kept)):
        before, ids = st["kv"][s] - n, st["table"][s].tolist()
        for i in range(a):
            of, to = before + path[first + i], before + i
            for pages in (k_pages, v_pages):
                pages[ids[to // page], :, to % page] = pages[ids[of // page], :, of % page].clone()
        first += n
        left.append(before + a)
    return _i32(left)


def _fork64(case, st, k_pages, v_pages):
    page, old, kv = case["page"], st["table"].tolist(), st["kv"]
    taken = {old[s][j] for s, L in enumerate(kv) for j in range(-(-L // page))}
    free = [p for p in range(k_pages.shape[0]) if p not in taken]
    source, add = st["source"].tolist(), st["add"].tolist()
    rows = [old[s][:-(-kv[s] // page)] for s in source]
    names, writers = {}, {}
    for i, s in enumerate(source):
        for p in rows[i]:
            names.setdefault(p, []).append(i)
        if add[i] > 0 and kv[s] % page:
            writers.setdefault(rows[i][-1], []).append(i)
    table, copies, missing = [], [], 0
    for i, s in enumerate(source):
        pages = list(rows[i])
        last = pages[-1]
        if i in writers.get(last, []) and len(names[last]) > 1 and not (len(names[last]) == len(writers[last])
                                                                       and writers[last][0] == i):
            pages.pop()
        while len(pages) < -(-(kv[s] + add[i]) // page):
            missing += not free
            pages.append(free.pop(0) if free else -1)
            if len(pages) == len(rows[i]):
                copies.append((last, pages[-1], kv[s] % page))
        table.append(pages + [-1] * (len(old[0]) - len(pages)))
    for of, to, n in copies:
        for pages in (k_pages, v_pages):
            pages[to, :, :n] = pages[of, :, :n]
    return {"table": _i32(table), "kv_len": _i32([kv[s] + a for s, a in zip(source, add)]), "missing": _i32([missing]),
            "k_pages": k_pages, "v_pages": v_pages}


def exact(case, seed):
    st, kind = _inputs(case, seed), case["kind"]
    if kind == "tree":
        return _tree64(case, st, st["q"], st["k_pages"], st["v_pages"])
    if kind == "probs":
        return _probs64(st["logits"], st["temperature"])
    if kind == "verify":
        return _verify64(case, st, st["logits"], st.get("draft"), case["draft"] == "greedy")
    k, v = st["k_pages"].to(torch.float64), st["v_pages"].to(torch.float64)
    if kind == "keep":
        kv = _keep64(case, st, k, v, st["path"].tolist(), st["kept"].tolist())
        return {"kv_len": kv, "k_pages": k, "v_pages": v}
    if kind == "fork":
        return _fork64(case, st, k, v)
    H, Hk, dh, page, t = case["heads"], case["kv_heads"], case["d_head"], case["page"], TDT[case["dtype"]]
    x = st["qkv"].view(-1, H + 2 * Hk, dh).to(torch.float64)
    phase = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), st["pos"].to(torch.float64) * st["freq"])
    z = torch.complex(x[:, :H + Hk, :dh // 2], x[:, :H + Hk, dh // 2:]) * phase[:, None]
    qk = torch.cat([z.real, z.imag], -1)
    first = 0
    for s, n in enumerate(st["nodes"]):
        token = torch.arange(st["kv"][s] - n, st["kv"][s], device=DEV)
        at = st["table"][s].long()[token // page], slice(None), token % page
        k[at], v[at] = qk[first:first + n, H:], x[first:first + n, H + Hk:]
        first += n
    # the attention reads what the store left in the cache, in the cache's type
    out = _tree64(case, st, qk[:, :H].reshape(-1, H * dh).to(t), k.to(t), v.to(t))
    p = _probs64(st["logits"], st["temperature"])
    got = _verify64(case, st, p, None, False)
    kv = _keep64(case, st, k, v, got["path"].tolist(), got["kept"].tolist())
    return {"out": out, "p": p, **got, "kv_len": kv, "k_pages": k, "v_pages": v}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _seen(case, tree, before):
    """(pairs of row and key, keys of the past that any row sees) of a tree."""
    W, sinks, pairs = case["window"], case["sinks"], 0
    for line in _lineage(tree):
        mine = before + len(line) - 1
        lo = max(0, min(before, mine - W + 1)) if W else 0
        pairs += before - lo + min(lo, sinks)
        pairs += sum(1 for up in range(len(line)) if not W or up < W or mine - up < sinks)
    lo = max(0, min(before, before - W + 1)) if W else 0
    return pairs, before - lo + min(lo, sinks)


def work(case):
    kind = case["kind"]
    es = 2 if case["dtype"] == "bf16" else 4
    if kind == "probs":
        return {"bytes": case["rows"] * (case["vocab"] * (es + 4) + 4), "flops": 4 * case["rows"] * case["vocab"]}
    nodes, past = _lengths(case)
    m, S, bytes_, flops = sum(nodes), case["seqs"], 0, 0
    if kind in ("tree", "step"):
        H, Hk, dh = case["heads"], case["kv_heads"], case["d_head"]
        pages = sum(-(-(a + b) // case["page"]) for a, b in zip(nodes, past))
        seen = [_seen(case, t, b) for t, b in zip(_parents(case), past)]
        bytes_ += 4 * (2 * S + 1 + pages + m) + 2 * m * H * dh * es + 2 * sum(k for _, k in seen) * Hk * dh * es
        bytes_ += 2 * m * Hk * dh * es
        flops += 4 * H * dh * sum(p for p, _ in seen)
    if kind == "step":
        bytes_ += 2 * m * (H + 2 * Hk) * dh * es + m * case["vocab"] * (es + 4)
        flops += 3 * m * (H + Hk) * dh + 4 * m * case["vocab"]
    if kind in ("verify", "step"):
        V, greedy = case["vocab"], case.get("draft") == "greedy"
        rows = m if greedy else S * (2 if case.get("draft") == "drawn" else 1)
        bytes_ += rows * V * (4 if kind == "step" else es) + 4 * (4 * m + 3 * S + 1)
        flops += rows * V
    if kind == "keep":
        # at most nine rows of a tree move; five do on average
        bytes_ += sum(2 * 2 * min(5, n // 4) * case["kv_heads"] * case["d_head"] * es for n in nodes) + 4 * (m + 4 * S)
        flops += 1
    if kind == "fork":
        page, n = case["page"], S * (1 + case["copies"])
        slots = sum(-(-b // page) for b in past)
        rows = sum(case["copies"] * (b % page) for b in past)
        bytes_ += 4 * slots * (2 + case["copies"]) + 12 * n + 2 * 2 * rows * case["kv_heads"] * case["d_head"] * es
        flops += 1
    return {"bytes": bytes_, "flops": flops}
