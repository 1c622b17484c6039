"""Plain fp64 forms of what decoding with drafted tokens does: attention of trees
over the paged cache, probabilities, verification, accepted rows moved together
and sequences continued by others; one row, one head and one token at a time, from
their definitions.  numpy only; nothing here is shared with the GPU path."""
from __future__ import annotations

import math
from typing import List, Optional

import numpy as np

MOST_NODES = 256


def ancestors(parent, q_start: int, i: int) -> List[int]:
    """Node i and those above it, upwards."""
    line = [i]
    while 0 <= parent[q_start + line[-1]] < line[-1]:
        line.append(int(parent[q_start + line[-1]]))
    return line


def tree_attention(q: np.ndarray, pages_k: np.ndarray, pages_v: np.ndarray, table, q_start, kv_len, parent,
                   window: int = 0, sinks: int = 0, max_kv: Optional[int] = None):
    """q [m, heads_q, d_head].  Returns (o, mean_abs, reach) as oracle.paged.attention
    does; rows of no sequence and nodes from the 256th on are NaN."""
    m, hq, dh = q.shape
    n_pages, hk, page, _ = pages_k.shape
    o = np.full((m, hq, dh), np.nan)
    mean_abs, reach = np.zeros((m, hq, dh)), np.zeros((m, hq))
    limit = table.shape[1] * page if max_kv is None else max_kv
    for s in range(len(kv_len)):
        start = int(q_start[s])
        n = int(q_start[s + 1]) - start
        L, first = min(int(kv_len[s]), limit), int(kv_len[s]) - n
        for i in range(min(n, MOST_NODES)):
            line = ancestors(parent, start, i)
            pos = first + len(line) - 1

            def near(p):
                return window == 0 or p > pos - window or p < sinks

            tokens = [j for j in range(max(0, min(first, L))) if near(j)]
            tokens += [first + a for up, a in enumerate(line) if near(pos - up) and 0 <= first + a < L]
            places = [(int(table[s][t // page]), t % page) for t in tokens]
            places = [w for w in places if 0 <= w[0] < n_pages]
            if not places:
                o[start + i] = 0.0
                continue
            at = np.array([w[0] for w in places]), np.array([w[1] for w in places])
            for h in range(hq):
                kk = pages_k[at[0], h // (hq // hk), at[1]].astype(np.float64)
                vv = pages_v[at[0], h // (hq // hk), at[1]].astype(np.float64)
                qq = q[start + i, h].astype(np.float64)
                score = kk @ qq / math.sqrt(dh)
                w = np.exp(score - score.max())
                w /= w.sum()
                o[start + i, h] = w @ vv
                mean_abs[start + i, h] = w @ np.abs(vv)
                reach[start + i, h] = (np.abs(kk) @ np.abs(qq)).max() / math.sqrt(dh)
    return o, mean_abs, reach


def probabilities(logits: np.ndarray, temperature=None) -> np.ndarray:
    x = logits.astype(np.float64)
    out = np.zeros_like(x)
    for r in range(x.shape[0]):
        T = 1.0 if temperature is None else float(temperature[r])
        if not T > 2.0 ** -100:
            known = np.where(np.isnan(x[r]), -np.inf, x[r])
            if known.max(initial=-np.inf) > -np.inf:
                out[r, int(np.argmax(known))] = 1.0
            continue
        with np.errstate(invalid="ignore"):
            e = np.where(x[r] == -np.inf, 0.0, np.exp((x[r] - np.max(x[r])) / T))
            out[r] = e / e.sum()
    return out


def _proper(x):
    x = np.asarray(x, dtype=np.float64)
    return np.where((x > 0) & (x < np.inf), x, 0.0)


def verify(p: np.ndarray, q_start, parent, tokens, random=None, draft: Optional[np.ndarray] = None):
    """(path [m], kept [n_seqs], next [n_seqs]); path is -2 where no sequence owns it."""
    m, V = p.shape
    S = len(q_start) - 1
    path, kept, after = np.full(m, -2, dtype=np.int64), np.zeros(S, dtype=np.int64), np.full(S, -1, dtype=np.int64)
    for s in range(S):
        start = min(max(int(q_start[s]), 0), m)
        n = max(min(max(int(q_start[s + 1]), 0), m) - start, 0)
        if n == 0:
            continue
        node, line = 0, [0]
        w, W = None, 1.0

        def best(row):
            known = np.where(np.isnan(p[row].astype(np.float64)), -np.inf, p[row].astype(np.float64))
            return int(np.argmax(known)) if known.max() > -np.inf else -1

        if random is not None:
            w = _proper(p[start])
        for i in range(1, min(n, MOST_NODES)):
            up = int(parent[start + i])
            if not 0 <= up < i or up != node:
                continue
            x = int(tokens[start + i])
            real = 0 <= x < V
            if random is None:
                take = real and x == best(start + node)
            else:
                r = float(random[start + i])
                d = None if draft is None else _proper(draft[start + node])
                chance = r * (1.0 if d is None else (d[x] if real else 0.0)) * W
                take = real and w[x] > 0 and bool(chance < w[x])
            if take:
                node = i
                line.append(i)
                if random is not None:
                    w, W = _proper(p[start + i]), 1.0
            elif random is not None and draft is None:
                if real:
                    W -= w[x]
                    w = w.copy()
                    w[x] = 0.0
            elif random is not None:
                rest = np.maximum(w / W - d, 0.0)
                if rest.sum() > 0:
                    w, W = rest, float(rest.sum())
        if random is None:
            after[s] = best(start + node)
        else:
            c = np.cumsum(w)
            over = np.flatnonzero((c > float(random[start]) * c[-1]) & (w > 0))
            some = np.flatnonzero(w > 0)
            after[s] = over[0] if len(over) else (some[-1] if len(some) else -1)
        path[start:start + n] = line + [-1] * (n - len(line))
        kept[s] = len(line)
    return path, kept, after


def keep(pages, table, q_start, kv_len, path, kept, max_kv: Optional[int] = None):
    """Rows moved in copies of the pages [n_pages, heads, page, d_head] (each of
    `pages`, in place); the lengths that remain."""
    n_pages, _, page, _ = pages[0].shape
    limit = table.shape[1] * page if max_kv is None else max_kv
    left = np.array(kv_len, dtype=np.int64)
    for s in range(len(kv_len)):
        start = int(q_start[s])
        n = int(q_start[s + 1]) - start
        if n <= 0:
            continue
        first, L = int(kv_len[s]) - n, min(int(kv_len[s]), limit)

        def place(t):
            if not 0 <= t < L or not 0 <= int(table[s][t // page]) < n_pages:
                return None
            return int(table[s][t // page]), t % page

        count = min(max(int(kept[s]), 0), n)
        for k in range(count):
            i = int(path[start + k])
            if not k < i < n:
                continue
            of, to = place(first + i), place(first + k)
            if of and to:
                for p in pages:
                    p[to[0], :, to[1]] = p[of[0], :, of[1]]
        left[s] = first + count
    return left


def fork(pages, table, kv_len, source, keep=None, add=None, max_kv: Optional[int] = None):
    """(table, kv_len, missing) of the new rows; copies are made in `pages`, in place."""
    n_pages, _, page, _ = pages[0].shape
    S, width = table.shape
    limit = width * page if max_kv is None else max_kv
    old_len = [min(max(int(n), 0), limit) for n in kv_len]
    entry = lambda s, j: int(table[s][j]) if 0 <= int(table[s][j]) < n_pages else -1
    used = {entry(s, j) for s in range(S) for j in range(-(-old_len[s] // page))}
    free = [p for p in range(n_pages) if p not in used]
    rows = []
    for i, s in enumerate(source):
        s = int(s)
        have = old_len[s] if 0 <= s < S else 0
        kept = have if keep is None else min(max(int(keep[i]), 0), have)
        length = min(kept + (0 if add is None else max(int(add[i]), 0)), width * page)
        rows.append((kept, length, [entry(s, j) for j in range(-(-kept // page))]))
    writes = [length > kept and kept % page != 0 and names[-1] >= 0 for kept, length, names in rows]
    out = np.full((len(rows), width), -1, dtype=np.int64)
    missing = 0
    copies = []
    for i, (kept, length, names) in enumerate(rows):
        mine = list(names)
        if writes[i]:
            last = names[-1]
            holders = sum(r[2].count(last) for r in rows)
            writers = [j for j in range(len(rows)) if writes[j] and rows[j][2][-1] == last]
            if holders > 1 and not (holders == len(writers) and writers[0] == i):
                mine.pop()
        copied = len(mine) < len(names)
        while len(mine) < -(-length // page):
            missing += not free
            mine.append(free.pop(0) if free else -1)
            if copied and len(mine) == len(names) and mine[-1] >= 0:
                copies.append((names[-1], mine[-1], kept % page))
        out[i, :len(mine)] = mine
    for of, to, n in copies:
        for p in pages:
            p[to, :, :n] = p[of, :, :n]
    return out, np.array([r[1] for r in rows], dtype=np.int64), missing
