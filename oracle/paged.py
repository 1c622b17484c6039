"""Plain fp64 forms of the rotary positions, the paged cache's store and the
attention over it: one row, one head and one token at a time, from their
definitions.  numpy only; nothing here is shared with the GPU path."""
from __future__ import annotations

import math
from typing import Optional

import numpy as np


def rotary(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, axis: np.ndarray, layout: str) -> np.ndarray:
    """x [m, heads, d_head], pos [m, axes]; an axis that is none leaves its pair."""
    out = np.array(x, dtype=np.float64)
    P = len(freq)
    for i in range(P):
        a, b = (i, i + P) if layout == "halves" else (2 * i, 2 * i + 1)
        if not 0 <= axis[i] < pos.shape[1]:
            continue
        angle = pos[:, axis[i]].astype(np.float64) * float(freq[i])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        u, w = x[:, :, a].astype(np.float64), x[:, :, b].astype(np.float64)
        out[:, :, a], out[:, :, b] = u * c - w * s, w * c + u * s
    return out


def _places(table_row, n_pages: int, page: int, tokens: int):
    """(page, row) of every token, None where the table names no page."""
    out = []
    for t in range(tokens):
        p = int(table_row[t // page])
        out.append((p, t % page) if 0 <= p < n_pages else None)
    return out


def store(pages_k: np.ndarray, pages_v: np.ndarray, k: np.ndarray, v: np.ndarray, table, q_start, kv_len,
          max_kv: Optional[int] = None) -> None:
    """Rows k, v [m, heads, d_head] of the batch's new tokens into copies of
    the pages [n_pages, heads, page, d_head], in place."""
    n_pages, _, page, _ = pages_k.shape
    limit = table.shape[1] * page if max_kv is None else max_kv
    for s in range(len(kv_len)):
        n = q_start[s + 1] - q_start[s]
        for i in range(n):
            t = int(kv_len[s]) - n + i
            if not 0 <= t < limit:
                continue
            p = int(table[s][t // page])
            if 0 <= p < n_pages:
                pages_k[p, :, t % page] = k[q_start[s] + i]
                pages_v[p, :, t % page] = v[q_start[s] + i]


def attention(q: np.ndarray, pages_k: np.ndarray, pages_v: np.ndarray, table, q_start, kv_len, causal: bool,
              window: int = 0, sinks: int = 0, max_kv: Optional[int] = None):
    """q [m, heads_q, d_head].  Returns (o, mean_abs, reach): the output, the
    same weights' mean of |v| (what a relative error of the weights is taken
    of), and per row and head the largest sum_d |q_d k_d| / sqrt(d_head) over
    the visible tokens (what the rounding of a score is taken of).  Rows of no
    sequence are NaN."""
    m, hq, dh = q.shape
    n_pages, hk, page, _ = pages_k.shape
    o = np.full((m, hq, dh), np.nan)
    mean_abs = np.zeros((m, hq, dh))
    reach = np.zeros((m, hq))
    limit = table.shape[1] * page if max_kv is None else max_kv
    for s in range(len(kv_len)):
        n = int(q_start[s + 1] - q_start[s])
        L = min(int(kv_len[s]), limit)
        where = _places(table[s], n_pages, page, L)
        for i in range(n):
            r, p = int(q_start[s]) + i, int(kv_len[s]) - n + i
            seen = [w for j, w in enumerate(where)
                    if w is not None and (not causal or j <= p) and (window == 0 or j > p - window or j < sinks)]
            if not seen:
                o[r] = 0.0
                continue
            at = np.array([w[0] for w in seen]), np.array([w[1] for w in seen])
            for h in range(hq):
                kk = pages_k[at[0], h // (hq // hk), at[1]].astype(np.float64)
                vv = pages_v[at[0], h // (hq // hk), at[1]].astype(np.float64)
                qq = q[r, h].astype(np.float64)
                score = kk @ qq / math.sqrt(dh)
                w = np.exp(score - score.max())
                w /= w.sum()
                o[r, h] = w @ vv
                mean_abs[r, h] = w @ np.abs(vv)
                reach[r, h] = (np.abs(kk) @ np.abs(qq)).max() / math.sqrt(dh)
    return o, mean_abs, reach
