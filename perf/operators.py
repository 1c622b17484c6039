"""Rotary positions, the paged key/value cache and the attention that reads
it, as cases to be timed.

Four kinds:

rotary     rotary positions with one to four axes on the rows of a product
store      new tokens: queries rotated, keys rotated into the pages of the
           cache, values into the pages
attention  a ragged batch of new rows over the paged cache: single tokens,
           chunks, whole frames; causal or every key; a window of last keys
           with the first ones kept visible
step       the store and the attention after it, as a decoding step runs them

With `own` false `run` computes the plain form in elementary torch operations
(32 bits; angles in 64), with `own` true it makes the calls of the binding.

Inputs are drawn on the GPU from the seed.  The lengths of a batch follow from
the case alone: new rows per sequence between rows_lo and rows_hi, tokens
before them between past_lo and past_hi, spread over their logarithm by
`lengths`, a number that starts the generator.  Sequences own pages in a
random order, as after many allocations and releases.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
TDT = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _rotary(name, rows, heads, d_head, axes, layout, dtype, wide):
    return {"name": name, "kind": "rotary", "rows": rows, "heads": heads, "d_head": d_head, "axes": axes,
            "layout": layout, "dtype": dtype, "wide": wide}


def _batch(name, kind, seqs, rows, past, heads, kv_heads, d_head, page, dtype, causal=True, window=0, sinks=0,
           axes=3, layout="halves", lengths=1):
    return {"name": name, "kind": kind, "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "past_lo": past[0],
            "past_hi": past[1], "heads": heads, "kv_heads": kv_heads, "d_head": d_head, "page": page, "dtype": dtype,
            "causal": causal, "window": window, "sinks": sinks, "axes": axes, "layout": layout, "lengths": lengths}


def listed():
    return [
        # one token of both guidance pathways: queries and keys of a 16-head layer
        _rotary("rotary_token", 2, 32, 64, 3, "halves", "bf16", True),
        # whole images (64 with both pathways, 320 rows each) straight from the
        # query/key/value product: the value columns stay where they are
        _rotary("rotary_images", 40960, 32, 64, 2, "neighbours", "bf16", True),
        # one new token each of many sequences, shared key/value heads
        _batch("store_tokens", "store", 48, (1, 1), (10, 4000), 16, 4, 128, 64, "bf16"),
        # prompts and frames of several lengths into the cache, d_head 80
        _batch("store_chunks", "store", 8, (600, 4000), (0, 3000), 16, 16, 80, 32, "bf16", lengths=2),
        # the smallest call: one sequence, one token, a few hundred keys
        _batch("attention_token", "attention", 1, (1, 1), (320, 320), 12, 12, 64, 16, "bf16"),
        # single tokens of many sequences of very different lengths
        _batch("attention_tokens", "attention", 64, (1, 1), (500, 16000), 32, 4, 128, 64, "bf16", lengths=3),
        # one token of one very long sequence: its keys have to be split
        _batch("attention_token_long", "attention", 1, (1, 1), (131000, 131000), 16, 2, 128, 64, "bf16"),
        # chunks of long prompts over what is cached already
        _batch("attention_chunks", "attention", 4, (900, 1100), (14000, 16000), 16, 4, 128, 64, "bf16", lengths=4),
        # frames: every row of the new frame sees the frame and all earlier ones
        _batch("attention_frames", "attention", 32, (256, 256), (320, 1344), 16, 16, 80, 32, "bf16", causal=False,
               lengths=5),
        # long sequences with a window and the buffer rows as sinks
        _batch("attention_window", "attention", 2, (15000, 16000), (0, 0), 16, 16, 64, 64, "bf16", window=1024,
               sinks=64, lengths=6),
        # the fp32 path on ragged chunks
        _batch("attention_f32", "attention", 5, (30, 300), (100, 1500), 12, 12, 64, 16, "f32", lengths=7),
        # a serving step: single tokens of many sequences beside a prompt's chunk
        _batch("step_mixed", "step", 33, (1, 700), (200, 4000), 16, 4, 64, 32, "bf16", window=2048, sinks=64,
               lengths=8),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rotary", "store", "attention", "attention", "attention", "step"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    layout = rng.choice(("halves", "neighbours"))
    axes = rng.randint(1, 4)
    if kind == "rotary":
        d_head = rng.choice((16, 48, 64, 64, 80, 96, 128))
        heads = rng.randint(1, 40)
        c = _rotary("", _log(rng, 1, 8000000 // (heads * d_head)), heads, d_head, axes, layout, dtype,
                    rng.random() < 0.5)
        del c["name"]
        return c
    group = rng.choice((1, 1, 2, 4, 7, 8))
    kv_heads = rng.choice((1, 2, 4, 8)) if group > 1 else rng.choice((4, 12, 16))
    d_head = rng.choice((32, 64, 64, 80, 112, 128, 128))
    page = rng.choice((16, 16, 32, 64, 128))
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 16, 4000), rng.choice((0, 1, 4, 64, 100)))
    form = rng.choice(("tokens", "chunks", "mixed")) if kind != "store" else rng.choice(("tokens", "chunks"))
    if form == "tokens":
        seqs, rows, past = _log(rng, 1, 96), (1, rng.choice((1, 1, 4))), (1, _log(rng, 64, 12000))
    elif form == "chunks":
        n = _log(rng, 5, 2000)
        seqs, rows, past = _log(rng, 1, 8), (max(1, n // 3), n), (0, _log(rng, 16, 6000))
    else:
        seqs, rows, past = rng.randint(4, 40), (1, _log(rng, 8, 600)), (1, _log(rng, 64, 6000))
    if dtype == "f32":
        seqs, past = min(seqs, 16), (past[0], min(past[1], 3000))
    c = _batch("", kind, seqs, rows, past, group * kv_heads, kv_heads, d_head, page, dtype, rng.random() < 0.75, window,
               sinks, axes, layout, rng.randint(10, 10**6))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _lengths(case):
    """New rows and cached tokens of every sequence."""
    r = random.Random(case["lengths"])
    rows = [_log(r, case["rows_lo"], case["rows_hi"]) for _ in range(case["seqs"])]
    past = [_log(r, case["past_lo"] + 1, case["past_hi"] + 1) - 1 for _ in range(case["seqs"])]
    if case["kind"] == "step" and rows and case["rows_hi"] > 1:
        # single tokens, and the longest sequence with its whole chunk
        rows = [1] * (case["seqs"] - 1) + [case["rows_hi"]]
    return rows, past


def _frequencies(d_head, axes):
    """The d_head / 2 pairs in equal sections, each with its own frequencies
    base^(-j / section), as image models lay out height and width."""
    pairs = d_head // 2
    freq, axis = [], []
    for a in range(axes):
        n = pairs // axes + (1 if a < pairs % axes else 0)
        freq += [BASE ** (-j / n) for j in range(n)]
        axis += [a] * n
    return (torch.tensor(freq, dtype=torch.float64, device=DEV), torch.tensor(axis, dtype=torch.int32, device=DEV))


def _positions(first, n, axes):
    """Positions of n tokens from token `first` on: time counts frames of 256
    tokens, height and width the place in a 16 x 16 frame; one axis alone
    counts tokens."""
    t = torch.arange(first, first + n, device=DEV)
    cols = [t] if axes == 1 else [t // 256, t % 256 // 16, t % 16, t][:axes]
    return torch.stack(cols, 1).to(torch.int32)


def _rotary_inputs(case, seed):
    g, H, dh = _gen(seed), case["heads"], case["d_head"]
    width = H * dh + (H // 2 * dh if case["wide"] else 0)
    x = _normal(g, (case["rows"], width), 1.0, TDT[case["dtype"]])
    start = int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
    freq, axis = _frequencies(dh, case["axes"])
    return {"x": x, "pos": _positions(start, case["rows"], case["axes"]), "freq": freq, "axis": axis}


def _batch_inputs(case, seed):
    g, t = _gen(seed), TDT[case["dtype"]]
    rows, past = _lengths(case)
    kv = [a + b for a, b in zip(rows, past)]
    page, Hk, H, dh = case["page"], case["kv_heads"], case["heads"], case["d_head"]
    m = sum(rows)
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + 3  # some pages belong to nobody
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((case["seqs"], max(need)), dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    start = [0]
    for n in rows:
        start.append(start[-1] + n)
    st = {"rows": rows, "kv": kv, "table": table,
          "q_start": torch.tensor(start, dtype=torch.int32, device=DEV),
          "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
          "k_pages": _normal(g, (n_pages, Hk, page, dh), 1.0, t), "v_pages": _normal(g, (n_pages, Hk, page, dh), 1.0, t)}
    if case["kind"] == "attention":
        st["q"] = _normal(g, (m, H * dh), 1.5, t)
    else:
        # the rows of a query/key/value product
        st["qkv"] = _normal(g, (m, (H + 2 * Hk) * dh), 1.0, t)
        st["freq"], st["axis"] = _frequencies(dh, case["axes"])
        st["pos"] = torch.cat([_positions(p, n, case["axes"]) for n, p in zip(rows, past)])
    return st


def prepare(case, seed):
    st = _rotary_inputs(case, seed) if case["kind"] == "rotary" else _batch_inputs(case, seed)
    st["case"] = case
    if not own:
        return st
    from paper_2503_12450_amd import binding as B
    H, dh, t = case["heads"], case["d_head"], TDT[case["dtype"]]
    if case["kind"] != "attention":
        st["rotary"] = B.Rotary(st["freq"], st["axis"], case["axes"], case["layout"])
    if case["kind"] == "rotary":
        st["out"] = torch.empty((case["rows"], H * dh), dtype=t, device=DEV)
        return st
    st["pages"] = B.MarPages(st["k_pages"], st["v_pages"])
    st["batch"] = B.PagedBatch(st["pages"], st["table"], st["q_start"], st["kv_len"], max_kv=max(st["kv"]))
    m = sum(st["rows"])
    if case["kind"] != "attention":
        st["q"] = torch.empty((m, H * dh), dtype=t, device=DEV)
    if case["kind"] != "store":
        st["out"] = torch.empty((m, H * dh), dtype=t, device=DEV)
        n = B.paged_attention_workspace_bytes(st["batch"], m, H, window=case["window"], sinks=case["sinks"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _rotate(x, pos, freq, axis, layout):
    """x [rows, heads, d_head] rotated, in 32 bits."""
    angle = pos.double()[:, axis.long()] * freq
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    if layout == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _plain_store(st, case):
    H, Hk, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    t = TDT[case["dtype"]]
    x = st["qkv"].view(-1, H + 2 * Hk, dh)
    qk = _rotate(x[:, :H + Hk], st["pos"], st["freq"], st["axis"], case["layout"]).to(t)
    row = torch.arange(x.shape[0], device=DEV)
    seq = torch.searchsorted(st["q_start"][1:].contiguous(), row.to(torch.int32), right=True)
    token = st["kv_len"][seq] - st["q_start"][seq + 1] + row
    where = st["table"][seq, token // page].long(), slice(None), token % page
    st["k_pages"][where] = qk[:, H:]
    st["v_pages"][where] = x[:, H + Hk:]
    return qk[:, :H].reshape(-1, H * dh)


def _plain_attention(st, case, q):
    H, Hk, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    G, W, sinks = H // Hk, case["window"], case["sinks"]
    out = torch.empty_like(q)
    first = 0
    for s, (n, L) in enumerate(zip(st["rows"], st["kv"])):
        ids = st["table"][s, :-(-L // page)].long()
        k, v = (p[ids].transpose(0, 1).reshape(Hk, -1, dh) for p in (st["k_pages"], st["v_pages"]))
        step = max(1, 2 ** 28 // (H * L)) if not W else 1024
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            p = torch.arange(L - n + r0, L - n + r1, device=DEV)[:, None]
            lo = max(0, L - n + r0 - W + 1) if W else 0
            hi = L - n + r1 if case["causal"] else L
            j = torch.arange(lo, hi, device=DEV)
            if lo and sinks:
                j = torch.cat([torch.arange(min(lo, sinks), device=DEV), j])
            kj, vj = k[:, j].float(), v[:, j].float()
            qs = q[first + r0:first + r1].float().view(r1 - r0, Hk, G, dh).permute(1, 2, 0, 3).reshape(Hk, -1, dh)
            score = torch.matmul(qs, kj.transpose(1, 2).contiguous()).view(Hk, G, r1 - r0, -1) * dh ** -0.5
            seen = torch.ones((r1 - r0, j.numel()), dtype=torch.bool, device=DEV)
            if case["causal"]:
                seen &= j <= p
            if W:
                seen &= (j > p - W) | (j < sinks)
            score = score.masked_fill(~seen, -math.inf)
            weight = torch.exp(score - score.amax(-1, keepdim=True))
            o = torch.matmul(weight.view(Hk, -1, j.numel()), vj).view(Hk, G, r1 - r0, dh)
            o = o / weight.sum(-1, keepdim=True)
            out[first + r0:first + r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, H * dh).to(out.dtype)
        first += n
    return out


def _plain(st):
    case = st["case"]
    if case["kind"] == "rotary":
        H, dh = case["heads"], case["d_head"]
        x = st["x"][:, :H * dh].view(-1, H, dh)
        return _rotate(x, st["pos"], st["freq"], st["axis"], case["layout"]).to(x.dtype).view(-1, H * dh)
    if case["kind"] == "attention":
        return _plain_attention(st, case, st["q"])
    q = _plain_store(st, case)
    pages = {"q": q, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    return pages if case["kind"] == "store" else {"out": _plain_attention(st, case, q), **pages}


def run(st):
    if not own:
        return _plain(st)
    from paper_2503_12450_amd import binding as B
    case = st["case"]
    H, Hk, dh = case["heads"], case["kv_heads"] if "kv_heads" in case else 0, case["d_head"]
    if case["kind"] == "rotary":
        B.k_rotary(st["rotary"], st["x"][:, :H * dh], st["pos"], st["out"], d_head=dh)
        return st["out"]
    if case["kind"] != "attention":
        x = st["qkv"]
        B.k_paged_store(st["batch"], x[:, H * dh:(H + Hk) * dh], x[:, (H + Hk) * dh:], q=x[:, :H * dh], q_out=st["q"],
                        rotary=st["rotary"], pos=st["pos"])
    pages = {"q": st["q"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if case["kind"] == "store":
        return pages
    B.k_paged_attention(st["batch"], st["q"], st["out"], causal=case["causal"], window=case["window"],
                        sinks=case["sinks"], workspace=st["workspace"])
    return st["out"] if case["kind"] == "attention" else {"out": st["out"], **pages}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

def _turn64(x, pos, freq, axis, layout):
    """Every pair as a complex number times e^(i angle)."""
    P = freq.numel()
    phase = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.to(torch.float64)[:, axis.long()] * freq)
    x = x.to(torch.float64)
    z = torch.complex(x[..., :P], x[..., P:]) if layout == "halves" else torch.complex(x[..., ::2], x[..., 1::2])
    z = z * phase[:, None, :]
    out = torch.empty_like(x)
    if layout == "halves":
        out[..., :P], out[..., P:] = z.real, z.imag
    else:
        out[..., ::2], out[..., 1::2] = z.real, z.imag
    return out


def _attend64(case, st, q, k_pages, v_pages):
    H, Hk, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    out = torch.zeros((q.shape[0], H, dh), dtype=torch.float64, device=DEV)
    q = q.view(-1, H, dh)
    first = 0
    for s in range(case["seqs"]):
        n, L = st["rows"][s], st["kv"][s]
        token = torch.arange(L, device=DEV)
        at = st["table"][s].long()[token // page], token % page
        for r0 in range(0, n, 4096):
            r1 = min(n, r0 + 4096)
            place = L - n + torch.arange(r0, r1, device=DEV)
            back = place[:, None] - token[None, :]  # how far back a key lies
            hidden = torch.zeros_like(back, dtype=torch.bool)
            if case["causal"]:
                hidden |= back < 0
            if case["window"]:
                hidden |= (back >= case["window"]) & (token >= case["sinks"])[None, :]
            for h in range(H):
                kh = k_pages[at[0], h * Hk // H, at[1]].to(torch.float64)
                vh = v_pages[at[0], h * Hk // H, at[1]].to(torch.float64)
                logit = (q[first + r0:first + r1, h].to(torch.float64) @ kh.T.contiguous()) / math.sqrt(dh)
                logit[hidden] = -math.inf
                out[first + r0:first + r1, h] = torch.exp(logit - torch.logsumexp(logit, 1, keepdim=True)) @ vh
        first += n
    return out.view(-1, H * dh)


def exact(case, seed):
    H, dh = case["heads"], case["d_head"]
    if case["kind"] == "rotary":
        st = _rotary_inputs(case, seed)
        x = st["x"][:, :H * dh].reshape(-1, H, dh)
        return _turn64(x, st["pos"], st["freq"], st["axis"], case["layout"]).view(-1, H * dh)
    st = _batch_inputs(case, seed)
    if case["kind"] == "attention":
        return _attend64(case, st, st["q"], st["k_pages"], st["v_pages"])
    Hk, page = case["kv_heads"], case["page"]
    x = st["qkv"].view(-1, H + 2 * Hk, dh)
    q, k = (_turn64(part, st["pos"], st["freq"], st["axis"], case["layout"]) for part in (x[:, :H], x[:, H:H + Hk]))
    kp, vp = st["k_pages"].to(torch.float64), st["v_pages"].to(torch.float64)
    first = 0
    for s in range(case["seqs"]):
        n, L = st["rows"][s], st["kv"][s]
        for i in range(0, n, page):  # at most one page's worth of rows at a time
            token = torch.arange(L - n + i, L - n + min(n, i + page), device=DEV)
            at = st["table"][s].long()[token // page], slice(None), token % page
            kp[at] = k[first + i:first + i + token.numel()]
            vp[at] = x[first + i:first + i + token.numel(), H + Hk:].to(torch.float64)
        first += n
    pages = {"q": q.view(-1, H * dh), "k_pages": kp, "v_pages": vp}
    if case["kind"] == "store":
        return pages
    # the attention reads what the store left in the cache, in the cache's type
    t = TDT[case["dtype"]]
    return {"out": _attend64(case, st, pages["q"].to(t), kp.to(t), vp.to(t)), **pages}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _visible(case, n, L):
    """(pairs of query and key, keys that any query sees) of a sequence."""
    W, sinks = case["window"], case["sinks"]
    pairs, p0 = 0, L - n
    for p in range(p0, L):
        hi = p + 1 if case["causal"] else L
        lo = max(0, p - W + 1) if W else 0
        pairs += hi - lo + min(lo, sinks)
    lo = max(0, p0 - W + 1) if W else 0
    return pairs, L - lo + min(lo, sinks)


def work(case):
    es, H, dh = 2 if case["dtype"] == "bf16" else 4, case["heads"], case["d_head"]
    if case["kind"] == "rotary":
        m = case["rows"]
        return {"bytes": 2 * m * H * dh * es + 4 * m * case["axes"] + 6 * dh, "flops": 3 * m * H * dh}
    Hk = case["kv_heads"]
    rows, past = _lengths(case)
    m, pages = sum(rows), sum(-(-(a + b) // case["page"]) for a, b in zip(rows, past))
    bytes_ = 4 * (2 * case["seqs"] + 1 + pages)
    flops = 0
    if case["kind"] != "attention":
        bytes_ += 2 * m * (H + 2 * Hk) * dh * es + 4 * m * case["axes"]
        flops += 3 * m * (H + Hk) * dh
    if case["kind"] != "store":
        seen = [_visible(case, n, n + p) for n, p in zip(rows, past)]
        # the new keys and values of a step are written and read once each
        bytes_ += 2 * m * H * dh * es + 2 * sum(k for _, k in seen) * Hk * dh * es
        flops += 4 * H * dh * sum(p for p, _ in seen)
    return {"bytes": bytes_, "flops": flops}
