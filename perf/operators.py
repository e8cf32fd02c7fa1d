"""The 8-bit paged cache (h1b_kv8_*): what its operators compute, on which sizes they are measured, and their plain forms.

Three operators share one pool of pages (codes [n_pages, Hkv, page_tokens, d], one fp32 scale per token and head) and one
description of a ragged batch (block_table [B, W], kv_len [B], row_start [B + 1]):

  append     new key and value rows are quantised as they are written: scale = amax / top, code = round(top * x / amax),
             top = 127 (int8, to the nearest integer, ties to even) or 448 (e4m3, to the nearest e4m3 number, ties to even);
  read       cached rows come back as code * scale, rounded once to fp16 or bf16;
  attention  the last rows of every sequence attend to its cached tokens, out = softmax(scale * q k) v, causal, optionally
             only the `window` last tokens and the `sinks` first ones; one row per sequence (decoding) up to whole prompts.

Row r of sequence b (row_start[b] <= r < row_start[b + 1]) is the token at position kv_len[b] - row_start[b + 1] + r.
"""
import math

import numpy as np
import torch

own = False

TOP = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TYPE = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one decode step of a ragged batch writes one token per sequence: the smallest call, all latency
        dict(name="append_step_16", op="append", seqs=16, rows_lo=1, rows_hi=1, kv_lo=4096, kv_hi=8192, hkv=8, d=128, page=64, fmt="int8", dtype="bf16"),
        # chunks of prompts of several users, narrow heads, odd lengths
        dict(name="append_chunks_64", op="append", seqs=12, rows_lo=17, rows_hi=1021, kv_lo=1021, kv_hi=3001, hkv=8, d=64, page=32, fmt="e4m3", dtype="bf16"),
        # a whole 8192-token prompt of a 7B-shaped model
        dict(name="append_prompt_8k", op="append", seqs=1, rows_lo=8192, rows_hi=8192, kv_lo=8192, kv_hi=8192, hkv=32, d=128, page=64, fmt="int8", dtype="fp16"),
        # a few hundred aged tokens go back to fp16, to be compressed further
        dict(name="read_aged_509", op="read", seqs=4, rows_lo=130, rows_hi=509, kv_lo=2000, kv_hi=4099, hkv=8, d=128, page=16, fmt="int8", dtype="fp16"),
        # whole sequences are read back (a prefix moves to another cache)
        dict(name="read_prefix_4k", op="read", seqs=8, rows_lo=2050, rows_hi=4096, kv_lo=4096, kv_hi=8192, hkv=32, d=128, page=64, fmt="e4m3", dtype="bf16"),
        # one short sequence of a small model: latency
        dict(name="decode_60m_777", op="attention", seqs=1, rows_lo=1, rows_hi=1, kv_lo=777, kv_hi=777, hq=8, hkv=8, d=64, page=32, fmt="int8", dtype="fp16", window=0, sinks=0),
        # batched decoding of a 7B-shaped model, ragged contexts
        dict(name="decode_7b_b16", op="attention", seqs=16, rows_lo=1, rows_hi=1, kv_lo=4096, kv_hi=8192, hq=32, hkv=32, d=128, page=64, fmt="int8", dtype="fp16", window=0, sinks=0),
        # long contexts with grouped query heads
        dict(name="decode_gqa_32k", op="attention", seqs=8, rows_lo=1, rows_hi=1, kv_lo=32768, kv_hi=32768, hq=32, hkv=8, d=128, page=128, fmt="e4m3", dtype="bf16", window=0, sinks=0),
        # streaming: a window and four sinks, contexts from shorter than the window to long
        dict(name="decode_window_b32", op="attention", seqs=32, rows_lo=1, rows_hi=1, kv_lo=100, kv_hi=32768, hq=32, hkv=8, d=64, page=32, fmt="e4m3", dtype="fp16", window=1024, sinks=4),
        # a step that verifies a few tokens for some users and takes chunks of others
        dict(name="chunk_ragged_6", op="attention", seqs=6, rows_lo=5, rows_hi=131, kv_lo=901, kv_hi=9001, hq=32, hkv=8, d=128, page=16, fmt="int8", dtype="bf16", window=0, sinks=0),
        # a chunk over a long cache, window and sinks
        dict(name="chunk_window_2k", op="attention", seqs=1, rows_lo=2048, rows_hi=2048, kv_lo=32768, kv_hi=32768, hq=32, hkv=8, d=128, page=64, fmt="e4m3", dtype="bf16", window=4096, sinks=64),
        # a whole prompt of a 7B-shaped model
        dict(name="prompt_7b_8k", op="attention", seqs=1, rows_lo=8192, rows_hi=8192, kv_lo=8192, kv_hi=8192, hq=32, hkv=32, d=128, page=64, fmt="int8", dtype="fp16", window=0, sinks=0),
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    while True:
        op = rng.choice(["append", "read", "decode", "decode", "chunk", "chunk"])
        c = dict(op=op if op in ("append", "read") else "attention", d=rng.choice([64, 128]), page=rng.choice([16, 32, 48, 64, 128, 256]),
                 fmt=rng.choice(["int8", "e4m3"]), dtype=rng.choice(["fp16", "bf16"]))
        c["hkv"] = rng.choice([1, 2, 4, 8, 8, 16, 32])
        if op == "decode":
            c.update(seqs=size(1, 64), rows_lo=1, rows_hi=1)
            c["kv_hi"] = size(1, 32768)
            c["kv_lo"] = size(1, c["kv_hi"])
            most = 131072 * 8
        else:
            c["seqs"] = size(1, 16)
            c["rows_hi"] = size(1, 4096)
            c["rows_lo"] = size(1, c["rows_hi"])
            c["kv_hi"] = min(32768, c["rows_hi"] + size(1, 16384) - 1)
            c["kv_lo"] = c["rows_hi"] + (0 if c["kv_hi"] == c["rows_hi"] else size(1, c["kv_hi"] - c["rows_hi"] + 1) - 1)
            most = 131072 * 4
        if c["op"] == "attention":
            c["hq"] = c["hkv"] * rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16])
            if c["hq"] > 64:
                continue
            c["window"] = rng.choice([0, 0, size(1, 8192)])
            c["sinks"] = size(1, 128) - 1 if c["window"] else 0
            # no more scores than the prompt's, in the plain form either
            if c["seqs"] * c["hq"] * c["rows_hi"] * c["kv_hi"] > 32 * 8192 * 8192:
                continue
        if c["seqs"] * c["kv_hi"] * c["hkv"] > most * 8:
            continue
        return c


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], ragged but the same every time; the largest one is hi."""
    at = [lo + int((hi - lo + 1) * ((0.31 + 0.6180339887498949 * i) % 1.0)) for i in range(n)]
    at[n // 2] = hi
    return at


def _plan(c):
    """Per sequence: new (or wanted) rows, cached tokens."""
    rows = _spread(c["rows_lo"], c["rows_hi"], c["seqs"])
    kv = [max(a, b) for a, b in zip(_spread(c["kv_lo"], c["kv_hi"], c["seqs"]), rows)]
    return rows, kv


def _pairs(c):
    """(query row, token) pairs, and tokens that some row of the sequence sees, over all sequences."""
    pairs = seen = 0
    w, s = c["window"], c["sinks"]
    for n, kv in zip(*_plan(c)):
        p = np.arange(kv - n, kv, dtype=np.int64)
        pairs += int((p + 1).sum()) if not w else int((np.minimum(p + 1, w) + np.minimum(s, np.maximum(0, p + 1 - w))).sum())
        first = 0 if not w else max(0, kv - n + 1 - w)
        seen += kv - first + min(s, first)
    return pairs, seen


def work(case):
    c = case
    rows, kv = _plan(c)
    n, d = sum(rows), c["d"]
    if c["op"] != "attention":  # two bytes and one byte a number, a scale a row, keys and values
        return {"bytes": n * c["hkv"] * 2 * (3 * d + 4), "flops": n * c["hkv"] * 2 * 3 * d}
    pairs, seen = _pairs(c)
    return {"bytes": seen * c["hkv"] * 2 * (d + 4) + n * c["hq"] * (4 * d + 4), "flops": pairs * c["hq"] * 4 * d}


# ---------------------------------------------------------------- inputs

def _quantise(x, fmt):
    """(codes, scales) of rows x [..., d]: in 32 bits every step but the quotient and the scale is exact."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    q = torch.where(amax > 0, (x * TOP[fmt]) / amax, torch.zeros_like(x))
    return (q.round() if fmt == "int8" else q).to(CODE[fmt]), (amax / TOP[fmt]).squeeze(-1)


def _rows(gen, n, heads, d, dtype, loud):
    x = torch.randn(n, heads, d, generator=gen, device="cuda", dtype=torch.float32)
    return (x * loud).to(TYPE[dtype])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    rng = np.random.default_rng(int(seed) + 1)
    rows, kv = _plan(c)
    page, hkv, d = c["page"], c["hkv"], c["d"]
    need = [-(-t // page) for t in kv]
    n_pages = sum(need) + 3
    order = rng.permutation(n_pages)[:sum(need)]
    table = np.full((c["seqs"], max(need)), -1, np.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    # one channel in a hundred is loud in keys and values
    loud = torch.where(torch.rand(hkv, d, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    shape = (n_pages, hkv, page, d)
    n = sum(rows)
    s = {"op": c["op"], "case": c, "n_rows": n, "max_rows": max(rows), "max_kv": max(kv),
         "block_table": torch.from_numpy(table).cuda(), "kv_len": torch.tensor(kv, dtype=torch.int32).cuda(),
         "row_start": torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).cuda()}
    if c["op"] == "append":
        s["k"], s["v"] = _rows(gen, n, hkv, d, c["dtype"], loud), _rows(gen, n, hkv, d, c["dtype"], loud)
        for x in ("k", "v"):
            s[x + "_pages"] = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(CODE[c["fmt"]])
            s[x + "_scale"] = torch.zeros(shape[:3], dtype=torch.float32, device="cuda")
        return s
    for x in ("k", "v"):
        pages = torch.empty(shape, dtype=torch.uint8, device="cuda")
        scale = torch.empty(shape[:3], dtype=torch.float32, device="cuda")
        step = max(1, (1 << 26) // (hkv * page * d))
        for p in range(0, n_pages, step):
            m = min(step, n_pages - p)
            codes, sc = _quantise(_rows(gen, m * page, hkv, d, c["dtype"], loud), c["fmt"])
            pages[p:p + m] = codes.view(torch.uint8).view(m, page, hkv, d).transpose(1, 2)
            scale[p:p + m] = sc.view(m, page, hkv).transpose(1, 2)
        s[x + "_pages"], s[x + "_scale"] = pages.view(CODE[c["fmt"]]), scale
    if c["op"] == "attention":
        s["q"] = _rows(gen, n, c["hq"], d, c["dtype"], 1.0)
        s["scale"] = 1.0 / math.sqrt(d)
    return s


# ---------------------------------------------------------------- the operators

def run(state):
    if own:
        return _call(state)
    return {"append": _append, "read": _read, "attention": _attention}[state["op"]](state)


def _call(s):
    from paper_2510_05529_b200 import binding
    if "pages" not in s:  # the pool's handle, which a program makes once
        s["pages"] = binding.KV8Pages(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
    pages, batch = s["pages"], (s["block_table"], s["kv_len"], s["row_start"])
    if s["op"] == "append":
        pages.h1b_kv8_append(s["k"], s["v"], *batch)
        return {"k": s["k_pages"], "v": s["v_pages"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if s["op"] == "read":
        k, v = pages.h1b_kv8_read(*batch, n_rows=s["n_rows"], dtype=TYPE[s["case"]["dtype"]])
        return {"k": k, "v": v}
    c = s["case"]
    out, lse = pages.h1b_kv8_attention(s["q"], *batch, scale=s["scale"], window=c["window"], sinks=c["sinks"], max_rows=s["max_rows"], return_lse=True)
    return {"out": out, "lse": lse}


def _slots(s, n):
    """Page and place in it of the rows 0 .. n - 1."""
    r = torch.arange(n, device="cuda")
    starts = s["row_start"].long()
    b = torch.searchsorted(starts, r, right=True) - 1
    pos = s["kv_len"].long()[b] - starts[b + 1] + r
    page = s["case"]["page"]
    return s["block_table"].long()[b, pos // page], pos % page


def _append(s):
    at = _slots(s, s["k"].shape[0])
    for x in ("k", "v"):
        codes, scale = _quantise(s[x], s["case"]["fmt"])
        s[x + "_pages"].view(torch.uint8)[at[0], :, at[1]] = codes.view(torch.uint8)
        s[x + "_scale"][at[0], :, at[1]] = scale
    return {"k": s["k_pages"], "v": s["v_pages"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _read(s):
    at = _slots(s, s["n_rows"])
    out = {}
    for x in ("k", "v"):
        codes = s[x + "_pages"].view(torch.uint8)[at[0], :, at[1]].view(CODE[s["case"]["fmt"]])
        out[x] = (codes.float() * s[x + "_scale"][at[0], :, at[1]].unsqueeze(-1)).to(TYPE[s["case"]["dtype"]])
    return out


def _attention(s):
    c, q, page = s["case"], s["q"], s["case"]["page"]
    n_rows, hq, d = q.shape
    hkv, m, t_max = c["hkv"], s["max_rows"], s["max_kv"]
    starts, kv = s["row_start"].long(), s["kv_len"].long()
    n = starts[1:] - starts[:-1]
    i, t = torch.arange(m, device="cuda"), torch.arange(t_max, device="cuda")
    row = (starts[:-1, None] + i).clamp(max=n_rows - 1)  # [B, m]
    slot = s["block_table"].long()[:, t // page].clamp(min=0)  # [B, T]

    def cached(x):  # [B, Hkv, T, d]
        codes = s[x + "_pages"].view(torch.uint8)[slot, :, t % page].view(CODE[c["fmt"]]).float()
        return (codes * s[x + "_scale"][slot, :, t % page].unsqueeze(-1)).transpose(1, 2)

    qs = q[row].float().view(-1, m, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)  # [B, Hkv, G, m, d]
    shape = qs.shape[:4]
    scores = (qs.reshape(shape[0], hkv, -1, d) @ cached("k").transpose(2, 3)).mul_(s["scale"]).view(*shape, t_max)
    pos = (kv - n)[:, None] + i  # [B, m]
    seen = (t <= pos[:, :, None]) & (i < n[:, None])[:, :, None]
    if c["window"]:
        seen &= (t > pos[:, :, None] - c["window"]) | (t < c["sinks"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(torch.isfinite(top), top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    got = (p.view(shape[0], hkv, -1, t_max) @ cached("v")).view(*shape, d) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    keep = i < n[:, None]  # [B, m]: the rows in order are the batch's rows
    out = got.permute(0, 3, 1, 2, 4).reshape(-1, m, hq, d)[keep].to(q.dtype)
    return {"out": out, "lse": lse.permute(0, 3, 1, 2).reshape(-1, m, hq)[keep]}


# ---------------------------------------------------------------- the definition, in 64 bits

def _number(codes, fmt):
    """The numbers that 8-bit codes stand for, from their bits."""
    b = codes.view(torch.uint8).to(torch.int64)
    if fmt == "int8":
        return torch.where(b > 127, b - 256, b).double()
    e, f = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e > 0, torch.ldexp(1 + f / 8, e - 7), f / 8 * 2.0 ** -6)
    return torch.where(b > 127, -mag, mag)


def _nearest(x, fmt):
    """x to the nearest number of the format, ties to even, in 64 bits."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    c, s = case, prepare(case, seed)
    rows, kv = _plan(c)
    table = s["block_table"].cpu().numpy()
    page, fmt, hkv, d = c["page"], c["fmt"], c["hkv"], c["d"]

    def places(b, lo, hi):
        t = np.arange(lo, hi)
        return torch.from_numpy(table[b, t // page].astype(np.int64)).cuda(), torch.from_numpy(t % page).cuda()

    if c["op"] == "append":
        out, r = {}, 0
        for x in ("k", "v"):
            out[x], out[x + "_scale"] = torch.zeros(s[x + "_pages"].shape, dtype=torch.float64, device="cuda"), torch.zeros_like(s[x + "_scale"], dtype=torch.float64)
        for b, (n, t) in enumerate(zip(rows, kv)):
            p, o = places(b, t - n, t)
            for x in ("k", "v"):
                v = s[x][r:r + n].double()
                amax = v.abs().amax(-1, keepdim=True)
                out[x][p, :, o] = torch.where(amax > 0, _nearest(v * TOP[fmt] / amax, fmt), 0.0)
                out[x + "_scale"][p, :, o] = amax.squeeze(-1) / TOP[fmt]
            r += n
        if fmt == "int8":
            out["k"], out["v"] = out["k"].to(torch.int8), out["v"].to(torch.int8)
        return out
    if c["op"] == "read":
        out = {"k": [], "v": []}
        for b, (n, t) in enumerate(zip(rows, kv)):
            p, o = places(b, t - n, t)
            for x in ("k", "v"):
                out[x].append(_number(s[x + "_pages"].view(torch.uint8)[p, :, o], fmt) * s[x + "_scale"][p, :, o].double().unsqueeze(-1))
        return {x: torch.cat(v) for x, v in out.items()}
    g = c["hq"] // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    r = 0
    for b, (n, t) in enumerate(zip(rows, kv)):
        p, o = places(b, 0, t)
        for h in range(hkv):
            k, v = (_number(s[x + "_pages"].view(torch.uint8)[p, h, o], fmt) * s[x + "_scale"][p, h, o].double()[:, None] for x in ("k", "v"))
            for r0 in range(0, n, 1024):
                m = min(1024, n - r0)
                q = s["q"][r + r0:r + r0 + m, h * g:(h + 1) * g].double()
                z = torch.einsum("ngd,td->ngt", q, k) * s["scale"]
                at = torch.arange(t - n + r0, t - n + r0 + m, device="cuda")[:, None]
                tok = torch.arange(t, device="cuda")[None]
                hidden = tok > at
                if c["window"]:
                    hidden = hidden | ((tok <= at - c["window"]) & (tok >= c["sinks"]))
                z = z.masked_fill(hidden[:, None], -math.inf)
                lse[r + r0:r + r0 + m, h * g:(h + 1) * g] = torch.logsumexp(z, -1)
                out[r + r0:r + r0 + m, h * g:(h + 1) * g] = torch.einsum("ngt,td->ngd", torch.softmax(z, -1), v)
        r += n
    return {"out": out, "lse": lse}
