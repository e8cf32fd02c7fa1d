"""Plain 64-bit statements of the 8-bit pages (h1b_kv8_*) and makers of small ragged batches, for the tests."""
import math

import numpy as np
import torch

TOP = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
EPS_HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # half a step, relative to the value


def numbers(codes: torch.Tensor, fmt: str) -> torch.Tensor:
    """The numbers 8-bit codes stand for, from their bits (float64)."""
    b = codes.view(torch.uint8).to(torch.int64)
    if fmt == "int8":
        return torch.where(b > 127, b - 256, b).double()
    e, f = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e > 0, torch.ldexp(1 + f / 8, e - 7), f / 8 * 2.0 ** -6)
    mag = torch.where((b & 127) == 127, math.nan, mag)
    return torch.where(b > 127, -mag, mag)


def nearest(x: torch.Tensor, fmt: str) -> torch.Tensor:
    """x (float64) to the nearest number of the format, ties to even."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def quantised(x: torch.Tensor, fmt: str):
    """(numbers, scales) of rows [..., d], float64; a row with an infinity or a NaN: zeros and NaN."""
    x = x.double()
    odd = ~torch.isfinite(x).all(-1)
    x = torch.where(odd[..., None], 0.0, x)
    amax = x.abs().amax(-1, keepdim=True)
    q = torch.where(amax > 0, nearest(x * TOP[fmt] / torch.where(amax > 0, amax, 1.0), fmt), 0.0)
    return q, torch.where(odd, math.nan, amax.squeeze(-1) / TOP[fmt])


class Batch:
    """A ragged batch on the host: rows and cached tokens per sequence, pages in shuffled order."""

    def __init__(self, rows, kv, page, seed=0, spare=2, extra_rows=0, width=None):
        rng = np.random.default_rng(seed)
        self.rows, self.kv, self.page = list(rows), list(kv), page
        need = [max(0, -(-t // page)) for t in kv]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(rows), width or max(need + [1])), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.free_pages = order[at:].tolist()
        self.row_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n_rows = int(self.row_start[-1]) + extra_rows

    def tensors(self, device="cuda"):
        return (torch.from_numpy(self.table).to(device), torch.tensor(self.kv, dtype=torch.int32, device=device),
                torch.from_numpy(self.row_start).to(device))

    def place(self, b, t):
        return int(self.table[b, t // self.page]), t % self.page


def empty_pool(n_pages, hkv, page, d, fmt, device="cuda", fill=0x5A):
    shape = (n_pages, hkv, page, d)
    k = torch.full(shape, fill, dtype=torch.uint8, device=device).view(CODE[fmt])
    v = torch.full(shape, fill, dtype=torch.uint8, device=device).view(CODE[fmt])
    return k, v, torch.full(shape[:3], -7.0, device=device), torch.full(shape[:3], -7.0, device=device)


def filled_pool(batch: Batch, hkv, d, fmt, seed, dtype=torch.float16, scale_spread=0.0):
    """Pages (on the host) holding quantised random rows for every cached token; everything no token lives in is garbage that
    must not matter: codes of all bits set and NaN scales."""
    g = torch.Generator().manual_seed(seed)
    k, v, ks, vs = empty_pool(batch.n_pages, hkv, batch.page, d, fmt, "cpu", fill=0x7F)
    ks.fill_(math.nan)
    vs.fill_(math.nan)
    loud = torch.where(torch.rand(hkv, d, generator=g) < 0.02, 8.0, 1.0)
    for b, t in enumerate(batch.kv):
        if t <= 0:
            continue
        pos = np.arange(t)
        p, o = torch.from_numpy(batch.table[b, pos // batch.page].astype(np.int64)), torch.from_numpy(pos % batch.page)
        for pages, scales in ((k, ks), (v, vs)):
            x = torch.randn(t, hkv, d, generator=g) * loud
            if scale_spread:
                x = x * torch.exp2(torch.randn(t, hkv, 1, generator=g) * scale_spread)
            q, sc = quantised(x.to(dtype), fmt)
            code = q.to(torch.int8).view(torch.uint8) if fmt == "int8" else q.float().to(torch.float8_e4m3fn).view(torch.uint8)
            pages.view(torch.uint8)[p, :, o] = code
            scales[p, :, o] = sc.float()
    return k, v, ks, vs


def attention(q, pool, batch: Batch, fmt, scale, window=0, sinks=0):
    """-> out, lse, mass = sum p |v|, reach = the largest sum |q_i k_i| |scale| of a row, grain = tokens seen times the largest
    value that the seen values' scales allow (all float64, on the host)."""
    k, v, ks, vs = pool
    hkv, d = k.shape[1], k.shape[3]
    hq = q.shape[1]
    g = hq // hkv
    out = torch.zeros(q.shape, dtype=torch.float64)
    mass, reach = torch.zeros_like(out), torch.zeros(q.shape[:2], dtype=torch.float64)
    grain = torch.zeros_like(reach)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    for b, (n, t) in enumerate(zip(batch.rows, batch.kv)):
        r0 = int(batch.row_start[b])
        if n == 0 or t <= 0:
            continue
        pos = np.arange(t)
        p, o = torch.from_numpy(batch.table[b, pos // batch.page].astype(np.int64)), torch.from_numpy(pos % batch.page)
        at = torch.arange(t - n, t)[:, None]
        tok = torch.arange(t)[None]
        seen = tok <= at
        if window:
            seen = seen & ((tok > at - window) | (tok < sinks))
        any_seen = seen.any(0)                            # what no row sees may be anything
        pp, oo = p.clamp(min=0), o
        for h in range(hkv):
            kk = numbers(k[pp, h, oo], fmt) * ks[pp, h, oo].double()[:, None]
            vv = numbers(v[pp, h, oo], fmt) * vs[pp, h, oo].double()[:, None]
            kk = torch.where(any_seen[:, None], kk, 0.0)
            vv = torch.where(any_seen[:, None], vv, 0.0)
            for j in range(g):
                x = q[r0:r0 + n, h * g + j].double()
                z = (x @ kk.T) * scale
                z = torch.where(seen, z, -math.inf)
                ab = torch.where(seen, (x.abs() @ kk.abs().T) * abs(scale), 0.0).amax(-1)
                w = torch.softmax(z, -1)
                w = torch.where(seen, w, 0.0)
                has = seen.any(-1)
                bad = torch.isnan(vv)
                y = torch.where(seen, w, 0.0) @ torch.where(bad, 0.0, vv)
                y = torch.where((seen.double() @ bad.double()) > 0, math.nan, y)      # a NaN value reaches the rows that see it
                out[r0:r0 + n, h * g + j] = torch.where(has[:, None], y, 0.0)
                mass[r0:r0 + n, h * g + j] = torch.where(has[:, None], w @ torch.where(bad, 0.0, vv).abs(), 0.0)
                lse[r0:r0 + n, h * g + j] = torch.logsumexp(z, -1)
                reach[r0:r0 + n, h * g + j] = ab
                grain[r0:r0 + n, h * g + j] = seen.sum(-1) * torch.where(seen, (vs[pp, h, oo].double() * TOP[fmt]).nan_to_num(0), 0.0).amax(-1)
    return out, lse, mass, reach, grain


def check_attention(got, got_lse, want, tag=""):
    """Tolerance, term by term. The dot product's products are exact and its fp32 sum of at most 128 terms loses at most
    2^-17 of sum |q k| (128 truncations of 2^-24 each); the scalings after it and the softmax reference lose a few 2^-24 of
    scores below 2^7 in size, the exponential 2^-21: together below 2^-16 + 2^-17 * reach in the exponent, twice (weight and
    sum). A weight is rounded to fp16: 2^-11, or, below 2^-14 of what it is carried in (2^9 or more of the largest, in units of
    at most twice the largest value scale), by 2^-25: at most 2^-33 of the largest value a token. The sums over tokens are fp32 chains of at most 2^11 truncations: 2^-13. All of
    it weighs on mass = sum p |v|. The result is rounded once: half a step."""
    out, lse, mass, reach, grain = want
    half = EPS_HALF[got.dtype]
    slack = 2 * (2.0 ** -16 + 2.0 ** -17 * reach)
    tol = half * out.abs() + (slack[..., None] + 2.0 ** -11 + 2.0 ** -13) * mass * (1 + half) + (2.0 ** -33 * grain)[..., None] + 2.0 ** -24
    g = got.cpu().double()
    assert torch.equal(torch.isnan(g), torch.isnan(out)), tag
    err = torch.where(torch.isnan(out), 0.0, (g - out).abs())
    worst = (err - tol).max().item() if err.numel() else -1.0
    assert worst <= 0, "%s: out is %.3g beyond its tolerance (largest error %.3g)" % (tag, worst, err.max().item())
    if got_lse is not None:
        gl = got_lse.cpu().double()
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(gl), empty), tag
        assert torch.equal(torch.isnan(gl), torch.isnan(lse)), tag
        fine = ~empty & ~torch.isnan(lse)
        ltol = slack + 2.0 ** -12 + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0, neginf=0)
        assert ((gl - lse).abs()[fine] <= ltol[fine]).all(), tag
