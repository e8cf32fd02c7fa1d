"""8-bit pages on the GPU: quantise-and-append and read-back bit for bit, attention against the 64-bit definition."""
import math

import numpy as np
import pytest
import torch

import kv8_testlib as lib
from kv8_testlib import Batch, attention, check_attention, empty_pool, filled_pool, numbers, quantised

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def binding():
    from paper_2510_05529_b200 import binding as b
    b.load_library()
    return b


def pages_of(binding, pool):
    return binding.KV8Pages(*(t.cuda() if not t.is_cuda else t for t in pool))


# ------------------------------------------------------------------------------------------------ append, read

def hard_rows(n, hkv, d, dtype, seed):
    """Rows with what quantisers get wrong: zeros, ties at amax / 2, one huge number, subnormals, infinities and NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, hkv, d, generator=g)
    flat = x.view(-1, d)
    m = flat.shape[0]
    flat[0 % m] = 0.0
    flat[1 % m, 0], flat[1 % m, 1] = 8.0, 4.0
    flat[2 % m] *= torch.finfo(dtype).tiny
    flat[3 % m] = torch.finfo(dtype).max * torch.linspace(-1, 1, d)
    flat[4 % m, d - 1] = math.inf
    flat[5 % m, 3] = math.nan
    flat[6 % m] = torch.linspace(-2, 2, d)
    flat[7 % m] = torch.randint(-7, 8, (d,), generator=g).float() * 32         # amax a multiple of 7: ties of e4m3
    return x.to(dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,kv,hkv,page", [
    ([1], [1], 1, 16),
    ([1, 0, 3], [1, 40, 33], 3, 32),
    ([1] * 40, list(range(1, 41)), 8, 48),
    ([130, 17, 0, 257], [130, 400, 5, 258], 5, 64),
])
def test_append_and_read_bit_for_bit(binding, d, fmt, dtype, rows, kv, hkv, page):
    b = Batch(rows, kv, page, seed=3, extra_rows=2)
    pages = pages_of(binding, empty_pool(b.n_pages, hkv, page, d, fmt))
    k, v = hard_rows(b.n_rows, hkv, d, dtype, 1), hard_rows(b.n_rows, hkv, d, dtype, 2).flip(0)
    args = b.tensors()
    pages.h1b_kv8_append(k.cuda(), v.cuda(), *args)
    pages.h1b_kv8_poll_status()
    want = [t.clone() for t in empty_pool(b.n_pages, hkv, page, d, fmt, "cpu")]
    r = 0
    for s, (n, t) in enumerate(zip(rows, kv)):
        for i in range(n):
            p, o = b.place(s, t - n + i)
            for x, codes, scales in ((k, want[0], want[2]), (v, want[1], want[3])):
                q, sc = quantised(x[r], fmt)
                q = q.to(torch.int8) if fmt == "int8" else (q.float() + 0.0 * x[r].float().nan_to_num(0, 0, 0)).to(torch.float8_e4m3fn)
                codes.view(torch.uint8)[p, :, o] = q.view(torch.uint8)
                scales[p, :, o] = sc.float()
            r += 1
    for got, w in zip((pages.k_pages, pages.v_pages), want[:2]):
        if fmt == "int8":
            assert torch.equal(got.cpu(), w)
        else:                                              # (a zero's sign is not part of the definition)
            assert torch.equal(numbers(got.cpu(), fmt).nan_to_num(nan=1e9), numbers(w, fmt).nan_to_num(nan=1e9))
    for got, w in zip((pages.k_scale, pages.v_scale), want[2:]):
        assert torch.equal(got.cpu().nan_to_num(nan=1e9), w.nan_to_num(nan=1e9))
    # read back: code * scale in fp32, rounded once; rows that are nobody's keep what they held
    for out_type in (F16, BF16):
        ko, vo = (torch.full((b.n_rows, hkv, d), 3.0, dtype=out_type, device="cuda") for _ in "kv")
        pages.h1b_kv8_read(*args, k=ko, v=vo)
        r = 0
        for s, (n, t) in enumerate(zip(rows, kv)):
            for i in range(n):
                p, o = b.place(s, t - n + i)
                for got, codes, scales in ((ko, want[0], want[2]), (vo, want[1], want[3])):
                    w = (numbers(codes[p, :, o], fmt).float() * scales[p, :, o][:, None]).to(out_type)
                    assert torch.equal(got[r].cpu().nan_to_num(nan=77.0), w.nan_to_num(nan=77.0))
                r += 1
        assert (ko[r:] == 3.0).all() and (vo[r:] == 3.0).all()
        only = torch.full_like(ko, 5.0)
        assert pages.h1b_kv8_read(*args, v=only)[0] is None
        assert torch.equal(only[:r].nan_to_num(nan=77.0), vo[:r].nan_to_num(nan=77.0))


@pytest.mark.parametrize("order", ["fused", "heads_first", "reversed_slices"])
def test_append_and_read_take_strided_rows(binding, order):
    b, hkv, d, n = Batch([5, 9], [30, 9], 16, seed=1), 4, 128, 14
    g = torch.Generator().manual_seed(5)
    if order == "fused":                                   # slices of one [n, (k v), hkv, d] tensor
        both = torch.randn(n, 2, hkv, d, generator=g).to(BF16).cuda()
        k, v = both[:, 0], both[:, 1]
    elif order == "heads_first":
        k, v = (torch.randn(hkv, n, d, generator=g).to(BF16).cuda().transpose(0, 1) for _ in "kv")
    else:                                                  # every second head, and one row repeated for all
        k = torch.randn(n, 2 * hkv, d, generator=g).to(BF16).cuda()[:, ::2]
        v = torch.randn(1, hkv, d, generator=g).to(BF16).cuda().expand(n, hkv, d)
    pools = [pages_of(binding, empty_pool(b.n_pages, hkv, 16, d, "int8")) for _ in "ab"]
    args = b.tensors()
    pools[0].h1b_kv8_append(k, v, *args)
    pools[1].h1b_kv8_append(k.contiguous(), v.contiguous(), *args)
    for a, c in zip((pools[0].k_pages, pools[0].v_scale), (pools[1].k_pages, pools[1].v_scale)):
        assert torch.equal(a, c)
    want = pools[0].h1b_kv8_read(*args, n_rows=n, dtype=BF16)
    wide = torch.zeros(hkv, n, 2 * d, dtype=BF16, device="cuda")
    pools[0].h1b_kv8_read(*args, k=wide[:, :, :d].transpose(0, 1), v=wide[:, :, d:].transpose(0, 1))
    assert torch.equal(wide[:, :, :d].transpose(0, 1), want[0]) and torch.equal(wide[:, :, d:].transpose(0, 1), want[1])


# ------------------------------------------------------------------------------------------------ attention

CASES = [
    # rows, kv, hq, hkv, d, page, fmt, dtype, window, sinks
    ([1], [1], 1, 1, 128, 16, "int8", F16, 0, 0),
    ([1], [17], 4, 4, 64, 16, "e4m3", F16, 0, 0),
    ([1, 1, 1], [5, 300, 1025], 8, 2, 128, 32, "int8", BF16, 0, 0),
    ([1] * 5, [1, 15, 16, 31, 700], 6, 2, 64, 48, "int8", F16, 0, 0),
    ([1, 1], [2000, 3333], 16, 1, 128, 64, "e4m3", BF16, 0, 0),
    ([1, 1], [500, 90], 7, 1, 128, 64, "e4m3", F16, 0, 0),
    ([1, 1], [900, 40], 64, 2, 64, 64, "int8", F16, 0, 0),
    ([1, 1, 1], [900, 40, 260], 8, 2, 128, 16, "int8", F16, 128, 4),
    ([1, 1, 1], [900, 40, 260], 8, 2, 64, 32, "e4m3", BF16, 1, 0),
    ([1, 1, 1], [900, 40, 260], 4, 4, 128, 64, "int8", BF16, 33, 100),
    ([1, 1], [700, 300], 4, 2, 128, 64, "int8", F16, 5000, 17),
    ([2, 0, 5, 1], [2, 100, 400, 77], 8, 2, 128, 32, "int8", F16, 0, 0),
    ([16, 3], [16, 203], 4, 4, 128, 16, "e4m3", BF16, 0, 0),
    ([33, 130, 1, 7], [33, 500, 64, 1200], 8, 2, 128, 16, "int8", BF16, 0, 0),
    ([300], [300], 4, 4, 128, 64, "int8", F16, 0, 0),
    ([300], [300], 3, 1, 64, 32, "e4m3", BF16, 0, 0),
    ([257, 128], [900, 128], 4, 1, 128, 48, "e4m3", F16, 0, 0),
    ([260], [1000], 2, 2, 128, 64, "int8", BF16, 200, 5),
    ([200, 75], [1000, 75], 8, 2, 64, 16, "int8", F16, 64, 130),
    ([140], [2100], 12, 4, 128, 128, "e4m3", BF16, 700, 1),
    ([513], [513], 2, 1, 128, 256, "int8", F16, 1, 1),
    ([129], [4000], 5, 1, 128, 64, "int8", BF16, 0, 0),
    # enough work for both kernels in one call: single tokens and short rows beside chunks
    ([1, 2, 40, 150, 8], [6000, 3000, 5000, 4000, 9], 8, 2, 128, 64, "int8", F16, 0, 0),
    ([150, 1, 0, 3, 70], [4000, 7000, 0, 5000, 70], 6, 2, 64, 32, "e4m3", BF16, 0, 0),
    ([100, 1, 4], [7000, 7000, 3000], 16, 4, 128, 16, "e4m3", F16, 3000, 9),
]


def run_case(binding, case, seed=0, scale_spread=0.0, scale=None, max_rows=None, **kw):
    rows, kv, hq, hkv, d, page, fmt, dtype, window, sinks = case
    b = Batch(rows, kv, page, seed=seed, extra_rows=3)
    pool = filled_pool(b, hkv, d, fmt, seed, dtype, scale_spread)
    g = torch.Generator().manual_seed(seed + 100)
    q = torch.randn(b.n_rows, hq, d, generator=g).to(dtype)
    scale = 1 / math.sqrt(d) if scale is None else scale
    pages = pages_of(binding, pool)
    out = torch.full(q.shape, 9.0, dtype=dtype, device="cuda")
    got, lse = pages.h1b_kv8_attention(q.cuda(), *b.tensors(), scale=scale, window=window, sinks=sinks, out=out, return_lse=True,
                                       max_rows=max(rows) if max_rows is None else max_rows, **kw)
    pages.h1b_kv8_poll_status()
    n = int(b.row_start[-1])
    assert (got[n:] == 9.0).all()                          # rows behind the last sequence stay
    want = attention(q[:n], pool, b, fmt, scale, window, sinks)
    return got[:n], lse[:n], want


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d_q%dk%d_d%d_p%d_%s_%s_w%d_s%d" % (
    max(c[0]), max(c[1]), c[2], c[3], c[4], c[5], c[6], "bf" if c[7] == BF16 else "fp", c[8], c[9]))
def test_attention(binding, case):
    got, lse, want = run_case(binding, case)
    check_attention(got, lse, want)


@pytest.mark.parametrize("case", [CASES[2], CASES[8], CASES[13], CASES[16], CASES[19]], ids=str)
def test_attention_of_uneven_scales_and_sharp_scores(binding, case):
    """Keys and values whose sizes differ by thousands from token to token, and scores that leave one token nearly all."""
    got, lse, want = run_case(binding, case, seed=7, scale_spread=3.0)
    check_attention(got, lse, want)
    got, lse, want = run_case(binding, case, seed=8, scale=2.0)
    check_attention(got, lse, want)
    got, lse, want = run_case(binding, case, seed=9, scale=0.0)
    check_attention(got, lse, want)
    got, lse, want = run_case(binding, case, seed=9, scale=-0.125)
    check_attention(got, lse, want)


@pytest.mark.parametrize("case", [CASES[3], CASES[13], CASES[14], CASES[21]], ids=str)
@pytest.mark.parametrize("max_rows", [0, 1, 7, 100000])
def test_max_rows_only_chooses_kernels(binding, case, max_rows):
    got, lse, want = run_case(binding, case, max_rows=max_rows)
    check_attention(got, lse, want)


def test_random_batches(binding):
    rng = np.random.default_rng(11)
    for i in range(40):
        hkv = int(rng.choice([1, 2, 3, 4]))
        seqs = int(rng.integers(1, 6))
        rows = [int(rng.choice([0, 1, 1, 2, rng.integers(1, 20), rng.integers(1, 300)])) for _ in range(seqs)]
        kv = [int(r + rng.choice([0, 1, rng.integers(0, 40), rng.integers(0, 900)])) for r in rows]
        window = int(rng.choice([0, 0, 1, rng.integers(1, 100), rng.integers(1, 700)]))
        case = (rows, kv, hkv * int(rng.choice([1, 2, 3, 4, 8])), hkv, int(rng.choice([64, 128])),
                int(rng.choice([16, 32, 48, 64, 256])), str(rng.choice(["int8", "e4m3"])), [F16, BF16][int(rng.integers(2))],
                window, int(rng.choice([0, 1, 4, 16, 70])))
        got, lse, want = run_case(binding, case, seed=i)
        check_attention(got, lse, want, tag=str(case))


@pytest.mark.parametrize("seqs", [33, 70, 1100])
def test_many_sequences(binding, seqs):
    """More sequences than a warp has lanes, empty ones among them, single rows and chunks in one batch."""
    rng = np.random.default_rng(seqs)
    rows = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 5], seqs)]
    rows[-1] = 1
    if seqs < 100:
        rows[3], rows[-2] = 90, 300
    kv = [r + int(rng.integers(0, 60)) for r in rows]
    got, lse, want = run_case(binding, (rows, kv, 4, 2, 64, 16, "int8", BF16, 0, 0), seed=3)
    check_attention(got, lse, want)
    b = Batch(rows, kv, 16, seed=1)
    pages = pages_of(binding, empty_pool(b.n_pages, 2, 16, 64, "int8"))
    k, v = (torch.randn(b.n_rows, 2, 64).to(F16) for _ in "kv")
    args = b.tensors()
    pages.h1b_kv8_append(k.cuda(), v.cuda(), *args)
    for x, y in zip((k, v), pages.h1b_kv8_read(*args, n_rows=b.n_rows)):
        q, sc = quantised(x, "int8")
        assert torch.equal(y.cpu(), (q.float() * sc.float()[..., None]).to(F16))
    pages.h1b_kv8_poll_status()


def test_rows_that_see_nothing(binding):
    """kv_len smaller than the rows: the first rows lie before the sequence and get zeros; the status says so."""
    for hq, n in ((2, 3), (8, 200)):
        b = Batch([n, 1], [n, 1], 32)
        pool = filled_pool(b, 2, 128, "int8", 1)
        pages = pages_of(binding, pool)
        q = torch.randn(b.n_rows, hq, 128).to(F16)
        table, kv, row_start = b.tensors()
        kv[0] -= 2
        out, lse = pages.h1b_kv8_attention(q.cuda(), table, kv, row_start, scale=0.1, return_lse=True)
        with pytest.raises(binding.H1BError) as e:
            pages.h1b_kv8_poll_status()
        assert e.value.code == -1
        pages.h1b_kv8_poll_status()
        assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all()
        b2 = Batch([n - 2, 1], [n - 2, 1], 32)
        b2.table = b.table
        want = attention(q[2:], pool, b2, "int8", 0.1)
        check_attention(out[2:], lse[2:], want)
        # an empty sequence, rows all the same; and nothing at all
        kv.zero_()
        out, lse = pages.h1b_kv8_attention(q.cuda(), table, kv, row_start, scale=0.1, return_lse=True)
        assert (out == 0).all() and torch.isneginf(lse).all()
        none = pages.h1b_kv8_attention(q[:0].cuda(), table[:0], kv[:0], row_start[:1], scale=0.1)
        assert none.shape == (0, hq, 128)


@pytest.mark.parametrize("n", [1, 150])
def test_a_nan_row_reaches_the_rows_that_see_it(binding, n):
    b = Batch([n, 1], [n + 260, 300], 64, seed=2)
    pool = filled_pool(b, 2, 128, "int8", 1)
    t_bad = n + 258                                        # the last row but one of sequence 0 (its own row, n > 1)
    p, o = b.place(0, t_bad)
    for which in (2, 3):
        bad = [t.clone() for t in pool]
        bad[which][p, 1, o] = math.nan
        q = torch.randn(b.n_rows, 4, 128, generator=torch.Generator().manual_seed(3)).to(F16)
        pages = pages_of(binding, bad)
        for window, sinks in ((0, 0), (1, 0), (40, 2)):
            got, lse = pages.h1b_kv8_attention(q.cuda(), *b.tensors(), scale=0.1, window=window, sinks=sinks, return_lse=True)
            want = list(attention(q, bad, b, "int8", 0.1, window, sinks))
            nan_rows = torch.isnan(want[0]).any(-1)
            if which == 2:
                assert torch.equal(torch.isnan(got).all(-1).cpu(), torch.isnan(want[1]))
                keep = ~torch.isnan(want[1])
                assert keep.any()
                check_attention(got.cpu()[keep], lse.cpu()[keep], [w[keep] for w in want])
            else:
                assert torch.equal(torch.isnan(got).any(-1).cpu(), nan_rows)
                keep = ~nan_rows
                check_attention(got.cpu()[keep], lse.cpu()[keep], [w[keep] for w in want])


def test_pages_behind_the_window_are_not_read(binding):
    rows, kv, page = [1, 40], [3000, 2500], 64
    b = Batch(rows, kv, page, seed=4)
    pool = filled_pool(b, 2, 128, "e4m3", 5)
    q = torch.randn(b.n_rows, 8, 128).to(BF16)
    want = attention(q, pool, b, "e4m3", 0.09, 500, 20)
    for s in range(2):                                     # the pages between the sinks and the window are given away
        first = (kv[s] - rows[s] - 500 + 1) // page
        b.table[s, 1:first] = -1
    pages = pages_of(binding, pool)
    got, lse = pages.h1b_kv8_attention(q.cuda(), *b.tensors(), scale=0.09, window=500, sinks=20, return_lse=True)
    pages.h1b_kv8_poll_status()
    check_attention(got, lse, want)


@pytest.mark.parametrize("n", [1, 150])
def test_bad_pages_and_lengths_are_reported(binding, n):
    b = Batch([n], [n + 200], 32, seed=6)
    pool = filled_pool(b, 2, 64, "int8", 5)
    pages = pages_of(binding, pool)
    q = torch.randn(n, 4, 64).to(F16)
    table, kv, row_start = b.tensors()
    kv_rows = torch.randn(n, 2, 64).to(F16).cuda()
    before = [t.clone() for t in (pages.k_pages, pages.k_scale)]
    for bad in (-1, b.n_pages, 2 ** 31 - 1):
        t2 = table.clone()
        t2[0, 2] = bad                                     # tokens 64 .. 95 are nobody's
        out, lse = pages.h1b_kv8_attention(q.cuda(), t2, kv, row_start, scale=0.1, return_lse=True)
        with pytest.raises(binding.H1BError) as e:
            pages.h1b_kv8_poll_status()
        assert e.value.code == -8
        hidden = [t.clone() for t in pool]
        p = int(table[0, 2])
        hidden[2][p], hidden[3][p] = -math.inf, 0.0
        hidden[0][p] = 0
        # 64-bit statement without those tokens: drop them
        keep = [t for t in range(n + 200) if not 64 <= t < 96]
        k = numbers(pool[0][table.cpu()[0].long()].transpose(0, 1).reshape(2, -1, 64), "int8") * pool[2][table.cpu()[0].long()].transpose(0, 1).reshape(2, -1, 1).double()
        v = numbers(pool[1][table.cpu()[0].long()].transpose(0, 1).reshape(2, -1, 64), "int8") * pool[3][table.cpu()[0].long()].transpose(0, 1).reshape(2, -1, 1).double()
        z = torch.einsum("nhd,htd->nht", q.double(), k.repeat_interleave(2, 0)[:, keep]) * 0.1
        z = torch.where(torch.tensor(keep)[None, None] <= torch.arange(200, 200 + n)[:, None, None], z, -math.inf)
        w = torch.softmax(z, -1)
        vv = v.repeat_interleave(2, 0)[:, keep]
        want = (torch.einsum("nht,htd->nhd", w, vv), torch.logsumexp(z, -1), torch.einsum("nht,htd->nhd", w, vv.abs()),
                torch.einsum("nhd,htd->nht", q.double().abs(), k.repeat_interleave(2, 0)[:, keep].abs()).amax(-1) * 0.1,
                torch.full((n, 4), float(vv.shape[1] * vv.abs().amax())).double())
        check_attention(out, lse, want)
        pages.h1b_kv8_read(t2, kv + 0, row_start, n_rows=n)
        last = t2.clone()
        last[0, (n + 199) // 32] = bad
        got = pages.h1b_kv8_read(last, kv, row_start, n_rows=n)[0]
        assert (got[-1] == 0).all()
        pages.h1b_kv8_append(kv_rows[:n], kv_rows[:n], torch.full_like(table, bad), kv, row_start)
        with pytest.raises(binding.H1BError) as e:
            pages.h1b_kv8_poll_status()
        assert e.value.code == -8
        for x, y in zip(before, (pages.k_pages, pages.k_scale)):
            assert torch.equal(x.nan_to_num(nan=5), y.nan_to_num(nan=5))
    # more tokens than the table has room for
    over = kv + 10 ** 6
    pages.h1b_kv8_append(kv_rows, kv_rows, table, over, row_start)
    with pytest.raises(binding.H1BError) as e:
        pages.h1b_kv8_poll_status()
    assert e.value.code == -4
    pages.h1b_kv8_attention(q.cuda(), table, over, row_start, scale=0.1)
    with pytest.raises(binding.H1BError):
        pages.h1b_kv8_poll_status()
    # row_start that goes down or leaves the tensors
    for starts in ([5, 2], [-3, n], [0, n + 7], [2 ** 31 - 1, -2 ** 31]):
        rs = torch.tensor(starts, dtype=torch.int32, device="cuda")
        pages.h1b_kv8_attention(q.cuda(), table, kv, rs, scale=0.1)
        pages.h1b_kv8_read(table, kv, rs, n_rows=n)
        with pytest.raises(binding.H1BError) as e:
            pages.h1b_kv8_poll_status()
        assert e.value.code in (-1, -8)
    for x, y in zip(before, (pages.k_pages, pages.k_scale)):
        assert torch.equal(x.nan_to_num(nan=5), y.nan_to_num(nan=5))


def test_offsets_beyond_32_bits(binding):
    """A pool of more than 2^32 bytes and one of more than 2^31 scales' bytes: pages at its end."""
    page, hkv, d = 256, 8, 128
    n_pages = 2 ** 32 // (page * hkv * d) + 40
    b = Batch([3, 1], [300, 700], page, seed=1)
    small = filled_pool(b, hkv, d, "int8", 3)
    big = [torch.empty((n_pages,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda") for t in small]
    shift = n_pages - b.n_pages
    for x, y in zip(big, small):
        x[shift:] = y.cuda()
    q = torch.randn(b.n_rows, 16, d).to(F16)
    want = attention(q, small, b, "int8", 0.1)
    table, kv, row_start = b.tensors()
    table = torch.where(table >= 0, table + shift, table)
    pages = binding.KV8Pages(*big)
    got, lse = pages.h1b_kv8_attention(q.cuda(), table, kv, row_start, scale=0.1, return_lse=True)
    check_attention(got, lse, want)
    k, v = torch.randn(4, hkv, d).to(F16), torch.randn(4, hkv, d).to(F16)
    pages.h1b_kv8_append(k.cuda(), v.cuda(), table, kv, row_start)
    rk, rv = pages.h1b_kv8_read(table, kv, row_start, n_rows=4)
    for x, y in ((k, rk), (v, rv)):
        qn, sc = quantised(x, "int8")
        assert torch.equal(y.cpu(), (qn.float() * sc.float()[..., None]).to(F16))


# ------------------------------------------------------------------------------------------------ used together

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_prompt_in_chunks_and_steps(binding, fmt):
    """A prompt in two chunks, then single tokens, each appended before it is attended: every row equals the row of the whole
    sequence attended at once, and the 64-bit definition."""
    hq, hkv, d, page, total = 8, 2, 128, 32, 333
    b = Batch([total, total], [total, total], page, seed=9)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(2, total, hkv, d, generator=g).to(BF16) for _ in "kv")
    q = torch.randn(2, total, hq, d, generator=g).to(BF16)
    pool = empty_pool(b.n_pages, hkv, page, d, fmt)
    pages = pages_of(binding, pool)
    table = b.tensors()[0]
    outs, lses = [[], []], [[], []]
    done = 0
    for n in (200, 129, 1, 1, 2):
        kv = torch.tensor([done + n] * 2, dtype=torch.int32, device="cuda")
        rs = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        cut = [x[:, done:done + n].reshape(2 * n, -1, d).cuda() for x in (k, v, q)]
        pages.h1b_kv8_append(cut[0], cut[1], table, kv, rs)
        o, l = pages.h1b_kv8_attention(cut[2], table, kv, rs, scale=0.1, max_rows=n, return_lse=True)
        for s in range(2):
            outs[s].append(o[s * n:(s + 1) * n])
            lses[s].append(l[s * n:(s + 1) * n])
        done += n
    pages.h1b_kv8_poll_status()
    host = [t.cpu() for t in (pages.k_pages, pages.v_pages, pages.k_scale, pages.v_scale)]
    want = attention(q.reshape(2 * total, hq, d), host, b, fmt, 0.1)
    check_attention(torch.cat(outs[0] + outs[1]), torch.cat(lses[0] + lses[1]), want)


def test_aged_tokens_move_to_the_compressed_cache(binding):
    """The hybrid use: tokens that left the 8-bit window are read back and appended to the 1-bit / 4-bit cache, which is then
    the same as if it had been given the read-back numbers from the start."""
    hkv, d, page, aged = 2, 128, 32, 96
    b = Batch([aged], [aged], page, seed=3)
    pages = pages_of(binding, empty_pool(b.n_pages, hkv, page, d, "int8"))
    k, v = (torch.randn(aged, hkv, d).to(F16).cuda() for _ in "kv")
    args = b.tensors()
    pages.h1b_kv8_append(k, v, *args)
    rk, rv = pages.h1b_kv8_read(*args, n_rows=aged)
    assert (rk.float() - k.float()).abs().amax() <= k.float().abs().amax() * (0.5 / 127 + 2.0 ** -10)
    caches = []
    for kk, vv in ((rk, rv), (rk.clone(), rv.clone())):
        cfg = binding.make_config(1, 4, hkv, d, 128, 32, max_batch=1, max_seq=256)
        cache = binding.H1BCache(cfg, seed=1)
        cache.h1b_append_kv(kk.view(1, 1, aged, hkv, d), vv.view(1, 1, aged, hkv, d))
        caches.append(cache)
    q = torch.randn(1, 1, 4, d).to(F16).cuda()
    outs = [c.h1b_decode_attention(q, 16.0) for c in caches]
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0]).all() and outs[0].abs().sum() > 0
    for c in caches:
        c.close()


def test_a_captured_step_replays_on_other_lengths(binding):
    hq, hkv, d, page = 8, 2, 128, 16
    b = Batch([1, 1, 1], [700, 30, 333], page, seed=9, width=50)
    pool = filled_pool(b, hkv, d, "int8", 1)
    pages = pages_of(binding, pool)
    table, kv, row_start = b.tensors()
    q = torch.randn(3, hq, d).to(F16).cuda()
    k, v = (torch.randn(3, hkv, d).to(F16).cuda() for _ in "kv")
    def step():
        pages.h1b_kv8_append(k, v, table, kv, row_start)
        return pages.h1b_kv8_attention(q, table, kv, row_start, scale=0.1, max_rows=1, return_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    for lens in ([700, 30, 333], [16, 1, 320], [641, 24, 9]):
        kv.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(torch.randn(3, hq, d))
        k.copy_(torch.randn(3, hkv, d))
        graph.replay()
        torch.cuda.synchronize()
        pages.h1b_kv8_poll_status()
        b.kv = lens
        host = [t.cpu() for t in (pages.k_pages, pages.v_pages, pages.k_scale, pages.v_scale)]
        for s, t in enumerate(lens):
            p, o = b.place(s, t - 1)
            assert torch.equal(numbers(host[0][p, :, o], "int8"), quantised(k[s].cpu(), "int8")[0])
        check_attention(out, lse, attention(q.cpu(), host, b, "int8", 0.1))


def test_two_streams_at_once(binding):
    """Calls on two streams, each with tensors and workspaces of its own stream, do not disturb one another."""
    case = ([1] * 4, [3000, 2500, 100, 1700], 8, 2, 128, 64, "int8", F16, 0, 0)
    jobs = []
    for seed in (1, 2):
        b = Batch(case[0], case[1], 64, seed=seed)
        pool = filled_pool(b, 2, 128, "int8", seed)
        q = torch.randn(4, 8, 128, generator=torch.Generator().manual_seed(seed)).to(F16)
        jobs.append((pages_of(binding, pool), q.cuda(), b.tensors(), torch.cuda.Stream(), attention(q, pool, b, "int8", 0.1)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (pages, q, args, stream, _) in enumerate(jobs):
            got[i].append(pages.h1b_kv8_attention(q, *args, scale=0.1, max_rows=1, return_lse=True, stream=stream))
    torch.cuda.synchronize()
    for i, job in enumerate(jobs):
        for o, l in got[i]:
            assert torch.equal(o, got[i][0][0])            # the same every time, bit for bit
        check_attention(got[i][0][0], got[i][0][1], job[4])


def test_q_and_out_may_be_strided(binding):
    b = Batch([3, 140], [50, 140], 32, seed=2)
    hq, hkv, d = 8, 2, 128
    pool = filled_pool(b, hkv, d, "int8", 4)
    pages = pages_of(binding, pool)
    fused = torch.randn(b.n_rows, hq + 2 * hkv, d).to(BF16).cuda()
    q = fused[:, :hq]
    out = torch.zeros(hq, b.n_rows, d, dtype=BF16, device="cuda").transpose(0, 1)
    got = pages.h1b_kv8_attention(q, *b.tensors(), scale=0.1, out=out)
    assert got is out
    check_attention(out, None, attention(q.cpu(), pool, b, "int8", 0.1))


def test_queries_of_any_size(binding):
    """bf16 queries far outside fp16's range, zeros among them."""
    b = Batch([4], [100], 32, seed=2)
    pool = filled_pool(b, 2, 64, "int8", 4, BF16)
    pages = pages_of(binding, pool)
    for size in (2.0 ** 100, 2.0 ** -100, 1.0):
        q = (torch.randn(4, 4, 64) * size).to(BF16)
        q[1] = 0
        got, lse = pages.h1b_kv8_attention(q.cuda(), *b.tensors(), scale=0.1 / size, return_lse=True)
        check_attention(got, lse, attention(q, pool, b, "int8", 0.1 / size))


@pytest.mark.parametrize("n,kv", [(1, 5000), (2, 300), (140, 2000), (60, 700)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_powers_of_two_pass_through(binding, n, kv, fmt):
    """Values times a power of two are results times that power, to the bit, and keys against queries likewise: up to sums over
    the tokens that fp32 cannot hold (all values positive and alike: 2^125 and their sum 2^137), and down to 2^-100."""
    b, hq, hkv, d = Batch([n, n], [kv, kv - 7], 64, seed=2), 8, 2, 128
    k, v, ks, vs = filled_pool(b, hkv, d, fmt, 2, BF16)
    v = v.view(torch.uint8).bitwise_and(0x7F).clamp(max=0x7E).view(v.dtype)
    vs = torch.where(vs.isnan(), vs, torch.exp2(torch.floor(torch.log2(vs))))
    g = torch.Generator().manual_seed(4)
    q = torch.randn(b.n_rows, hq, d, generator=g).to(BF16)

    def run(q_pow, k_pow, v_pow, scale=0.02):
        pages = pages_of(binding, (k, v, ks * 2.0 ** k_pow, vs * 2.0 ** v_pow))
        out, lse = pages.h1b_kv8_attention((q.double() * 2.0 ** q_pow).to(BF16).cuda(), *b.tensors(), scale=scale, max_rows=n,
                                           return_lse=True)
        pages.h1b_kv8_poll_status()
        return out.double().cpu(), lse.cpu()

    top = 125 - int(torch.log2(vs[~vs.isnan()].max() * {"int8": 127, "e4m3": 448}[fmt]).floor())
    for scale in (0.02, 0.0):
        want, want_lse = run(0, 0, 0, scale)
        assert want.isfinite().all() and (want > 0).all()
        for powers in ((0, 0, top), (0, 0, -100), (-80, 80, 0), (20, -20, 3)):
            got, lse = run(*powers, scale)
            assert torch.equal(got, want * 2.0 ** powers[2]), powers
            assert torch.equal(lse, want_lse), powers


@pytest.mark.parametrize("n", [1, 33])
@pytest.mark.parametrize("what", ["row_start", "kv_len", "capacity"])
def test_sequences_without_rows_are_checked_too(binding, n, what):
    """Of many sequences, one that has no rows does not fit: each call says so, and computes the others."""
    seqs, hq, hkv, d = 120, 2, 1, 64
    rows = [n if s % 40 == 7 else 0 for s in range(seqs)]
    b = Batch(rows, [40] * seqs, 16, seed=1)
    table, kv_len, row_start = b.tensors()
    if what == "row_start":
        row_start[100] = 10 ** 6                           # (behind the last row: up and down again)
    elif what == "kv_len":
        kv_len[70] = -1
    else:
        kv_len[119] = 49
    pages = pages_of(binding, filled_pool(b, hkv, d, "int8", 1))
    x = torch.randn(b.n_rows, hkv, d, generator=torch.Generator().manual_seed(1)).half().cuda()
    q = torch.randn(b.n_rows, hq, d, generator=torch.Generator().manual_seed(2)).half().cuda()
    calls = [lambda: pages.h1b_kv8_append(x, x, table, kv_len, row_start),
             lambda: pages.h1b_kv8_read(table, kv_len, row_start, n_rows=b.n_rows),
             lambda: pages.h1b_kv8_attention(q, table, kv_len, row_start, scale=1.0, max_rows=n),
             lambda: pages.h1b_kv8_attention(q, table, kv_len, row_start, scale=1.0, max_rows=64)]
    for call in calls:
        call()
        with pytest.raises(binding.H1BError):
            pages.h1b_kv8_poll_status()
        pages.h1b_kv8_poll_status()                        # (once)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_many_rows_are_appended_and_read_like_few(binding, d, fmt):
    """A warp takes more heads where there are many rows: the same bits as row for row in small calls."""
    rows, hkv, page = [3000, 0, 2300], 21, 32
    b = Batch(rows, [3000, 9, 2404], page, seed=6)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(b.n_rows, hkv, d, generator=g).to(BF16).cuda() for _ in "kv")
    table, kv_len, row_start = b.tensors()
    one, many = (pages_of(binding, empty_pool(b.n_pages, hkv, page, d, fmt)) for _ in "ab")
    one.h1b_kv8_append(k, v, table, kv_len, row_start)
    wk, wv = one.h1b_kv8_read(table, kv_len, row_start, n_rows=b.n_rows, dtype=BF16)
    step, r = 100, 0
    for s in (0, 2):
        for at in range(0, rows[s], step):
            part = (table[s:s + 1], torch.tensor([b.kv[s] - rows[s] + at + step], dtype=torch.int32, device="cuda"),
                    torch.tensor([0, step], dtype=torch.int32, device="cuda"))
            many.h1b_kv8_append(k[r:r + step], v[r:r + step], *part)
            gk, gv = one.h1b_kv8_read(*part, n_rows=step, dtype=BF16)
            assert torch.equal(gk, wk[r:r + step]) and torch.equal(gv, wv[r:r + step])
            r += step
    for p in (one, many):
        p.h1b_kv8_poll_status()
    for a, c in zip((one.k_pages, one.v_pages, one.k_scale, one.v_scale), (many.k_pages, many.v_pages, many.k_scale, many.v_scale)):
        assert torch.equal(a.view(torch.uint8), c.view(torch.uint8))
    # half a step of the codes at amax, and the rounding to bf16
    assert (wk.double() - k.double()).abs().max() <= ({"int8": 0.5 / 127, "e4m3": 16 / 448}[fmt] + 2.0 ** -8) * k.double().abs().max()


@pytest.mark.parametrize("rows,kv", [([1], [700]), ([1] * 3, [40, 9000, 5000]), ([1], [20000]), ([150, 1, 40], [6000, 5000, 900]), ([300], [300])])
def test_the_result_may_take_the_place_of_q(binding, rows, kv):
    hq, hkv, d = 8, 2, 128
    b = Batch(rows, kv, 64, seed=4)
    pages = pages_of(binding, filled_pool(b, hkv, d, "int8", 4, BF16))
    q = torch.randn(b.n_rows, hq, d, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    want = pages.h1b_kv8_attention(q, *b.tensors(), scale=0.1, max_rows=max(rows))
    assert pages.h1b_kv8_attention(q, *b.tensors(), scale=0.1, max_rows=max(rows), out=q) is q
    pages.h1b_kv8_poll_status()
    assert torch.equal(q, want)
