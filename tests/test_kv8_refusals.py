"""What the 8-bit pages refuse (host-side checks only: every call here is turned down before anything is launched), and
the quantiser's definition against itself. No GPU."""
import ctypes
import math

import pytest
import torch

import kv8_testlib as lib
from paper_2510_05529_b200 import binding

P = 1 << 20                                                # an aligned address that nothing reads


@pytest.fixture(scope="module")
def so():
    return binding.load_library()


def pool(**kw):
    f = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=4, n_kv_heads=2, page_tokens=32, head_dim=128, format=0, device=0)
    f.update(kw)
    return binding.h1b_kv8_pool(**f)


def batch(**kw):
    f = dict(block_table=P, kv_len=P, row_start=P, status=None, n_seqs=2, table_width=3, n_rows=5)
    f.update(kw)
    return binding.h1b_kv8_batch(**f)


def rows(**kw):
    f = dict(data=P, row_stride=512, head_stride=128)
    f.update(kw)
    return binding.h1b_kv8_rows(**f)


def attention(so, p=None, b=None, q=None, out=None, hq=4, dtype=0, scale=0.1, window=0, sinks=0, max_rows=1, ws=P, size=1 << 40):
    r = ctypes.byref
    return so.h1b_kv8_attention(r(p or pool()), r(b or batch()), r(q or rows()), r(out or rows()), None, hq, dtype, scale, window,
                                sinks, max_rows, ws, size, None)


BAD_POOLS = [
    (dict(head_dim=96), -3), (dict(head_dim=0), -3), (dict(format=2), -1), (dict(format=-1), -1), (dict(n_pages=0), -1),
    (dict(n_kv_heads=0), -1), (dict(page_tokens=0), -1), (dict(page_tokens=24), -1), (dict(page_tokens=-16), -1), (dict(device=-1), -1),
    (dict(k=None), -2), (dict(v=None), -2), (dict(k_scale=None), -2), (dict(v_scale=None), -2), (dict(k=P + 8), -1), (dict(v_scale=P + 4), -1),
]
BAD_BATCHES = [
    (dict(n_seqs=-1), -1), (dict(n_seqs=2 ** 20 + 1), -1), (dict(n_rows=-1), -1), (dict(table_width=0), -1), (dict(table_width=1 << 26), -1), (dict(block_table=None), -2),
    (dict(kv_len=None), -2), (dict(row_start=None), -2),
]
BAD_IN = [(dict(data=None), -2), (dict(data=P + 2), -1), (dict(row_stride=12), -1), (dict(head_stride=4), -1)]
BAD_OUT = BAD_IN + [(dict(row_stride=128), -1), (dict(head_stride=64), -1), (dict(row_stride=0), -1), (dict(head_stride=0), -1)]


def calls(so, p, b, x):
    r = ctypes.byref
    yield so.h1b_kv8_append(r(p), r(b), r(x), r(rows()), 0, None)
    yield so.h1b_kv8_append(r(p), r(b), r(rows()), r(x), 0, None)


@pytest.mark.parametrize("change,code", BAD_POOLS)
def test_bad_pools(so, change, code):
    p, r = pool(**change), ctypes.byref
    assert all(rc == code for rc in calls(so, p, batch(), rows()))
    assert so.h1b_kv8_read(r(p), r(batch()), r(rows()), r(rows()), 0, None) == code
    assert attention(so, p=p) == code
    assert so.h1b_last_error(None)
    assert so.h1b_kv8_attention_bytes(r(p), r(batch()), 4, 0, 0, 1) == 0


@pytest.mark.parametrize("change,code", BAD_BATCHES)
def test_bad_batches(so, change, code):
    b, r = batch(**change), ctypes.byref
    assert all(rc == code for rc in calls(so, pool(), b, rows()))
    assert so.h1b_kv8_read(r(pool()), r(b), r(rows()), r(rows()), 0, None) == code
    assert attention(so, b=b) == code


@pytest.mark.parametrize("change,code", BAD_IN)
def test_bad_inputs(so, change, code):
    assert all(rc == code for rc in calls(so, pool(), batch(), rows(**change)))
    assert attention(so, q=rows(**change)) == code


@pytest.mark.parametrize("change,code", BAD_OUT)
def test_bad_outputs(so, change, code):
    r = ctypes.byref
    assert attention(so, out=rows(**change)) == code
    if code != -2:                                         # (read takes NULL for what is not wanted)
        assert so.h1b_kv8_read(r(pool()), r(batch()), r(rows(**change)), r(rows()), 0, None) == code
        assert so.h1b_kv8_read(r(pool()), r(batch()), r(rows()), r(rows(**change)), 0, None) == code


def test_bad_numbers(so):
    r = ctypes.byref
    for kw in (dict(hq=0), dict(hq=3), dict(hq=2 * 129), dict(hq=-2), dict(dtype=2), dict(dtype=-1), dict(scale=math.nan), dict(scale=math.inf),
               dict(window=-1), dict(sinks=-1), dict(max_rows=-1), dict(window=2 ** 31 - 1)):
        assert attention(so, **kw) == -1, kw
    assert so.h1b_kv8_append(None, r(batch()), r(rows()), r(rows()), 0, None) == -2
    assert so.h1b_kv8_append(r(pool()), None, r(rows()), r(rows()), 0, None) == -2
    assert so.h1b_kv8_append(r(pool()), r(batch()), None, r(rows()), 0, None) == -2
    assert so.h1b_kv8_append(r(pool()), r(batch()), r(rows()), r(rows()), 7, None) == -1
    assert so.h1b_kv8_attention(r(pool()), r(batch()), None, r(rows()), None, 4, 0, 0.1, 0, 0, 1, P, 1 << 40, None) == -2
    big = batch(n_rows=2 ** 29)
    assert attention(so, b=big) == -1
    assert so.h1b_kv8_append(r(pool()), r(batch(n_rows=2 ** 30)), r(rows(row_stride=0)), r(rows(row_stride=0)), 0, None) == -1
    assert so.h1b_kv8_append(r(pool(n_pages=2 ** 31 - 1)), r(batch()), r(rows()), r(rows()), 0, None) == -3


def test_workspace_is_checked(so):
    b = batch(table_width=1024)
    need = so.h1b_kv8_attention_bytes(ctypes.byref(pool()), ctypes.byref(b), 4, 0, 0, 1)
    assert need > 0
    assert attention(so, b=b, ws=None, size=need) == -5
    assert attention(so, b=b, size=need - 1) == -5
    assert attention(so, b=b, ws=P + 4, size=need) == -5
    assert b"workspace" in so.h1b_last_error(None)


def test_nothing_to_do_is_no_error(so):
    r = ctypes.byref
    for b in (batch(n_rows=0), batch(n_seqs=0)):
        none = rows(data=None) if b.n_rows == 0 else rows()
        assert so.h1b_kv8_append(r(pool()), r(b), r(none), r(none), 0, None) == 0
        assert so.h1b_kv8_read(r(pool()), r(b), r(none), r(none), 0, None) == 0
        assert attention(so, b=b, q=none, out=none) == 0
        assert so.h1b_kv8_attention_bytes(r(pool()), r(b), 4, 0, 0, 1) == 0
    assert so.h1b_kv8_read(r(pool()), r(batch()), None, None, 0, None) == 0


def test_the_python_binding_refuses():
    cpu = torch.zeros(2, 2, 16, 64, dtype=torch.int8)
    s = torch.zeros(2, 2, 16)
    with pytest.raises(TypeError):
        binding.KV8Pages(cpu, cpu, s, s)
    with pytest.raises(ValueError):
        binding._int32("window", 2 ** 31)
    rows3 = torch.zeros(3, 2, 64)
    with pytest.raises(TypeError):
        binding._kv8_rows(rows3, "q", 2, 64, torch.float16, -1)
    with pytest.raises(TypeError):
        binding._kv8_rows(rows3, "q", 2, 64, torch.float32, 0)
    with pytest.raises(ValueError):
        binding._kv8_rows(rows3.transpose(1, 2), "q", 64, 2, torch.float32, -1)
    with pytest.raises(ValueError):
        binding._kv8_rows(rows3, "q", 4, 64, torch.float32, -1)


def test_the_structures_packed_by_hand_are_the_header_s():
    """The binding packs h1b_kv8_rows and h1b_kv8_batch itself (it is faster): the same bytes as ctypes would lay out."""
    t = torch.zeros(5, 4, 64)[:, ::2]
    assert binding._kv8_rows(t, "q", 2, 64, torch.float32, -1) == bytes(binding.h1b_kv8_rows(t.data_ptr(), 256, 128))
    packed = binding._BATCH(1, 2, 3, 4, 5, 6, 7)
    assert packed == bytes(binding.h1b_kv8_batch(1, 2, 3, 4, 5, 6, 7)) and len(packed) == ctypes.sizeof(binding.h1b_kv8_batch)
    assert binding._ROWS(1, -2, 3) == bytes(binding.h1b_kv8_rows(1, -2, 3))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_quantiser_is_defined_to_the_bit(fmt, dtype):
    """The fp32 quotient of TOP * x and amax rounds to the same code as the exact one, ties included: what lets the kernels'
    codes be compared for equality."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4000, 64, generator=g).to(dtype)
    x[:, 0] = x[:, 0].abs() + 4
    x[:, 1] = (x[:, 0].double() / 2).to(dtype)                              # ties of int8
    x[::2] = torch.round(x[::2].float() * 8).to(dtype)                      # few-bit numbers: many ties of e4m3
    x[:, 0] = x.float().abs().amax(-1).clamp(min=1).to(dtype)
    amax = x.float().abs().amax(-1, keepdim=True)
    q = (x.float() * lib.TOP[fmt]) / amax
    got = q.round().double() if fmt == "int8" else q.to(torch.float8_e4m3fn).double()
    want, _ = lib.quantised(x, fmt)
    assert torch.equal(got, want)
    # off by at most half a step: 1/254 of the largest for int8, 2^-4 of the value (2^-10 * amax / 448 below 2^-6) for e4m3
    err = (want - x.double() * lib.TOP[fmt] / amax.double()).abs()
    bound = torch.full_like(err, 0.5) if fmt == "int8" else torch.maximum(want.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10).double())
    assert (err <= bound * (1 + 1e-12)).all()
