"""Normed heads, caches of 8-bit elements and shared prefixes on the CPU: the
refusals, which answer before anything touches a GPU, and the references' own
invariants."""
import math

import pytest
import torch

from kv8_ref import element_values, normed, page_bytes, quantise, split_page, values_of
from paper_2608_22643_amd import binding as B

GOOD = dict(layers=32, heads=32, kv_heads=8, head_dim=128, page_size=64, n_pages=1000, max_seqs=64, seq_pages=128,
            dtype="f16")


def shape(**kw):
    return B.make_kv_shape(**dict(GOOD, **kw))


def refused(call, status=B.NP_ERR_INVALID_ARG):
    with pytest.raises(B.NPError) as e:
        call()
    assert e.value.status == status, e.value


def batch(**kw):
    a = dict(n_seq=2, n_tokens=2, max_tokens=1, max_len=100, seqs=None, cu_tokens=None, pos0=16)
    a.update(kw)
    return B.np_kv_batch(a["n_seq"], a["n_tokens"], a["max_tokens"], a["max_len"], a["seqs"], a["cu_tokens"], a["pos0"])


def rows(**kw):
    a = dict(q=16, k=16, v=16, q_out=32, q_stride=6144, k_stride=6144, v_stride=6144, q_out_stride=4096)
    a.update(kw)
    return B.np_kv_rows(*[a[n] for n in ("q", "k", "v", "q_out", "q_stride", "k_stride", "v_stride", "q_out_stride")])


EMPTY = dict(n_seq=0, n_tokens=0, pos0=None)


def test_shapes_of_8_bit_caches():
    for dim in (16, 64, 80, 128, 256):
        for dtype in ("f32", "f16", "bf16"):
            s = shape(head_dim=dim, dtype=dtype, cache="e4m3")
            B.np_kv_shape_check(s)
            assert B.kv_pool_shape(s) == (32, 1000, 2, 8, 64 * (dim + 1))
            assert B.np_kv_workspace_size(s) == B.np_kv_workspace_size(shape(head_dim=dim, dtype=dtype))
    assert B.kv_pool_shape(shape()) == (32, 1000, 2, 8, 64, 128)
    refused(lambda: B.np_kv_shape_check(shape(head_dim=8, cache="e4m3")))
    refused(lambda: B.np_kv_shape_check(shape(head_dim=120, cache="e4m3")))
    refused(lambda: B.np_kv_shape_check(shape(dtype=3 | B.NP_KV_E4M3)))
    refused(lambda: B.np_kv_shape_check(shape(dtype=1 | 0x200)))
    refused(lambda: B.np_kv_shape_check(shape(dtype=-1)))
    with pytest.raises(ValueError):
        shape(cache="e5m2")


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_append_norm_refusals(cache):
    s = shape(cache=cache)

    def append(norm=B.np_qk_norm(16, 16, 1e-6), rot=None, table=16, pool=16, ws=16, layer=0, b=None, **kw):
        B.np_kv_append_norm(s, layer, batch() if b is None else b, table, rows(**kw), norm, rot, pool, ws)

    for kw in (dict(norm=B.np_qk_norm(24, 16, 1e-6)), dict(norm=B.np_qk_norm(16, 2, 1e-6)),
               dict(norm=B.np_qk_norm(16, 16, -1e-6)), dict(norm=B.np_qk_norm(16, 16, math.nan)),
               dict(norm=B.np_qk_norm(16, 16, math.inf)),
               dict(q=None), dict(k=24), dict(v=0), dict(q_out=None), dict(q_stride=4000), dict(k_stride=1020),
               dict(q_out=16), dict(table=4), dict(pool=None), dict(ws=None), dict(layer=32),
               dict(b=batch(n_tokens=7)), dict(rot=B.np_rotary(16, 16, 8, 10, 0)),
               dict(rot=B.np_rotary(None, 16, 128, 10, 0))):
        refused(lambda: append(**kw))
    append(b=batch(**EMPTY), q=None, k=None, v=None, q_out=None)  # no tokens: nothing enqueued
    append(norm=None, b=batch(**EMPTY))
    append(norm=B.np_qk_norm(None, None, 0.0), b=batch(**EMPTY))
    with pytest.raises(ValueError):
        B.make_qk_norm(torch.ones(2, 8))
    with pytest.raises(ValueError):
        B.make_qk_norm(None, torch.ones(16)[::2])


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_read_refusals(cache):
    s = shape(cache=cache)

    def read(k=16, ks=1024, v=32, vs=1024, table=16, pool=16, ws=16, layer=0, b=None):
        st = B.lib().np_kv_read(B.ctypes.byref(s), layer, B.ctypes.byref(batch() if b is None else b), table, pool, k,
                                ks, v, vs, ws, None)
        if st != B.NP_OK:
            raise B.NPError(st, "np_kv_read", B.lib().np_last_error().decode())

    for kw in (dict(k=24), dict(v=8), dict(ks=1020), dict(vs=1000), dict(v=16), dict(table=None), dict(pool=8),
               dict(ws=None), dict(layer=-1), dict(b=batch(pos0=None)), dict(b=batch(n_tokens=5))):
        refused(lambda: read(**kw))
    read(k=None, ks=0, v=None, vs=0)  # nothing asked for
    read(b=batch(**EMPTY))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_shared_refusals(cache):
    s = shape(cache=cache)

    def attn(shared=B.np_kv_shared(100, 16, 16), layer=0, b=None, table=16, q=16, qs=4096, pool=16, scale=0.1, window=0,
             out=32, os_=4096, ws=16):
        st = B.lib().np_attn_decode_shared(B.ctypes.byref(s), layer, B.ctypes.byref(batch() if b is None else b),
                                           None if shared is None else B.ctypes.byref(shared), table, q, qs, pool,
                                           scale, window, out, os_, ws, None)
        if st != B.NP_OK:
            raise B.NPError(st, "np_attn_decode_shared", B.lib().np_last_error().decode())

    for kw in (dict(shared=None), dict(shared=B.np_kv_shared(-1, 16, 16)), dict(shared=B.np_kv_shared(9, None, 16)),
               dict(shared=B.np_kv_shared(9, 16, None)), dict(shared=B.np_kv_shared(9, 18, 16)),
               dict(shared=B.np_kv_shared(9, 16, 18)), dict(b=batch(cu_tokens=16)), dict(layer=32), dict(table=None),
               dict(q=24), dict(qs=4100), dict(pool=None), dict(scale=math.nan), dict(window=-1), dict(out=None),
               dict(ws=24), dict(out=16, os_=4104), dict(b=batch(n_seq=65, n_tokens=65)), dict(b=batch(pos0=18))):
        refused(lambda: attn(**kw))
    attn(b=batch(**EMPTY), shared=B.np_kv_shared(0, None, None))
    with pytest.raises(ValueError):
        B.make_kv_shared(torch.zeros(4, dtype=torch.int32)[::2], torch.zeros(2, dtype=torch.int32), 5)


def test_elements_reference():
    """The table against torch's type, the search against torch's conversion, the
    scale's definition, and the error that the format promises."""
    v = element_values()
    assert torch.equal(v, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
    g = torch.Generator().manual_seed(0)
    x = torch.randn(400, 32, generator=g, dtype=torch.float64) * torch.exp2(
        torch.randint(-30, 15, (400, 1), generator=g).double())
    x[0], x[1, 3], x[2] = 0.0, -0.0, 448.0
    x[3] = torch.linspace(0, 460, 32, dtype=torch.float64)
    x = x.half().double()
    byte, scale, value = quantise(x, "f16")
    e = scale.double() - 127
    m = x.abs().amax(-1)
    assert (m <= 448 * torch.exp2(e)).all() and ((m > 448 * torch.exp2(e - 1)) | (scale == 1)).all()
    y = (x / torch.exp2(e)[:, None]).float()
    sat = e >= 8
    assert torch.equal(byte[~sat], y[~sat].to(torch.float8_e4m3fn).view(torch.uint8))
    off = (value - x).abs()
    top = m[:, None] > 65504 * (1 - 2.0 ** -4)
    assert ((off <= 2.0 ** -4 * x.abs()) | (off <= torch.exp2(e - 10)[:, None]) | (top & (off <= 65504 / 16))).all()
    assert torch.equal(value, value.half().double()), "the type holds every value exactly"
    assert torch.equal(values_of(byte, scale), value)
    b, s = split_page(page_bytes(byte[None], scale[None]), 400, 32)
    assert torch.equal(b[0], byte) and torch.equal(s[0], scale)


def test_elements_at_the_ends_of_the_types():
    top = torch.tensor([[65504.0, -65504.0, 60000.0, 1.0]], dtype=torch.float64)
    byte, scale, value = quantise(top, "f16")
    assert int(scale) == 135 and value.abs().max() == 240 * 256 and torch.isfinite(value.half()).all()
    big = torch.finfo(torch.bfloat16).max
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        _, scale, value = quantise(torch.tensor([[big, -big, 1e30, 0.0]], dtype=torch.float64), dtype)
        assert int(scale) == 247 and torch.isfinite(value.to(dt)).all()
    _, scale, value = quantise(torch.tensor([[2.0 ** -149, 0.0, -2.0 ** -133]], dtype=torch.float64), "f32")
    assert int(scale) == 1
    byte, scale, value = quantise(torch.tensor([[math.inf, math.nan, -3.0, 0.5]], dtype=torch.float64), "f32")
    assert byte[0, 0] == byte[0, 1] == 127 and value[0, 2] == -3 and value[0, 3] == 0.5


def test_norm_reference():
    x = torch.tensor([[[3.0, 4.0, 0.0, 0.0]]])
    assert torch.allclose(normed(x, None, 0.0), x.double() / 2.5)
    assert torch.equal(normed(torch.zeros(1, 1, 8), None, 0.0), torch.zeros(1, 1, 8, dtype=torch.float64))
    w = torch.tensor([1.0, 2.0, 3.0, 4.0])
    assert torch.allclose(normed(x, w, 0.75), x.double() * w / math.sqrt(7.0))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_tensors_of_other_sizes_are_refused(cache):
    """The binding knows what the pointers cannot tell: nothing is read or written past a tensor."""
    s, b = shape(cache=cache), batch()
    half, D, n = torch.float16, s.head_dim, b.n_tokens
    norms = [B.make_qk_norm(torch.ones(D // 2, dtype=half)), B.make_qk_norm(None, torch.ones(2 * D, dtype=half)),
             B.make_qk_norm(torch.ones(D))]
    outs = [torch.zeros(n - 1, s.kv_heads, D, dtype=half), torch.zeros(n, s.kv_heads + 1, D, dtype=half),
            torch.zeros(n, s.kv_heads, D // 2, dtype=half), torch.zeros(n, s.kv_heads, D)]
    for norm in norms:
        with pytest.raises(ValueError):
            B.np_kv_append_norm(s, 0, b, 16, rows(), norm, None, 16, 16)
    for x in outs:
        for k, v in ((x, None), (None, x)):
            with pytest.raises(ValueError):
                B.np_kv_read(s, 0, b, 16, 16, k, v, 16)
    i32 = torch.zeros(b.n_seq + 1, dtype=torch.int32)
    q = torch.zeros(b.n_seq, s.heads, D, dtype=half)
    with pytest.raises(ValueError):
        B.np_attn_decode_shared(s, 0, b, B.make_kv_shared(i32, i32, 5), 16, q, 16, 1.0, 0, q, 16)
    for x in (i32.long(), i32.float(), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            B.make_kv_shared(x, i32, 5)
        with pytest.raises(ValueError):
            B.make_kv_shared(i32, x, 5)
