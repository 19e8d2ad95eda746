"""The cache and attention calls on the CPU: exports, argument checks that
answer before anything touches a GPU, and the references' own invariants."""
import ctypes
import os
import random
import re

import pytest
import torch

from kv_ref import PageModel, attention, rotate
from paper_2608_22643_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "neuroprefetch_kv.h")

GOOD = dict(layers=32, heads=32, kv_heads=8, head_dim=128, page_size=64, n_pages=1000, max_seqs=64, seq_pages=128,
            dtype="f16")


def shape(**kw):
    return B.make_kv_shape(**dict(GOOD, **kw))


def test_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(np_[a-z_]+)\s*\(", text))
    assert names == set(B.KV_EXPORTS)
    for n in names:
        assert hasattr(B.lib(), n), n


@pytest.mark.parametrize("change", [
    dict(layers=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=5), dict(heads=2048, kv_heads=8), dict(head_dim=0),
    dict(head_dim=4), dict(head_dim=132), dict(head_dim=264), dict(page_size=8), dict(page_size=48),
    dict(page_size=512), dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(max_seqs=0), dict(max_seqs=4097),
    dict(seq_pages=0), dict(seq_pages=1 << 25), dict(dtype=3)])
def test_shape_refusals(change):
    s = shape(**change)
    assert B.lib().np_kv_shape_check(ctypes.byref(s)) == B.NP_ERR_INVALID_ARG
    with pytest.raises(B.NPError):
        B.np_kv_workspace_size(s)


def test_good_shapes():
    for change in (dict(), dict(head_dim=8), dict(head_dim=256, dtype="f32"), dict(kv_heads=32), dict(kv_heads=1),
                   dict(page_size=16), dict(page_size=256), dict(max_seqs=4096), dict(n_pages=1 << 20)):
        B.np_kv_shape_check(shape(**change))
    assert B.np_kv_workspace_size(shape()) % 256 == 0


def refused(call, status=B.NP_ERR_INVALID_ARG):
    with pytest.raises(B.NPError) as e:
        call()
    assert e.value.status == status, e.value


def test_call_refusals():
    s = shape()
    st = B.np_kv_state(16, 16, 16)

    def batch(**kw):
        a = dict(n_seq=2, n_tokens=2, max_tokens=1, max_len=100, seqs=None, cu_tokens=None, pos0=16)
        a.update(kw)
        return B.np_kv_batch(a["n_seq"], a["n_tokens"], a["max_tokens"], a["max_len"], a["seqs"], a["cu_tokens"],
                             a["pos0"])

    def rows(**kw):
        a = dict(q=16, k=16, v=16, q_out=32, q_stride=6144, k_stride=6144, v_stride=6144, q_out_stride=4096)
        a.update(kw)
        return B.np_kv_rows(*[a[n] for n in ("q", "k", "v", "q_out", "q_stride", "k_stride", "v_stride",
                                             "q_out_stride")])

    def attn(fn, layer=0, b=None, table=16, q=16, qs=4096, pool=16, scale=0.1, window=0, out=32, os_=4096, ws=16):
        b = batch() if b is None else b
        st_ = getattr(B.lib(), fn)(ctypes.byref(s), layer, ctypes.byref(b), table, q, qs, pool, scale, window, out, os_,
                                   ws, None)
        if st_ != B.NP_OK:
            raise B.NPError(st_, fn, B.lib().np_last_error().decode())

    for fn in ("np_attn_decode", "np_attn_prompt"):
        for kw in (dict(layer=-1), dict(layer=32), dict(table=None), dict(table=8), dict(q=None), dict(q=24),
                   dict(qs=4088), dict(qs=4100), dict(os_=100), dict(pool=None), dict(scale=float("nan")),
                   dict(scale=float("inf")), dict(window=-1), dict(out=None), dict(ws=24),
                   dict(out=16, os_=4104),
                   dict(b=batch(n_seq=-1)), dict(b=batch(n_seq=65, n_tokens=65)), dict(b=batch(n_tokens=3)),
                   dict(b=batch(n_tokens=-1, cu_tokens=16)), dict(b=batch(pos0=None)), dict(b=batch(pos0=18)),
                   dict(b=batch(seqs=18)), dict(b=batch(max_len=-1))):
            refused(lambda: attn(fn, **kw))
        attn(fn, b=batch(n_seq=0, n_tokens=0, pos0=None))  # nothing to do, nothing enqueued
    refused(lambda: attn("np_attn_decode", b=batch(cu_tokens=16)))
    refused(lambda: attn("np_attn_prompt", b=batch(cu_tokens=16, n_tokens=1 << 28)))
    refused(lambda: attn("np_attn_prompt", b=batch(cu_tokens=18)))

    def append(rot=None, table=16, pool=16, ws=16, layer=0, b=None, **kw):
        B.np_kv_append(s, layer, batch() if b is None else b, table, rows(**kw), rot, pool, ws)

    for kw in (dict(q=None), dict(k=24), dict(v=0), dict(q_out=None), dict(q_stride=4000), dict(k_stride=1020),
               dict(v_stride=1028), dict(q_out_stride=8), dict(q_out=16), dict(table=4), dict(pool=None),
               dict(ws=None), dict(layer=32), dict(b=batch(n_tokens=7)),
               dict(rot=B.np_rotary(16, 16, 8, 10, 0)), dict(rot=B.np_rotary(16, 16, 144, 10, 0)),
               dict(rot=B.np_rotary(16, 16, 24, 10, 0)), dict(rot=B.np_rotary(16, 16, 128, 0, 0)),
               dict(rot=B.np_rotary(None, 16, 128, 10, 0)), dict(rot=B.np_rotary(16, 20, 128, 10, 0))):
        refused(lambda: append(**kw))

    bad_state = B.np_kv_state(16, None, 16)
    for call in (lambda: B.np_kv_reset(s, bad_state, 16), lambda: B.np_kv_reset(s, st, None),
                 lambda: B.np_kv_extend(s, bad_state, 16, 1, None, None, 16, 16),
                 lambda: B.np_kv_extend(s, st, None, 1, None, None, 16, 16),
                 lambda: B.np_kv_extend(s, st, 16, 65, None, None, 16, 16),
                 lambda: B.np_kv_extend(s, st, 16, -1, None, None, 16, 16),
                 lambda: B.np_kv_extend(s, st, 16, 1, None, None, None, 16),
                 lambda: B.np_kv_extend(s, st, 16, 1, 18, None, 16, 16),
                 lambda: B.np_kv_fork(s, st, 1, None, 16, None, 16),
                 lambda: B.np_kv_fork(s, st, 1, 16, 18, None, 16),
                 lambda: B.np_kv_fork(s, st, 65, 16, 16, None, 16),
                 lambda: B.np_kv_free(s, st, -1, 16, 16), lambda: B.np_kv_free(s, st, 1, 18, 16),
                 lambda: B.np_kv_compact(s, st, None, None, 16), lambda: B.np_kv_compact(s, st, 16, 18, 16)):
        refused(call)
    B.np_kv_extend(s, st, 16, 0, None, None, None, 16)
    B.np_kv_fork(s, st, 0, None, None, None, 16)
    B.np_kv_free(s, st, 0, None, 16)


def test_token_strides():
    x = torch.zeros(5, 6, 8)
    assert B._token_stride(x[:, 2:4]) == 48
    assert B._token_stride(x[:1, 2:4]) == 48
    with pytest.raises(ValueError):
        B._token_stride(x.transpose(0, 1))
    with pytest.raises(ValueError):
        B._token_stride(x[:, ::2])


def test_page_model_keeps_its_invariants():
    """Reference counts are the holders, free pages are held by nobody, and
    every sequence reads back what was written to it, through forks, copies
    and compactions."""
    rng = random.Random(5)
    S, N, M, P = 8, 40, 10, 4
    m = PageModel(S, N, M, P)
    text = [[] for _ in range(S)]
    token = 0
    for _ in range(600):
        op = rng.random()
        if op < 0.55:
            seqs = rng.sample(range(S), rng.randint(1, S))
            new = [rng.randint(0, 6) for _ in seqs]
            for s, n, p0 in zip(seqs, new, m.extend(seqs, new)):
                for i in range(n if p0 >= 0 else 0):
                    m.data[m.table[s][(p0 + i) // P]][(p0 + i) % P] = token
                    text[s].append(token)
                    token += 1
        elif op < 0.75:
            a, b = rng.randrange(S), rng.randrange(S)
            n = rng.randint(0, len(text[a]))
            if not text[b]:
                m.fork([a], [b], [n])
                if a != b:
                    text[b] = text[a][:n]
        elif op < 0.92:
            s = rng.randrange(S)
            m.free([s])
            text[s] = []
        else:
            m.compact()
            used = [p for p in range(N) if m.refs[p]]
            assert used == list(range(len(used)))
        held = [p for t in m.table for p in t]
        assert m.refs == [held.count(p) for p in range(N)]
        for s in range(S):
            assert m.len[s] == len(text[s]) and len(m.table[s]) == -(-m.len[s] // P)
            assert [m.data[m.table[s][i // P]][i % P] for i in range(m.len[s])] == text[s]


def test_attention_reference():
    """One key: the value itself.  Equal keys: the mean.  A window of one: the
    token's own value.  The order of the keys does not matter."""
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(*s, generator=g) for s in ((3, 4, 8), (2, 5, 8), (2, 5, 8)))
    out, tol = attention(q, k, v, 2, 0.3, 1, "f32")
    for i in range(3):
        for h in range(4):
            assert torch.allclose(out[i, h], v[h // 2, 2 + i].double())
    same = k[:, :1].expand(2, 5, 8)
    out, _ = attention(q, same, v, 2, 0.3, 0, "f32")
    assert torch.allclose(out[2, 3], v[1].double().mean(0))
    perm = torch.tensor([3, 0, 4, 1, 2])
    a, _ = attention(q[2:], k, v, 4, 0.3, 0, "f32")
    b, _ = attention(q[2:], k[:, perm], v[:, perm], 4, 0.3, 0, "f32")
    assert torch.allclose(a, b)
    zero, _ = attention(q, k, v, -1, 0.3, 0, "f32")
    assert (zero == 0).all() and (tol > 0).all()


def test_rotation_reference():
    """Lengths stay, position 0 stays, and q.k depends on the distance only."""
    g = torch.Generator().manual_seed(0)
    ang = torch.arange(50, dtype=torch.float64)[:, None] * torch.tensor([0.5, 0.1, 0.02, 0.003], dtype=torch.float64)
    cos, sin = ang.cos(), ang.sin()
    q, k = torch.randn(1, 1, 10, generator=g), torch.randn(1, 1, 10, generator=g)
    for inter in (False, True):
        at = lambda x, p: rotate(x, cos, sin, torch.tensor([p]), inter)
        assert torch.allclose(at(q, 0), q.double())
        assert torch.allclose(at(q, 33).norm(), q.double().norm())
        d = [float((at(q, p + 7) * at(k, p)).sum()) for p in (0, 11, 40)]
        assert max(d) - min(d) < 1e-9
