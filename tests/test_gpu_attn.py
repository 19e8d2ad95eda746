"""np_attn_decode and np_attn_prompt against float64 attention, elementwise
within a bound derived from the kernels' arithmetic (kv_ref.attention): types,
head layouts, page sizes, ragged rows, windows, rows that see nothing, strides,
in-place outputs, poisoned memory, tables that name no page, HIP graphs."""
import math

import pytest
import torch

from kv_ref import DT, attention, div_up
from paper_2608_22643_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Setup:
    """A cache of one layer holding random keys and values for rows
    (p0, n): every slot that no token may see is NaN."""

    def __init__(self, rows, Hq, Hkv, D, P, dtype, seed=0, extra_pages=3, layers=1, layer=0, pages=None):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.rows, self.Hq, self.Hkv, self.D, self.P, self.dtype = rows, Hq, Hkv, D, P, dtype
        self.layer = layer
        lens = [max(p0 + n, 0) if p0 >= 0 else 0 for p0, n in rows]
        need = [div_up(x, P) for x in lens]
        self.N = pages or sum(need) + extra_pages
        self.M = max(max(need), 1) + 1
        order = torch.randperm(self.N, generator=g).tolist()
        self.S = len(rows)
        table = torch.full((self.S, self.M), -1, dtype=torch.int32)
        self.keys, self.values = [], []
        pool = torch.full((layers, self.N, 2, Hkv, P, D), float("nan"), dtype=dt)
        at = 0
        for b, ln in enumerate(lens):
            k = torch.randn(Hkv, ln, D, generator=g).to(dt)
            v = torch.randn(Hkv, ln, D, generator=g).to(dt)
            self.keys.append(k)
            self.values.append(v)
            for j in range(need[b]):
                page = order[at]
                at += 1
                table[b, j] = page
                e = min(P, ln - j * P)
                pool[layer, page, 0, :, :e] = k[:, j * P:j * P + e]
                pool[layer, page, 1, :, :e] = v[:, j * P:j * P + e]
        self.T = sum(n for _, n in rows)
        self.q = torch.randn(self.T, Hq, D, generator=g).to(dt)
        cu = [0]
        for _, n in rows:
            cu.append(cu[-1] + n)
        self.cu_host = cu
        self.table, self.pool = table.to(DEV), pool.to(DEV)
        self.qd = self.q.to(DEV)
        self.cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
        self.pos0 = torch.tensor([p0 for p0, _ in rows], dtype=torch.int32, device=DEV)
        self.shape = B.make_kv_shape(layers, Hq, Hkv, D, P, self.N, self.S, self.M, dtype)
        self.ws = torch.zeros(B.np_kv_workspace_size(self.shape), dtype=torch.uint8, device=DEV)
        self.max_len = max(max(lens), 1)
        self.scale = 1.0 / math.sqrt(D)

    def batch(self, cu=True, **kw):
        args = dict(n_seq=len(self.rows), n_tokens=self.T, max_tokens=max(n for _, n in self.rows),
                    max_len=self.max_len, pos0=self.pos0, cu_tokens=self.cu if cu else None)
        args.update(kw)
        return B.make_kv_batch(**args)

    def run(self, call, window=0, scale=None, q=None, out=None, batch=None):
        out = torch.full((self.T, self.Hq, self.D), 7.0, dtype=DT[self.dtype], device=DEV) if out is None else out
        call(self.shape, self.layer, batch or self.batch(cu=call is B.np_attn_prompt), self.table,
             self.qd if q is None else q, self.pool, self.scale if scale is None else scale, window, out, self.ws)
        torch.cuda.synchronize()
        return out.cpu()

    def check(self, out, window=0, scale=None, rows=None):
        for b, (p0, n) in enumerate(self.rows):
            if rows is not None and b not in rows:
                continue
            t = slice(self.cu_host[b], self.cu_host[b + 1])
            ref, tol = attention(self.q[t], self.keys[b], self.values[b], p0,
                                 self.scale if scale is None else scale, window, self.dtype)
            err = (out[t].double() - ref).abs()
            bad = ~(err <= tol)
            assert not bad.any(), (b, p0, n, int(bad.sum()), float(err.max()), float((err / tol).max()))

    def error(self):
        return B.np_device_error(self.ws)


HEADS = [(1, 1), (4, 2), (8, 1), (32, 8), (5, 5), (6, 2), (40, 2)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (8, 32), (80, 16), (96, 128), (256, 16), (256, 256), (200, 32)])
def test_decode_lengths(dtype, D, P):
    """Lengths from one key on, around page and step edges, one row not served."""
    rows = [(p - 1, 1) for p in (1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 129, 300)] + [(-1, 1), (5, 1)]
    s = Setup(rows, 4, 2, D, P, dtype)
    out = s.run(B.np_attn_decode)
    s.check(out)
    assert (out[12] == 0).all()
    assert s.error() == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_decode_heads(dtype, Hq, Hkv):
    s = Setup([(99, 1), (0, 1), (513, 1)], Hq, Hkv, 64, 16, dtype, seed=1)
    out = s.run(B.np_attn_decode)
    s.check(out)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("window", [1, 7, 16, 100, 5000])
def test_decode_window(dtype, window):
    s = Setup([(0, 1), (6, 1), (120, 1), (999, 1), (2303, 1)], 4, 2, 64, 32, dtype, seed=2)
    s.check(s.run(B.np_attn_decode, window=window), window=window)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_decode_long_is_split_and_joined(dtype):
    """70 001 keys: many splits; the same call twice gives the same bits."""
    s = Setup([(70000, 1)], 2, 1, 64, 64, dtype, seed=3)
    a = s.run(B.np_attn_decode)
    s.check(a)
    assert torch.equal(a, s.run(B.np_attn_decode))


PROMPTS = [
    [(0, 1)],
    [(0, 37), (0, 1), (0, 64), (0, 129)],
    [(0, 250), (13, 5), (-1, 9), (100, 70), (63, 1), (0, 0), (31, 97)],
    [(300, 3), (0, 2)],
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", range(len(PROMPTS)))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 32), (3, 3, 256, 64), (10, 2, 80, 16)])
def test_prompt_rows(dtype, rows, Hq, Hkv, D, P):
    s = Setup(PROMPTS[rows], Hq, Hkv, D, P, dtype, seed=4)
    out = s.run(B.np_attn_prompt)
    s.check(out)
    assert s.error() == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("window", [1, 33, 64, 150])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2)])
def test_prompt_window(dtype, window, Hq, Hkv):
    s = Setup([(0, 300), (170, 41), (0, 10)], Hq, Hkv, 64, 16, dtype, seed=5)
    s.check(s.run(B.np_attn_prompt, window=window), window=window)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("rows", [[(40, 1), (200, 1)], [(0, 150)]])
def test_scales(dtype, scale, rows):
    s = Setup(rows, 2, 1, 64, 16, dtype, seed=6)
    s.check(s.run(B.np_attn_prompt, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_prompt_of_single_tokens_equals_decode(dtype):
    s = Setup([(70, 1), (3, 1), (1000, 1)], 4, 2, 128, 64, dtype, seed=7)
    assert torch.equal(s.run(B.np_attn_decode), s.run(B.np_attn_prompt))


@pytest.mark.parametrize("call", [B.np_attn_decode, B.np_attn_prompt])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_views_and_in_place(call, dtype):
    """q as a view of a fused projection; out a view of a wider buffer whose
    other columns stay; out in place of q."""
    rows = [(70, 1), (3, 1)] if call is B.np_attn_decode else [(0, 90), (7, 3)]
    s = Setup(rows, 4, 2, 64, 16, dtype, seed=8)
    plain = s.run(call)
    wide = torch.full((s.T, 9, 64), 3.0, dtype=DT[dtype], device=DEV)
    wide[:, 1:5] = s.qd
    res = torch.full((s.T, 7, 64), 5.0, dtype=DT[dtype], device=DEV)
    s.run(call, q=wide[:, 1:5], out=res[:, 2:6])
    assert torch.equal(res[:, 2:6].cpu(), plain)
    assert (res[:, :2] == 5).all() and (res[:, 6:] == 5).all()
    s.run(call, q=wide[:, 1:5], out=wide[:, 1:5])
    assert torch.equal(wide[:, 1:5].cpu(), plain)
    assert (wide[:, 0] == 3).all() and (wide[:, 5:] == 3).all()


def test_rows_name_their_sequences():
    """seqs: any order of cache rows; the other layer of the pool is NaN."""
    s = Setup([(40, 1), (9, 1), (200, 1)], 4, 2, 64, 16, "f16", seed=9, layers=2, layer=1)
    base = s.run(B.np_attn_decode)
    s.check(base)
    perm = [2, 0]
    seqs = torch.tensor(perm, dtype=torch.int32, device=DEV)
    pos0 = s.pos0[perm].contiguous()
    out = torch.empty(2, 4, 64, dtype=torch.float16, device=DEV)
    batch = B.make_kv_batch(2, 2, 1, s.max_len, pos0, seqs=seqs)
    B.np_attn_decode(s.shape, 1, batch, s.table, s.qd[perm].contiguous(), s.pool, s.scale, 0, out, s.ws)
    assert torch.equal(out.cpu(), base[perm])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [[(200, 1), (90, 1)], [(150, 100), (0, 20)], [(20, 7), (0, 3)]])
def test_a_missing_page_is_not_visible(dtype, rows):
    """A table entry that names no page: reported, its keys left out, every
    other row untouched."""
    s = Setup(rows, 4, 2, 64, 16, dtype, seed=10)
    s.table[0, 1] = s.N + 5  # keys 16..31 of row 0
    call = B.np_attn_prompt
    out = s.run(call)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    s.check(out, rows=[1])
    keep = [j for j in range(s.keys[0].shape[1]) if not 16 <= j < 32]
    p0, n = rows[0]
    for i in range(n):
        vis = [j for j in keep if j <= p0 + i]
        ref, tol = attention(s.q[i:i + 1], s.keys[0][:, vis], s.values[0][:, vis], len(vis) - 1, s.scale, 0, dtype)
        assert ((out[i:i + 1].double() - ref).abs() <= tol).all(), i


def test_bad_batches_are_reported_and_not_served():
    for change in ("seq", "pos", "len"):
        s = Setup([(40, 1), (9, 1), (12, 1)], 4, 2, 64, 16, "f16", seed=11)
        seqs = torch.arange(3, dtype=torch.int32, device=DEV)
        batch = s.batch(cu=False, seqs=seqs)
        if change == "seq":
            seqs[1] = 77
        elif change == "pos":
            s.pos0[1] = 1 << 29
        else:
            s.pos0[1] = 41  # max_len is 41
        out = s.run(B.np_attn_decode, batch=batch)
        assert s.error() == B.NP_DEVERR_STATE
        assert (out[1] == 0).all()
        s.check(out, rows=[0, 2])
    s = Setup([(0, 40), (0, 9), (0, 12)], 4, 2, 64, 16, "f16", seed=11)
    s.cu[1] = 1000
    out = s.run(B.np_attn_prompt)  # rows 0 and 1 have no tokens then
    assert s.error() == B.NP_DEVERR_STATE
    s.check(out, rows=[2])
    assert (out[:49] == 7).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_pool_past_4_gib(dtype):
    """A layer whose pages lie past 32-bit byte offsets."""
    w = 2 if dtype == "f16" else 4
    Hkv, P, D = 8, 256, 128
    pages = (5 << 30) // (2 * Hkv * P * D * w)
    lens = 600
    g = torch.Generator().manual_seed(1)
    shape = B.make_kv_shape(2, 8, Hkv, D, P, pages, 1, 4, dtype)
    pool = torch.empty(2, pages, 2, Hkv, P, D, dtype=DT[dtype], device=DEV)
    k = torch.randn(Hkv, lens, D, generator=g).to(DT[dtype])
    v = torch.randn(Hkv, lens, D, generator=g).to(DT[dtype])
    ids = [pages - 1, pages - 3, 0]
    for j, p in enumerate(ids):
        e = min(P, lens - j * P)
        pool[1, p, 0, :, :e] = k[:, j * P:j * P + e].to(DEV)
        pool[1, p, 1, :, :e] = v[:, j * P:j * P + e].to(DEV)
    table = torch.tensor([ids + [-1]], dtype=torch.int32, device=DEV)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    for n, p0 in ((1, lens - 1), (70, lens - 70)):
        q = torch.randn(n, 8, D, generator=g).to(DT[dtype])
        out = torch.empty(n, 8, D, dtype=DT[dtype], device=DEV)
        pos0 = torch.tensor([p0], dtype=torch.int32, device=DEV)
        cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        batch = B.make_kv_batch(1, n, n, lens, pos0, cu_tokens=cu)
        B.np_attn_prompt(shape, 1, batch, table, q.to(DEV), pool, 0.1, 0, out, ws)
        ref, tol = attention(q, k, v, p0, 0.1, 0, dtype)
        assert ((out.cpu().double() - ref).abs() <= tol).all()
    assert B.np_device_error(ws) == 0
    del pool
    torch.cuda.empty_cache()


def test_graph_replays_follow_the_device_arrays():
    """One captured decode call, replayed while positions and queries change
    on the device, with eager work between: every replay equals the eager
    call."""
    s = Setup([(900, 1), (400, 1)], 8, 2, 128, 64, "bf16", seed=12)
    out = torch.empty_like(s.qd)
    stream = torch.cuda.Stream()
    batch = s.batch(cu=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream, capture_error_mode="thread_local"):
        B.np_attn_decode(s.shape, 0, batch, s.table, s.qd, s.pool, s.scale, 0, out, s.ws, stream)
    for i in range(4):
        s.pos0.copy_(torch.tensor([900 - 200 * i, 400 - 133 * i], dtype=torch.int32))
        s.qd.copy_(torch.roll(s.qd, 1, 0))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        eager = s.run(B.np_attn_decode, batch=batch)
        assert torch.equal(got.cpu(), eager), i


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,Hq,Hkv,D,P,top", [(70, 4, 2, 64, 16, 2500), (200, 2, 1, 64, 64, 900),
                                              (5, 40, 2, 128, 32, 9000), (3, 8, 8, 96, 16, 9000),
                                              (130, 3, 3, 256, 128, 700)])
@pytest.mark.parametrize("window", [0, 333])
def test_decode_of_ragged_batches(dtype, n, Hq, Hkv, D, P, top, window):
    """Many rows of very different lengths in one call, more keys than the
    card takes at once: rows of one key, rows not served, one row far longer
    than the rest; the second call with the same workspace gives the same
    bits."""
    g = torch.Generator().manual_seed(n)
    lens = [int(2 ** (float(torch.rand(1, generator=g)) * math.log2(top))) for _ in range(n)]
    rows = [(x - 1, 1) for x in lens]
    rows[0], rows[n // 2], rows[-1] = (top - 1, 1), (0, 1), (-1, 1)
    s = Setup(rows, Hq, Hkv, D, P, dtype, seed=13)
    out = s.run(B.np_attn_decode, window=window)
    s.check(out, window=window)
    assert (out[-1] == 0).all() and s.error() == 0
    assert torch.equal(out, s.run(B.np_attn_decode, window=window))


def test_bad_rows_of_a_ragged_batch_are_reported():
    rows = [(1999, 1)] * 100
    s = Setup(rows, 4, 4, 64, 64, "f16", seed=14)
    s.pos0[77] = 5000
    out = s.run(B.np_attn_decode)
    assert s.error() == B.NP_DEVERR_STATE
    assert (out[77] == 0).all()
    s.check(out, rows=[0, 76, 78, 99])
