"""np_attn_decode and np_attn_prompt over caches of 8-bit elements against float64
attention over the values that the elements stand for (which the type holds
exactly, so that the plain caches' bound holds: kv_ref.attention), and against
the same calls over a plain cache of those values."""
import math

import pytest
import torch

from kv8_ref import page_bytes, quantise
from kv_ref import DT, attention, div_up
from paper_2608_22643_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Setup:
    """A cache of one layer holding random keys and values for rows (p0, n): every
    slot that no token may see has NaN elements and the scale byte 255."""

    def __init__(self, rows, Hq, Hkv, D, P, dtype, seed=0, layers=1, layer=0, pages=None):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.rows, self.Hq, self.Hkv, self.D, self.P, self.dtype, self.layer = rows, Hq, Hkv, D, P, dtype, layer
        lens = [max(p0 + n, 0) if p0 >= 0 else 0 for p0, n in rows]
        need = [div_up(x, P) for x in lens]
        self.N = pages or sum(need) + 3
        self.M = max(max(need), 1) + 1
        order = torch.randperm(self.N, generator=g).tolist()
        self.S = len(rows)
        table = torch.full((self.S, self.M), -1, dtype=torch.int32)
        self.keys, self.values = [], []
        self.shape = B.make_kv_shape(layers, Hq, Hkv, D, P, self.N, self.S, self.M, dtype, "e4m3")
        pool = torch.full(B.kv_pool_shape(self.shape), 255, dtype=torch.uint8)
        at = 0
        for b, ln in enumerate(lens):
            x = torch.randn(2, Hkv, ln, D, generator=g) * torch.exp2(
                torch.randint(-3, 3, (2, Hkv, ln, 1), generator=g).float())
            byte, scale, value = quantise(x.to(dt).double(), dtype) if ln else (x.byte(), x[..., 0].byte(), x.double())
            self.keys.append(value[0])
            self.values.append(value[1])
            for j in range(need[b]):
                page = order[at]
                at += 1
                table[b, j] = page
                e = min(P, ln - j * P)
                body = torch.full((2, Hkv, P, D), 127, dtype=torch.uint8)
                sc = torch.full((2, Hkv, P), 255, dtype=torch.uint8)
                body[:, :, :e], sc[:, :, :e] = byte[:, :, j * P:j * P + e], scale[:, :, j * P:j * P + e]
                pool[layer, page] = page_bytes(body, sc)
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

    def plain(self, call, window=0, scale=None):
        """The same call over a plain cache of the values."""
        shape = B.make_kv_shape(self.shape.layers, self.Hq, self.Hkv, self.D, self.P, self.N, self.S, self.M, self.dtype)
        pool = torch.full(B.kv_pool_shape(shape), math.nan, dtype=DT[self.dtype])
        for b in range(self.S):
            for j in range(div_up(self.keys[b].shape[1], self.P)):
                for kv, x in enumerate((self.keys[b], self.values[b])):
                    y = x[:, j * self.P:(j + 1) * self.P]
                    pool[self.layer, int(self.table[b, j]), kv, :, :y.shape[1]] = y.to(DT[self.dtype])
        out = torch.zeros((self.T, self.Hq, self.D), dtype=DT[self.dtype], device=DEV)
        call(shape, self.layer, self.batch(cu=call is B.np_attn_prompt), self.table, self.qd, pool.to(DEV),
             self.scale if scale is None else scale, window, out, self.ws)
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


DTYPES = ["f32", "f16", "bf16"]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (16, 32), (80, 16), (96, 128), (256, 16), (256, 256), (208, 32),
                                 (48, 16)])
def test_decode_lengths(dtype, D, P):
    rows = [(p - 1, 1) for p in (1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 129, 300)] + [(-1, 1), (5, 1)]
    s = Setup(rows, 4, 2, D, P, dtype)
    out = s.run(B.np_attn_decode)
    s.check(out)
    assert (out[12] == 0).all() and s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (32, 8), (5, 5), (40, 2)])
def test_decode_heads(dtype, Hq, Hkv):
    s = Setup([(99, 1), (0, 1), (513, 1)], Hq, Hkv, 64, 16, dtype, seed=1)
    s.check(s.run(B.np_attn_decode))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 7, 16, 100, 5000])
def test_decode_window(dtype, window):
    s = Setup([(0, 1), (6, 1), (120, 1), (999, 1), (2303, 1)], 4, 2, 64, 32, dtype, seed=2)
    s.check(s.run(B.np_attn_decode, window=window), window=window)


@pytest.mark.parametrize("dtype", DTYPES)
def test_decode_long_is_split_and_joined(dtype):
    s = Setup([(70000, 1)], 2, 1, 64, 64, dtype, seed=3)
    a = s.run(B.np_attn_decode)
    s.check(a)
    assert torch.equal(a, s.run(B.np_attn_decode))


PROMPTS = [
    [(0, 1)],
    [(0, 37), (0, 1), (0, 64), (0, 129)],
    [(0, 250), (13, 5), (-1, 9), (100, 70), (63, 1), (0, 0), (31, 97)],
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", range(len(PROMPTS)))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 32), (3, 3, 256, 64), (10, 2, 80, 16)])
def test_prompt_rows(dtype, rows, Hq, Hkv, D, P):
    s = Setup(PROMPTS[rows], Hq, Hkv, D, P, dtype, seed=4)
    s.check(s.run(B.np_attn_prompt))
    assert s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 33, 150])
def test_prompt_window(dtype, window):
    s = Setup([(0, 300), (170, 41), (0, 10)], 8, 2, 64, 16, dtype, seed=5)
    s.check(s.run(B.np_attn_prompt, window=window), window=window)


# batches large enough for the tile kernel (16-bit types): many pairs of query and key
TILES = [
    ([(0, 1100), (700, 300), (-1, 40), (0, 0), (3, 77)], 8, 2, 128, 32, 0),
    ([(0, 900), (2000, 130)], 16, 4, 64, 16, 0),
    ([(10, 1000), (0, 513)], 32, 4, 64, 256, 333),
    ([(0, 700), (900, 100)], 16, 4, 256, 64, 0),
    ([(5, 800), (0, 300)], 16, 2, 208, 16, 700),
    ([(0, 1000), (300, 65)], 12, 4, 80, 32, 0),
    ([(2500, 64)], 64, 8, 128, 64, 0),
    ([(30000, 60)], 8, 2, 128, 64, 0),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", range(len(TILES)))
def test_prompt_tiles(dtype, case):
    """Some tokens of each batch in float64; all of them against the plain cache of the same values, whose kernel has
    the same sums in the same order."""
    rows, Hq, Hkv, D, P, window = TILES[case]
    s = Setup(rows, Hq, Hkv, D, P, dtype, seed=6 + case)
    out = s.run(B.np_attn_prompt, window=window)
    assert torch.equal(out, s.plain(B.np_attn_prompt, window=window))
    assert torch.equal(out, s.run(B.np_attn_prompt, window=window))
    for b, (p0, n) in enumerate(rows):
        t0 = s.cu_host[b]
        if p0 < 0:
            assert (out[t0:t0 + n] == 0).all()
            continue
        for i in sorted({0, n // 3, n - 1} & set(range(n))):
            ref, tol = attention(s.q[t0 + i:t0 + i + 1], s.keys[b], s.values[b], p0 + i, s.scale, window, dtype)
            assert ((out[t0 + i].double() - ref[0]).abs() <= tol[0]).all(), (b, i)
    assert s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_prompt_of_many_rows_in_row_blocks(dtype):
    s = Setup([(10, 1000), (0, 513)], 8, 1, 64, 256, dtype, seed=8)
    s.check(s.run(B.np_attn_prompt, window=333), window=333)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("rows", [[(40, 1), (200, 1)], [(0, 150)]])
def test_scales(dtype, scale, rows):
    s = Setup(rows, 2, 1, 64, 16, dtype, seed=14)
    s.check(s.run(B.np_attn_prompt, scale=scale), scale=scale)


@pytest.mark.parametrize("call", [B.np_attn_decode, B.np_attn_prompt])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_views_and_in_place(call, dtype):
    rows = [(70, 1), (3, 1)] if call is B.np_attn_decode else [(0, 90), (7, 3)]
    s = Setup(rows, 4, 2, 64, 16, dtype, seed=15)
    plain = s.run(call)
    wide = torch.full((s.T, 9, 64), 3.0, dtype=DT[dtype], device=DEV)
    wide[:, 1:5] = s.qd
    s.run(call, q=wide[:, 1:5], out=wide[:, 1:5])
    assert torch.equal(wide[:, 1:5].cpu(), plain)
    assert (wide[:, 0] == 3).all() and (wide[:, 5:] == 3).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [-1, 1 << 20])
@pytest.mark.parametrize("rows,Hq", [([(200, 1)], 4), ([(0, 100)], 4), ([(0, 1000)], 64)])
def test_missing_pages(dtype, bad, rows, Hq):
    """Keys without a page count as not visible; the others' results are those of a cache without them."""
    if dtype == "f32" and Hq == 64:
        pytest.skip("tiles are for 16-bit types")
    s = Setup(rows, Hq, 2, 64, 16, dtype, seed=16)
    s.table[0, 2] = bad  # positions 32 .. 47
    out = s.run(B.np_attn_prompt)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    p0, n = rows[0]
    keep = torch.cat((torch.arange(32), torch.arange(48, p0 + n)))
    for i in sorted({0, n // 2, n - 1}):
        p = p0 + i
        at = keep[keep <= p]
        ref, tol = attention(s.q[i:i + 1], s.keys[0][:, at], s.values[0][:, at], len(at) - 1, s.scale, 0, dtype)
        assert ((out[i].double() - ref[0]).abs() <= tol[0]).all(), i


@pytest.mark.parametrize("dtype", DTYPES)
def test_past_4_gib(dtype):
    """Pages beyond 4 GiB of a layer, in the second layer."""
    D, P, H = 128, 256, 8
    per = 2 * H * P * (D + 1)
    pages = (1 << 32) // per + 50
    s = Setup([(700, 1), (300, 1)], H, H, D, P, dtype, seed=17)
    shape = B.make_kv_shape(2, H, H, D, P, pages, s.S, s.M, dtype, "e4m3")
    pool = torch.zeros(B.kv_pool_shape(shape), dtype=torch.uint8, device=DEV)
    pool[1, pages - s.N:] = s.pool[0]
    table = torch.where(s.table >= 0, s.table + pages - s.N, s.table)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(s.qd)
    B.np_attn_decode(shape, 1, s.batch(cu=False), table, s.qd, pool, s.scale, 0, out, ws)
    s.check(out.cpu())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_scales_that_leave_little(dtype):
    """Rows with the least scale (zeros, the smallest numbers) beside ordinary ones."""
    s = Setup([(120, 1), (0, 60)], 4, 2, 64, 16, dtype, seed=18)
    for b, ln in enumerate((121, 60)):
        for p in range(0, ln, 5):
            page, slot = int(s.table[b, p // 16]), p % 16
            s.pool[0, page, :, :, slot * 64:(slot + 1) * 64] = 0
            s.pool[0, page, :, :, 16 * 64 + slot] = 1
            s.keys[b][:, p] = 0
            s.values[b][:, p] = 0
    s.check(s.run(B.np_attn_prompt))


def test_graph_replays():
    s = Setup([(700, 1), (31, 1), (2000, 1)], 8, 2, 128, 16, "bf16", seed=19)
    out = torch.zeros_like(s.qd)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    batch = s.batch(cu=False)
    B.np_attn_decode(s.shape, 0, batch, s.table, s.qd, s.pool, s.scale, 0, out, s.ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.np_attn_decode(s.shape, 0, batch, s.table, s.qd, s.pool, s.scale, 0, out, s.ws, side)
    g = torch.Generator().manual_seed(20)
    for i in range(4):
        s.qd.copy_(torch.randn(s.q.shape, generator=g).to(s.q.dtype))
        s.pos0.copy_(torch.tensor([700 - i, 31 - i, 2000 - 7 * i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got.cpu(), s.run(B.np_attn_decode, batch=batch))
