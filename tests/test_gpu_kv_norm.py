"""np_kv_append_norm, appends into caches of 8-bit elements, and np_kv_read: heads
against float64 within a bound derived from the arithmetic (kv8_ref.norm_rotate),
stored elements bit for bit against a search among all of them, page calls over
8-bit pages, what is not served, HIP graphs."""
import math

import pytest
import torch

from kv8_ref import norm_rotate, quantise, split_page, values_of
from kv_ref import DT, PageModel, div_up
from paper_2608_22643_amd import binding as B
from paper_2608_22643_amd.kvcache import rotary_tables

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [(0, 37), (13, 5), (-1, 3), (100, 1), (0, 0), (31, 33)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Setup:
    def __init__(self, rows, Hq, Hkv, D, P, dtype, cache="same", seed=0, layers=1, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.Hq, self.Hkv, self.D, self.P, self.dtype, self.cache = rows, Hq, Hkv, D, P, dtype, cache
        lens = [p0 + n if p0 >= 0 else 0 for p0, n in rows]
        need = [div_up(x, P) for x in lens]
        self.N, self.M, S = sum(need) + 2, max(max(need), 1) + 1, len(rows)
        order = torch.randperm(self.N, generator=g).tolist()
        self.table = torch.full((S, self.M), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
            at += k
        self.T = T = sum(n for _, n in rows)
        dt = DT[dtype]
        # heads of very different sizes
        size = torch.exp2(torch.randint(-6, 4, (T, Hq + 2 * Hkv, 1), generator=g).float()) * scale
        self.qkv = (torch.randn(T, Hq + 2 * Hkv, D, generator=g) * size).to(dt)
        self.wq, self.wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(dt) for _ in range(2))
        self.pos = torch.cat([torch.arange(p0, p0 + n) if p0 >= 0 else torch.full((n,), -1) for p0, n in rows])
        self.row = torch.cat([torch.full((n,), b) for b, (_, n) in enumerate(rows)])
        cu = [0]
        for _, n in rows:
            cu.append(cu[-1] + n)
        self.shape = B.make_kv_shape(layers, Hq, Hkv, D, P, self.N, S, self.M, dtype, cache)
        self.pool = torch.full(B.kv_pool_shape(self.shape), 111 if cache == "e4m3" else 7,
                               dtype=torch.uint8 if cache == "e4m3" else dt, device=DEV)
        self.ws = torch.zeros(B.np_kv_workspace_size(self.shape), dtype=torch.uint8, device=DEV)
        self.dev = self.qkv.to(DEV)
        self.tab = self.table.to(DEV)
        self.q_out = torch.full((T, Hq, D), 5.0, dtype=dt, device=DEV)
        self.longest = max(max(lens), 1)
        self.batch = B.make_kv_batch(S, T, max(n for _, n in rows), self.longest, i32([p0 for p0, _ in rows]),
                                     cu_tokens=i32(cu))

    def heads(self):
        Hq, Hkv = self.Hq, self.Hkv
        return self.dev[:, :Hq], self.dev[:, Hq:Hq + Hkv], self.dev[:, Hq + Hkv:]

    def append(self, eps=None, weights=True, rotary=None, layer=0, stream=None):
        q, k, v = self.heads()
        norm = None
        if eps is not None:
            norm = B.make_qk_norm(*((self.wq.to(DEV), self.wk.to(DEV)) if weights else (None, None)), eps)
        B.np_kv_append_norm(self.shape, layer, self.batch, self.tab, B.make_qkv(q, k, v, self.q_out), norm, rotary,
                            self.pool, self.ws, stream)

    def read(self, layer=0):
        k, v = (torch.full((self.T, self.Hkv, self.D), 9.0, dtype=DT[self.dtype], device=DEV) for _ in range(2))
        B.np_kv_read(self.shape, layer, self.batch, self.tab, self.pool, k, v, self.ws)
        return k.cpu(), v.cpu()

    def stored(self, layer=0):
        """Served tokens' keys and values as they lie in the pool: elements of w, or (bytes, scales)."""
        at = self.pos >= 0
        page = self.table[self.row[at], self.pos[at] // self.P].long()
        slot = self.pos[at] % self.P
        pool = self.pool[layer].cpu()
        if self.cache == "e4m3":
            body, scale = split_page(pool, self.P, self.D)
            return [(body[page, kv, :, slot], scale[page, kv, :, slot]) for kv in (0, 1)]
        return [pool[page, kv, :, slot] for kv in (0, 1)]

    def untouched(self):
        """Pool bytes that no served token has: what they were."""
        mask = torch.ones(self.N, self.P, dtype=torch.bool)
        at = self.pos >= 0
        mask[self.table[self.row[at], self.pos[at] // self.P].long(), self.pos[at] % self.P] = False
        pool = self.pool[0].cpu()
        if self.cache != "e4m3":
            return (pool.permute(0, 3, 1, 2, 4)[mask] == 7).all()
        body, scale = split_page(pool, self.P, self.D)
        return (body.permute(0, 3, 1, 2, 4)[mask] == 111).all() and (scale.permute(0, 3, 1, 2)[mask] == 111).all()


def check(s, got, x, weight, eps, cos, sin, inter):
    at = s.pos >= 0
    ref, tol = norm_rotate(x.cpu()[at], weight, eps, cos, sin, s.pos[at], inter, s.dtype)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), (float(err.max()), float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,D,P,R,inter", [
    (4, 2, 64, 16, 64, False), (8, 1, 128, 64, 64, True), (3, 3, 256, 32, 16, False), (10, 2, 80, 16, 32, False),
    (5, 5, 8, 32, 0, False), (40, 8, 128, 128, 128, False), (2, 1, 256, 16, 256, True), (4, 4, 96, 256, 96, False)])
def test_norm(dtype, Hq, Hkv, D, P, R, inter):
    s = Setup(ROWS, Hq, Hkv, D, P, dtype, seed=D + R)
    cos, sin = rotary_tables(R, s.longest) if R else (None, None)
    s.append(1e-5, rotary=B.make_rotary(cos, sin, inter) if R else None)
    c, n = (cos.cpu(), sin.cpu()) if R else (None, None)
    q, k, v = s.heads()
    at = s.pos >= 0
    check(s, s.q_out.cpu()[at], q, s.wq, 1e-5, c, n, inter)
    keys, values = s.stored()
    check(s, keys, k, s.wk, 1e-5, c, n, inter)
    assert torch.equal(values, v.cpu()[at])
    assert (s.q_out.cpu()[~at] == 5).all() and s.untouched()
    assert B.np_device_error(s.ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weights", [True, False])
def test_norm_without_weights_or_rotation(dtype, weights):
    s = Setup(ROWS, 4, 2, 64, 16, dtype, seed=1)
    s.append(0.5, weights=weights)
    at = s.pos >= 0
    check(s, s.q_out.cpu()[at], s.heads()[0], s.wq if weights else None, 0.5, None, None, False)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_norm_none_is_plain_append(cache):
    """The same queries bit for bit, and in a plain cache the same pool."""
    rot = B.make_rotary(*rotary_tables(64, 200))
    a, b = Setup(ROWS, 4, 2, 64, 16, "bf16", cache, seed=2), Setup(ROWS, 4, 2, 64, 16, "bf16", cache, seed=2)
    a.append(None, rotary=rot)
    q, k, v = b.heads()
    B.np_kv_append(b.shape, 0, b.batch, b.tab, B.make_qkv(q, k, v, b.q_out), rot, b.pool, b.ws)
    assert torch.equal(a.q_out, b.q_out) and torch.equal(a.pool, b.pool)


def test_norm_far_sizes():
    """Sums of squares past both ends of fp32, heads of zeros, eps of 0, and what is not finite."""
    for eps in (0.0, 1e-6, 1e-30):
        s = Setup([(0, 12)], 2, 1, 64, 16, "f32", seed=3)
        q = s.qkv[:, :2].clone()
        for t, size in enumerate((1e25, 1e-25, 3e38, 1e-38, 1e19, 1e-19, 1e-13)):
            q[t] = q[t] / q[t].abs().amax(-1, keepdim=True) * size
        q[7] = 0
        q[8, :, 3], q[9, :, 5] = math.inf, math.nan
        s.dev[:, :2] = q.to(DEV)
        s.append(eps, weights=False)
        got = s.q_out.cpu()
        ref, tol = norm_rotate(q[:8], None, eps, None, None, None, False, "f32")
        # magnitudes next to 1e-38 have fewer digits: a denormal step of each term
        tol = tol + 2.0 ** -149 * (1 + 1 / q[:8].double().abs().amax(-1, keepdim=True).clamp(min=1e-38))
        assert ((got[:8].double() - ref).abs() <= tol).all(), (eps, (got[:8].double() - ref).abs().amax((1, 2)))
        assert (got[8, :, :3] == 0).all() and got[8, :, 3].isnan().all() and (got[8, :, 4:] == 0).all()
        assert got[9].isnan().all()
        assert torch.isfinite(got[10:]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,D,P,R,inter", [
    (4, 2, 64, 16, 64, False), (8, 1, 128, 64, 64, True), (3, 3, 256, 32, 16, False), (10, 2, 80, 16, 32, False),
    (5, 5, 16, 32, 0, False), (40, 8, 128, 128, 128, False), (2, 1, 256, 16, 256, True)])
@pytest.mark.parametrize("eps", [None, 1e-5])
def test_elements_bit_for_bit(dtype, Hq, Hkv, D, P, R, inter, eps):
    """The cache holds the elements of the exact keys, rounded to w, and of the values."""
    s = Setup(ROWS, Hq, Hkv, D, P, dtype, "e4m3", seed=4)
    cos, sin = rotary_tables(R, 200) if R else (None, None)
    s.append(eps, rotary=B.make_rotary(cos, sin, inter) if R else None)
    at = s.pos >= 0
    c, n = (cos.cpu(), sin.cpu()) if R else (None, None)
    q, k, v = (x.cpu() for x in s.heads())
    check(s, s.q_out.cpu()[at], q, s.wq, eps, c, n, inter)
    keys, _ = norm_rotate(k[at], s.wk, eps, c, n, s.pos[at], inter, dtype)
    back = s.read()
    for x, (byte, scale), r in zip((keys.float().to(DT[dtype]), v[at]), s.stored(), back):
        eb, es, ev = quantise(x.double(), dtype)
        assert torch.equal(scale, es) and torch.equal(byte, eb)
        assert torch.equal(r[at].double(), ev) and torch.equal(values_of(byte, scale), ev)
        assert (r[~at] == 0).all()
    assert s.untouched() and B.np_device_error(s.ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_elements_of_every_size(dtype):
    """Rows from the smallest numbers of the type to its largest, ties, zeros and what is not finite."""
    s = Setup([(0, 64)], 2, 2, 64, 16, dtype, "e4m3", seed=5)
    lo, hi = {"f16": (-24, 15), "bf16": (-130, 127), "f32": (-140, 127)}[dtype]
    x = s.qkv.float()
    for t in range(60):
        x[t] = x[t] / x[t].abs().amax(-1, keepdim=True) * 2.0 ** (lo + (hi - lo) * t / 59)
    x = x.to(DT[dtype])
    x[40] = torch.finfo(DT[dtype]).max * torch.sign(x[40].float()).to(DT[dtype])
    x[41, :, ::2] = 0.0
    x[42] = torch.arange(64).to(DT[dtype]) * 1.0625  # ties among them
    x[60] = 0.0
    x[61, :, 7], x[61, :, 8], x[62, :, 9] = math.inf, -math.inf, math.nan
    x[63] = math.inf
    s.dev.copy_(x)
    s.append(None)
    for j, (byte, scale) in enumerate(s.stored()):
        eb, es, ev = quantise(x[:, 2 + 2 * j:4 + 2 * j].double(), dtype)
        assert torch.equal(scale, es), (scale - es).nonzero()
        bad = (byte != eb) & ~((byte & 127 == 127) & (eb & 127 == 127))  # NaN has either sign
        assert not bad.any(), (bad.nonzero()[:5], byte[bad][:5], eb[bad][:5])
        got = s.read()[j]
        assert torch.equal(got.double().nan_to_num(1e300), ev.nan_to_num(1e300))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_read_plain_cache_and_missing_pages(dtype):
    s = Setup(ROWS, 4, 2, 64, 16, dtype, seed=6)
    s.append(None)
    at = s.pos >= 0
    k, v = s.read()
    for got, x in ((k, s.heads()[1]), (v, s.heads()[2])):
        assert torch.equal(got[at], x.cpu()[at]) and (got[~at] == 0).all()
    only = torch.full_like(s.q_out[:, :2], 3.0)
    B.np_kv_read(s.shape, 0, s.batch, s.tab, s.pool, None, only, s.ws)
    assert torch.equal(only.cpu(), v)
    assert B.np_device_error(s.ws) == 0
    s.tab[0, 1] = -1  # positions 16 .. 31 of row 0
    s.tab[3, 100 // 16] = s.N
    k2, _ = s.read()
    gone = ((s.row == 0) & (s.pos >= 16) & (s.pos < 32)) | (s.row == 3)
    assert (k2[gone] == 0).all() and torch.equal(k2[~gone], k[~gone])
    assert B.np_device_error(s.ws) == B.NP_DEVERR_NOT_RESIDENT


def test_read_strided_views_and_nobodys_tokens():
    s = Setup(ROWS, 4, 2, 64, 16, "bf16", "e4m3", seed=7)
    s.append(None)
    k, v = s.read()
    wide = torch.full((s.T + 3, 6, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    b = s.batch
    more = B.make_kv_batch(b.n_seq, s.T + 3, b.max_tokens, s.longest, b._kept[0], cu_tokens=b._kept[2])
    B.np_kv_read(s.shape, 0, more, s.tab, s.pool, wide[:, 1:3], wide[:, 4:6], s.ws)
    w = wide.cpu()
    assert torch.equal(w[:s.T, 1:3], k) and torch.equal(w[:s.T, 4:6], v)
    assert (w[:, 0] == 3).all() and (w[:, 3] == 3).all() and (w[s.T:] == 3).all()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_in_place_and_other_layers(cache):
    """q_out in place of q; the other layers of the pool stay."""
    a, b = (Setup(ROWS, 4, 2, 64, 16, "f16", cache, seed=8, layers=3) for _ in range(2))
    a.append(1e-6, layer=1)
    q, k, v = b.heads()
    B.np_kv_append_norm(b.shape, 1, b.batch, b.tab, B.make_qkv(q, k, v, q), B.make_qk_norm(b.wq.to(DEV), b.wk.to(DEV)),
                        None, b.pool, b.ws)
    at = (a.pos >= 0).to(DEV)
    assert torch.equal(a.q_out[at], q[at]) and torch.equal(a.pool, b.pool)
    assert (a.pool[::2] == (111 if cache == "e4m3" else 7)).all()


def test_bad_rows_are_left_out():
    """A position past the rotary tables, and one past max_len."""
    s = Setup([(0, 4), (50, 2)], 4, 2, 64, 16, "f16", "e4m3", seed=9)
    s.append(1e-6, rotary=B.make_rotary(*rotary_tables(64, 51)))
    assert B.np_device_error(s.ws) == B.NP_DEVERR_STATE
    assert (s.q_out.cpu()[5] == 5).all() and (s.q_out.cpu()[:5] != 5).any(-1).all()
    k, _ = s.read()
    assert torch.isfinite(k[:5]).all()


def test_page_calls_on_8_bit_pages():
    """Sequences that grow, fork, are freed and compacted: what np_kv_read reads back is what was appended."""
    g = torch.Generator().manual_seed(10)
    S, N, M, P, H, D, L = 5, 24, 6, 16, 2, 32, 2
    shape = B.make_kv_shape(L, H, H, D, P, N, S, M, "f16", "e4m3")
    table, kv_len, refs = (torch.empty(n, dtype=torch.int32, device=DEV) for n in ((S, M), S, N))
    state = B.make_kv_state(table, kv_len, refs)
    pool = torch.zeros(B.kv_pool_shape(shape), dtype=torch.uint8, device=DEV)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    B.np_kv_reset(shape, state, ws)
    model, text = PageModel(S, N, M, P), [[] for _ in range(S)]

    def grow(seqs, new):
        T = sum(new)
        x = torch.randn(T, L, 2 * H, D, generator=g).half()
        pos0 = torch.empty(len(seqs), dtype=torch.int32, device=DEV)
        sd, cu = i32(seqs), i32([sum(new[:i]) for i in range(len(new) + 1)])
        B.np_kv_extend(shape, state, pool, len(seqs), sd, i32(new), pos0, ws)
        assert pos0.tolist() == model.extend(seqs, new)
        batch = B.make_kv_batch(len(seqs), T, max(new), M * P, pos0, seqs=sd, cu_tokens=cu)
        q = torch.zeros(T, H, D, dtype=torch.float16, device=DEV)
        for layer in range(L):
            y = x[:, layer].to(DEV)
            B.np_kv_append(shape, layer, batch, table, B.make_qkv(q, y[:, :H], y[:, H:], q), None, pool, ws)
        t = 0
        for s, n in zip(seqs, new):
            text[s] += list(x[t:t + n])
            t += n

    def fork(a, b, n):
        B.np_kv_fork(shape, state, 1, i32([a]), i32([b]), i32([n]), ws)
        model.fork([a], [b], [n])
        text[b] = text[a][:n]

    def see():
        assert table.tolist() == model.tables() and refs.tolist() == model.refs
        seqs = [s for s in range(S) if text[s]]
        n = [len(text[s]) for s in seqs]
        batch = B.make_kv_batch(len(seqs), sum(n), max(n), M * P, i32([0] * len(seqs)), seqs=i32(seqs),
                                cu_tokens=i32([sum(n[:i]) for i in range(len(n) + 1)]))
        k, v = (torch.zeros(sum(n), H, D, dtype=torch.float16, device=DEV) for _ in range(2))
        want = torch.stack([x for s in seqs for x in text[s]])
        for layer in range(L):
            B.np_kv_read(shape, layer, batch, table, pool, k, v, ws)
            _, _, ev = quantise(want[:, layer].double(), "f16")
            assert torch.equal(torch.cat((k, v), 1).cpu().double(), ev)

    grow([0, 2], [37, 20])
    fork(0, 1, 37)
    fork(0, 3, 21)
    see()
    grow([1, 0, 3, 2], [1, 30, 5, 12])  # copies of shared last pages
    see()
    B.np_kv_free(shape, state, 1, i32([0]), ws)
    model.free([0])
    text[0] = []
    B.np_kv_compact(shape, state, pool, None, ws)
    model.compact()
    see()
    grow([4], [50])
    see()
    assert B.np_device_error(ws) == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_graph_replays(cache):
    """One captured step of append and read, replayed with new heads between eager work."""
    s = Setup([(3, 1), (40, 1), (16, 1)], 8, 2, 128, 16, "bf16", cache, seed=11)
    rot = B.make_rotary(*rotary_tables(128, 100))
    q, k, v = s.heads()
    qkv, norm = B.make_qkv(q, k, v, s.q_out), B.make_qk_norm(s.wq.to(DEV), s.wk.to(DEV))
    ko, vo = (torch.empty(3, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step(stream):
        B.np_kv_append_norm(s.shape, 0, s.batch, s.tab, qkv, norm, rot, s.pool, s.ws, stream)
        B.np_kv_read(s.shape, 0, s.batch, s.tab, s.pool, ko, vo, s.ws, stream)

    step(None)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    g = torch.Generator().manual_seed(12)
    for _ in range(4):
        s.dev.copy_(torch.randn(s.dev.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (s.q_out, s.pool, ko, vo)]
        step(None)
        torch.cuda.synchronize()
        for a, b in zip(got, (s.q_out, s.pool, ko, vo)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_past_4_gib(dtype):
    """Elements, scales and read tokens beyond 4 GiB of a layer, in the second layer: the bytes of a small pool."""
    s = Setup([(250, 20), (0, 30)], 8, 8, 128, 256, dtype, "e4m3", seed=12)
    rot = B.make_rotary(*rotary_tables(128, 300))
    s.append(1e-6, rotary=rot)
    small, want = s.pool, s.read()
    q_out, n = s.q_out.clone(), s.N
    pages = (1 << 32) // (2 * 8 * 256 * 129) + 50
    s.shape = B.make_kv_shape(2, 8, 8, 128, 256, pages, len(s.rows), s.M, dtype, "e4m3")
    s.pool = torch.full(B.kv_pool_shape(s.shape), 111, dtype=torch.uint8, device=DEV)
    s.ws = torch.zeros(B.np_kv_workspace_size(s.shape), dtype=torch.uint8, device=DEV)
    s.tab = torch.where(s.tab >= 0, s.tab + pages - n, s.tab)
    s.q_out.fill_(5)
    s.append(1e-6, rotary=rot, layer=1)
    assert torch.equal(s.pool[1, pages - n:], small[0]) and torch.equal(s.q_out, q_out)
    assert (s.pool[1, :pages - n] == 111).all() and (s.pool[0] == 111).all()
    assert all(torch.equal(x, y) for x, y in zip(s.read(1), want))
    assert B.np_device_error(s.ws) == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_the_largest_batches(cache):
    """A token in each of 4096 rows; 2^24 tokens, more than a launch has workgroups of 256 threads along an axis."""
    s = Setup([(b % 7, 1) for b in range(4096)], 2, 1, 16, 16, "f16", cache, seed=13)
    s.append(0.0, weights=False)
    k, v = s.read()
    x = s.qkv[:, 3:].double()
    assert torch.equal(v.double(), quantise(x, "f16")[2] if cache == "e4m3" else x)
    T = 1 << 24
    dev = torch.zeros(T, 4, 16, dtype=torch.float16, device=DEV)
    at = [0, 1, T // 2, T - 2, T - 1]
    dev[at] = s.dev[:5]
    # rows of two, one and two tokens, and the tokens between in rows that are not served
    cu = i32([0, 2, T // 2, T // 2 + 1, T - 2, T])
    pos0, seqs = i32([0, -1, 2, -1, 14]), i32([0, 3, 1, 3, 2])
    batch = B.make_kv_batch(5, T, T, 16, pos0, seqs=seqs, cu_tokens=cu)
    table = i32([[3], [1], [2], [0], [-1]])
    shape = B.make_kv_shape(1, 2, 1, 16, 16, 4, 5, 1, "f16", cache)
    pool = torch.zeros(B.kv_pool_shape(shape), dtype=s.pool.dtype, device=DEV)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    q_out = torch.full((T, 2, 16), 5.0, dtype=torch.float16, device=DEV)
    B.np_kv_append_norm(shape, 0, batch, table, B.make_qkv(dev[:, :2], dev[:, 2:3], dev[:, 3:], q_out),
                        B.make_qk_norm(None, None, 0.0), None, pool, ws)
    assert torch.equal(q_out[at], s.q_out[:5]) and (q_out[2:T // 2] == 5).all() and (q_out[T // 2 + 1:T - 2] == 5).all()
    ko, vo = (torch.full((T, 1, 16), 9.0, dtype=torch.float16, device=DEV) for _ in range(2))
    B.np_kv_read(shape, 0, batch, table, pool, ko, vo, ws)
    assert torch.equal(ko[at].cpu(), k[:5]) and torch.equal(vo[at].cpu(), v[:5])
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert not ko[rest].any() and not vo[rest].any()  # tokens of rows that are not served
    assert B.np_device_error(ws) == 0
