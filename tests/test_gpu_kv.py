"""np_kv_* on the GPU: the page bookkeeping against a list model (exact page
ids, lengths, reference counts, page contents), the append against float64
rotary positions, refusals found on the device."""
import random

import pytest
import torch

from kv_ref import DT, UNIT, PageModel, rotate
from paper_2608_22643_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


class Cache:
    """Device cache and list model side by side.  Slot contents are token
    numbers, written by torch (the calls only move them)."""

    def __init__(self, S, N, M, P, dtype="f32", layers=2, Hkv=1, D=8):
        self.m = PageModel(S, N, M, P)
        self.shape = B.make_kv_shape(layers, Hkv, Hkv, D, P, N, S, M, dtype)
        self.pool = torch.zeros(layers, N, 2, Hkv, P, D, dtype=DT[dtype], device=DEV)
        self.table = torch.full((S, M), -9, dtype=torch.int32, device=DEV)
        self.kv_len = torch.full((S,), -9, dtype=torch.int32, device=DEV)
        self.refs = torch.full((N,), -9, dtype=torch.int32, device=DEV)
        self.kv = B.make_kv_state(self.table, self.kv_len, self.refs)
        self.ws = torch.full((B.np_kv_workspace_size(self.shape),), 0x5A, dtype=torch.uint8, device=DEV)
        B.np_kv_reset(self.shape, self.kv, self.ws)
        self.next = 1
        self.same()

    def same(self):
        torch.cuda.synchronize()
        assert self.kv_len.tolist() == self.m.len
        assert self.refs.tolist() == self.m.refs
        assert self.table.tolist() == self.m.tables()

    def contents(self):
        """Every token of every sequence, in every layer, is the model's."""
        L = self.pool.shape[0]
        pool = self.pool.cpu()
        for s in range(self.m.S):
            for i in range(self.m.len[s]):
                page, slot = self.m.table[s][i // self.m.P], i % self.m.P
                want = self.m.data[page][slot]
                if want is None:
                    continue
                for layer in range(L):
                    k, v = pool[layer, page, 0, :, slot], pool[layer, page, 1, :, slot]
                    assert (k == want + layer).all() and (v == -want - layer).all(), (s, i, layer)

    def write(self, seqs, new, pos0):
        L = self.pool.shape[0]
        off = torch.arange(L, device=DEV, dtype=torch.float32)[:, None, None]
        for s, n, p0 in zip(seqs, new, pos0):
            for i in range(n if p0 >= 0 else 0):
                page, slot = self.m.table[s][(p0 + i) // self.m.P], (p0 + i) % self.m.P
                self.m.data[page][slot] = self.next
                self.pool[:, page, 0, :, slot] = (self.next + off).to(self.pool.dtype)
                self.pool[:, page, 1, :, slot] = (-self.next - off).to(self.pool.dtype)
                self.next += 1

    def extend(self, seqs, new):
        pos0 = torch.full((len(seqs),), -5, dtype=torch.int32, device=DEV)
        B.np_kv_extend(self.shape, self.kv, self.pool, len(seqs), i32(seqs), i32(new), pos0, self.ws)
        want = self.m.extend(seqs, new)
        self.same()
        assert pos0.tolist() == want
        return want

    def fork(self, src, dst, lens=None):
        B.np_kv_fork(self.shape, self.kv, len(src), i32(src), i32(dst), None if lens is None else i32(lens), self.ws)
        self.m.fork(src, dst, lens)
        self.same()

    def free(self, seqs):
        B.np_kv_free(self.shape, self.kv, len(seqs), i32(seqs), self.ws)
        self.m.free(seqs)
        self.same()

    def compact(self):
        moved = i32([-1])
        B.np_kv_compact(self.shape, self.kv, self.pool, moved, self.ws)
        want = self.m.compact()
        self.same()
        assert moved.tolist() == [want]

    def error(self):
        return B.np_device_error(self.ws)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("P,N,S", [(16, 40, 9), (32, 17, 5), (64, 300, 40)])
def test_random_serving_follows_the_model(seed, P, N, S):
    rng = random.Random(seed)
    c = Cache(S, N, M=12, P=P)
    for _ in range(40):
        op = rng.random()
        if op < 0.5:
            seqs = rng.sample(range(S), rng.randint(1, S))
            new = [rng.choice([0, 1, 1, 1, P - 1, P, P + 1, rng.randint(1, 3 * P)]) for _ in seqs]
            c.write(seqs, new, c.extend(seqs, new))
        elif op < 0.75:
            n = rng.randint(1, max(1, S // 2))
            src = [rng.randrange(S) for _ in range(n)]
            dst = [rng.randrange(S) for _ in range(n)]
            lens = None if rng.random() < 0.5 else [rng.randint(0, max(c.m.len[s], 0)) for s in src]
            c.fork(src, dst, lens)
        elif op < 0.9:
            c.free([rng.randrange(S) for _ in range(rng.randint(1, max(1, S // 3)))])
        else:
            c.compact()
        c.contents()


def test_defaults_take_every_sequence_and_one_token():
    """seqs NULL: sequence b; n_new NULL: one token each; lens NULL: all."""
    c = Cache(4, 20, 4, 16)
    pos0 = torch.full((4,), -5, dtype=torch.int32, device=DEV)
    for step in range(20):
        B.np_kv_extend(c.shape, c.kv, c.pool, 4, None, None, pos0, c.ws)
        assert c.m.extend(range(4), [1] * 4) == [step] * 4
        c.same()
        assert pos0.tolist() == [step] * 4
    B.np_kv_free(c.shape, c.kv, 2, None, c.ws)
    c.m.free([0, 1])
    c.same()
    assert c.error() == 0


def test_the_last_holder_keeps_a_shared_page():
    """A parent and its children extend in one call: all holders of the page
    are there, the first row keeps it, the others get copies."""
    c = Cache(4, 12, 4, 16)
    c.write([1], [20], c.extend([1], [20]))
    c.fork([1, 1], [0, 3])
    page = c.m.table[1][1]
    c.write([3, 1, 0], [1, 1, 1], c.extend([3, 1, 0], [1, 1, 1]))
    assert c.m.table[3][1] == page and c.m.table[1][1] != page and c.m.table[0][1] != page
    c.contents()
    # a whole shared page is not copied: nothing is written to it
    c.fork([1], [2], [16])
    c.write([2], [1], c.extend([2], [1]))
    assert c.m.table[2][0] == c.m.table[1][0]
    c.contents()
    assert c.error() == 0


def test_too_few_pages_change_nothing():
    c = Cache(3, 4, 8, 16)
    c.write([0, 1], [30, 16], c.extend([0, 1], [30, 16]))
    assert c.extend([0, 1, 2], [1, 1, 17]) == [-1, -1, -1]
    assert c.error() == B.NP_DEVERR_OVERFLOW
    assert c.extend([0, 1], [2, 16]) == [30, 16]
    assert c.extend([0], [2000]) == [-1]  # past M P tokens
    c.contents()


def test_bad_rows_are_left_out():
    c = Cache(6, 30, 4, 16)
    assert c.extend([0, 7, 0, -1, 2], [3, 1, 1, 1, -2]) == [0, -1, -1, -1, -1]
    assert c.error() == B.NP_DEVERR_STATE
    c.fork([0, 0, 9, 0], [1, 1, 2, 0])      # named twice, outside, not empty
    c.fork([0, 0], [2, 3], [4, -1])         # longer than it is, negative
    c.free([1, 1, 77, 3])
    assert c.m.len == [3, 0, 0, 0, 0, 0]
    assert c.error() == B.NP_DEVERR_STATE


@pytest.mark.parametrize("dtype,Hkv,D,P", [("f16", 3, 80, 16), ("bf16", 8, 128, 64), ("f32", 2, 256, 32)])
def test_copies_move_whole_heads(dtype, Hkv, D, P):
    """Contents of pages with several heads and odd head sizes, after a fork
    and a compaction, against the sequences' values."""
    g = torch.Generator().manual_seed(3)
    L, N, S, M = 3, 24, 6, 4
    shape = B.make_kv_shape(L, Hkv, Hkv, D, P, N, S, M, dtype)
    m = PageModel(S, N, M, P)
    pool = torch.randn(L, N, 2, Hkv, P, D, generator=g).to(DT[dtype]).to(DEV)
    table = torch.empty(S, M, dtype=torch.int32, device=DEV)
    kv_len, refs = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (S, N))
    kv = B.make_kv_state(table, kv_len, refs)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    B.np_kv_reset(shape, kv, ws)
    pos0 = torch.empty(S, dtype=torch.int32, device=DEV)

    def read(s):
        n = m.len[s]
        x = pool[:, torch.tensor(m.table[s], device=DEV)]  # [L][pages][2][Hkv][P][D]
        return x.permute(0, 2, 3, 1, 4, 5).reshape(L, 2, Hkv, -1, D)[:, :, :, :n].cpu()

    def extend(seqs, new):
        B.np_kv_extend(shape, kv, pool, len(seqs), i32(seqs), i32(new), pos0, ws)
        m.extend(seqs, new)

    extend([0, 1, 2], [2 * P + 5, P, P - 3])
    held = [read(s) for s in range(3)]
    B.np_kv_fork(shape, kv, 2, i32([0, 2]), i32([4, 5]), None, ws)
    m.fork([0, 2], [4, 5])
    before = pool.clone()
    extend([4, 5], [1, 9])
    for s, parent in ((4, 0), (5, 2)):
        n = held[parent].shape[3]
        assert torch.equal(read(s)[:, :, :, :n], held[parent]), s
    # slots past the copied tokens keep what they held
    new = m.table[4][2]
    assert torch.equal(pool[:, new, :, :, 5:], before[:, new, :, :, 5:])
    whole = {s: read(s) for s in (2, 4, 5)}
    B.np_kv_free(shape, kv, 2, i32([0, 1]), ws)
    m.free([0, 1])
    B.np_kv_compact(shape, kv, pool, None, ws)
    assert m.compact() > 0
    assert table.tolist() == m.tables() and refs.tolist() == m.refs
    for s, x in whole.items():
        assert torch.equal(read(s), x), s
    assert B.np_device_error(ws) == 0


ROWS = [[(0, 1)], [(5, 1), (31, 1), (-1, 1), (16, 1), (0, 1)], [(0, 70), (-1, 4), (14, 5), (0, 0), (33, 1)]]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,D,P,R,inter", [(4, 2, 64, 16, 64, False), (4, 2, 64, 16, 64, True),
                                                (3, 1, 80, 32, 16, False), (3, 1, 80, 32, 48, True),
                                                (32, 8, 128, 64, 128, False), (2, 2, 256, 16, 0, False),
                                                (5, 5, 24, 16, 16, True), (2, 1, 8, 16, 0, False)])
@pytest.mark.parametrize("rows", range(len(ROWS)))
def test_append(dtype, Hq, Hkv, D, P, R, inter, rows):
    """Rotated queries and keys within the rounding of one fp32 rotation and
    one conversion, values and everything not turned bit for bit, nothing
    else written."""
    rows = ROWS[rows]
    g = torch.Generator().manual_seed(11)
    dt = DT[dtype]
    T, S = sum(n for _, n in rows), len(rows)
    M, layers, layer = 6, 2, 1
    N = S * M
    table = torch.randperm(N, generator=g).int().view(S, M)
    cu = [0]
    for _, n in rows:
        cu.append(cu[-1] + n)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dt)
    dev = qkv.to(DEV)
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    pool = torch.full((layers, N, 2, Hkv, P, D), 9.0, dtype=dt, device=DEV)
    out = torch.full((T, Hq, D), 9.0, dtype=dt, device=DEV)
    ang = torch.rand(120, max(R // 2, 1), generator=g, dtype=torch.float64) * 6.3
    cos, sin = ang.cos().float(), ang.sin().float()
    shape = B.make_kv_shape(layers, Hq, Hkv, D, P, N, S, M, dtype)
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    ones = all(n == 1 for _, n in rows)
    batch = B.make_kv_batch(S, T, max(n for _, n in rows), 200, i32(p0 for p0, _ in rows),
                            cu_tokens=None if ones else i32(cu))
    rot = B.make_rotary(cos.to(DEV), sin.to(DEV), inter) if R else None
    B.np_kv_append(shape, layer, batch, table.to(DEV), B.make_qkv(q, k, v, out), rot, pool, ws)
    torch.cuda.synchronize()
    assert B.np_device_error(ws) == 0
    want_out = torch.full((T, Hq, D), 9.0, dtype=torch.float64)
    want = torch.full(tuple(pool.shape), 9.0, dtype=torch.float64)
    for b, (p0, n) in enumerate(rows):
        if p0 < 0 or n == 0:
            continue
        x = qkv[cu[b]:cu[b + 1]]
        pos = torch.arange(p0, p0 + n)
        turn = (lambda y: rotate(y, cos, sin, pos, inter)) if R else (lambda y: y.double())
        want_out[cu[b]:cu[b + 1]] = turn(x[:, :Hq])
        kk, vv = turn(x[:, Hq:Hq + Hkv]), x[:, Hq + Hkv:].double()
        for i in range(n):
            page, slot = int(table[b, (p0 + i) // P]), (p0 + i) % P
            want[layer, page, 0, :, slot] = kk[i]
            want[layer, page, 1, :, slot] = vv[i]
    # two products and a sum in fp32 (3 roundings of terms up to |a| + |b|),
    # then one rounding to the type
    big = 2 * float(qkv.double().abs().max())
    for got, ref in ((out, want_out), (pool, want)):
        err = (got.cpu().double() - ref).abs()
        tol = 3 * 2.0 ** -24 * big + UNIT[dtype] * (ref.abs() + 1e-6) * 1.0001
        assert (err <= tol).all(), float((err / tol).max())
    assert torch.equal(pool[layer, :, 1].cpu().double(), want[layer, :, 1])
    assert (pool[0] == 9).all()
    # in place: the same bits
    B.np_kv_append(shape, layer, batch, table.to(DEV), B.make_qkv(q, k, v, q), rot, pool, ws)
    served = torch.zeros(T, dtype=torch.bool)
    for b, (p0, n) in enumerate(rows):
        served[cu[b]:cu[b + 1]] = p0 >= 0
    assert torch.equal(dev[:, :Hq].cpu()[served], out.cpu()[served])
    assert torch.equal(dev[:, Hq:].cpu(), qkv[:, Hq:])


def test_append_refuses_on_the_device():
    shape = B.make_kv_shape(1, 2, 1, 16, 16, 4, 2, 2, "f32")
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    x = torch.randn(2, 4, 16, device=DEV)
    qkv = B.make_qkv(x[:, :2], x[:, 2:3], x[:, 3:], torch.zeros(2, 2, 16, device=DEV))
    cos = torch.ones(10, 8, device=DEV)
    for pos, table, code in (([3, 31], [[0, 1], [2, -1]], B.NP_DEVERR_NOT_RESIDENT),
                             ([3, 12], [[0, 1], [2, 3]], B.NP_DEVERR_STATE),   # past max_pos
                             ([3, 32], [[0, 1], [2, 3]], B.NP_DEVERR_STATE)):  # past M P
        pool = torch.zeros(1, 4, 2, 1, 16, 16, device=DEV)
        ws.zero_()
        batch = B.make_kv_batch(2, 2, 1, 1000, i32(pos))
        rot = None if code == B.NP_DEVERR_NOT_RESIDENT else B.make_rotary(cos, cos, False)
        B.np_kv_append(shape, 0, batch, i32(sum(table, [])), qkv, rot, pool, ws)
        assert B.np_device_error(ws) == code
        assert (pool[0, 0, 0, 0, 3] != 0).any() and (pool[0, 1:] == 0).all()


def test_extend_and_fork_in_a_graph():
    """A captured step (extend, NULL lists) replayed: the device lengths go
    on from replay to replay."""
    c = Cache(3, 30, 5, 16)
    pos0 = torch.full((3,), -5, dtype=torch.int32, device=DEV)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream, capture_error_mode="thread_local"):
        B.np_kv_extend(c.shape, c.kv, c.pool, 3, None, None, pos0, c.ws, stream)
    for step in range(18):
        graph.replay()
        torch.cuda.synchronize()
        assert pos0.tolist() == c.m.extend(range(3), [1] * 3)
        c.same()
        if step == 8:  # eager work between replays
            c.free([1])
