"""np_attn_decode_shared against float64 attention, elementwise within the bound of
the decode (kv_ref.attention; what joining more parts adds is in its 32 roundings
beside the keys'): groups of all sizes, prefixes that end inside pages and steps,
windows, rows that are not served, bad leads, missing pages, large batches, both
kinds of cache, HIP graphs."""
import math

import pytest
import torch

from kv8_ref import page_bytes, quantise
from kv_ref import DT, attention, div_up
from paper_2608_22643_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = ["f32", "f16", "bf16"]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Setup:
    """groups: (prefix, [own tokens of each row]); own tokens -1: the row is not
    served.  A row's length is prefix + own; with own <= 0 it ends inside the
    prefix.  What no row may see is NaN."""

    def __init__(self, groups, Hq, Hkv, D, P, dtype, cache="same", seed=0, order=None):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.Hq, self.Hkv, self.D, self.P, self.dtype = Hq, Hkv, D, P, dtype
        self.lead, self.prefix, self.len, tables = [], [], [], []
        self.keys, self.values = [], []
        page, pages = 0, []
        for p, owns in groups:
            L = len(self.lead)
            head = self.data(g, p)
            for b, own in enumerate(owns):
                own = None if own == "none" else own
                ln = p + (own or 0)
                self.lead.append(L)
                self.prefix.append(p)
                self.len.append(ln if own is not None else 0)
                tail = self.data(g, max(own or 0, 0))
                k, v = (torch.cat((a[:, :max(ln, 0)], c), 1) for a, c in zip(head, tail))
                self.keys.append(k)
                self.values.append(v)
                # the lead holds all of the prefix's pages, the others share the whole ones
                table, have = [], max(ln, p) if b == 0 else ln
                full = torch.cat((head[0], tail[0]), 1), torch.cat((head[1], tail[1]), 1)
                for j in range(div_up(have, P)):
                    if b and (j + 1) * P <= p:
                        table.append(tables[L][j])
                    else:
                        pages.append([x[:, j * P:(j + 1) * P] for x in full])
                        table.append(page)
                        page += 1
                tables.append(table)
        n = len(self.lead)
        self.n, self.N = n, page + 2
        perm = torch.randperm(self.N, generator=g).tolist()
        self.M = max(max(map(len, tables)), 1) + 1
        self.table = torch.full((n, self.M), -1, dtype=torch.int32)
        for b, t in enumerate(tables):
            self.table[b, :len(t)] = torch.tensor([perm[x] for x in t], dtype=torch.int32)
        self.shape = B.make_kv_shape(1, Hq, Hkv, D, P, self.N, n, self.M, dtype, cache)
        e4m3 = cache == "e4m3"
        pool = torch.full(B.kv_pool_shape(self.shape), 255 if e4m3 else math.nan, dtype=torch.uint8 if e4m3 else dt)
        for i, kv in enumerate(pages):
            e = kv[0].shape[1]
            x = torch.full((2, Hkv, P, D), math.nan, dtype=torch.float64)
            x[:, :, :e] = torch.stack(kv).to(dt).double()
            if e4m3:
                byte, scale, _ = quantise(x, dtype)
                scale[:, :, e:] = 255
                pool[0, perm[i]] = page_bytes(byte, scale)
            else:
                pool[0, perm[i]] = x.to(dt)
        if e4m3:
            self.keys, self.values = ([quantise(x.to(dt).double(), dtype)[2] if x.shape[1] else x.double() for x in y]
                                      for y in (self.keys, self.values))
        self.q = torch.randn(n, Hq, D, generator=g).to(dt)
        # rows of the batch may name the sequences in another order
        self.pos = [x - 1 for x in self.len]
        self.pool, self.qd = pool.to(DEV), self.q.to(DEV)
        self.ws = torch.zeros(B.np_kv_workspace_size(self.shape), dtype=torch.uint8, device=DEV)
        self.scale, self.max_len = 1 / math.sqrt(D), max(max(self.len), 1)

    def data(self, g, n):
        dt = DT[self.dtype]
        return [torch.randn(self.Hkv, n, self.D, generator=g).to(dt) for _ in range(2)]

    def batch(self, **kw):
        a = dict(n_seq=self.n, n_tokens=self.n, max_tokens=1, max_len=self.max_len, pos0=i32(self.pos))
        return B.make_kv_batch(**dict(a, **kw))

    def bound(self):
        """A max_prefix that lets sharing look worth while, so that small cases take its kernels too."""
        row = self.D if self.shape.dtype & B.NP_KV_E4M3 else self.D * DT[self.dtype].itemsize
        return max(max(self.prefix), (32 + self.n) * 1000000 // max(1, (self.n - 1) * self.Hkv * 2 * row) + 1)

    def shared(self, lead=None, prefix=None, most=None):
        return B.make_kv_shared(i32(self.lead if lead is None else lead), i32(self.prefix if prefix is None else prefix),
                                self.bound() if most is None else most)

    def run(self, shared=None, window=0, batch=None, table=None, out=None, q=None):
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device=DEV) if out is None else out
        B.np_attn_decode_shared(self.shape, 0, batch or self.batch(), shared or self.shared(),
                                self.table.to(DEV) if table is None else table, self.qd if q is None else q, self.pool,
                                self.scale, window, out, self.ws)
        torch.cuda.synchronize()
        return out.cpu()

    def check(self, out, window=0, rows=None):
        for b in range(self.n) if rows is None else rows:
            if self.pos[b] < 0:
                assert (out[b] == 0).all(), b
                continue
            ln = self.len[b]
            ref, tol = attention(self.q[b:b + 1], self.keys[b][:, :ln], self.values[b][:, :ln], self.pos[b], self.scale,
                                 window, self.dtype)
            err = (out[b].double() - ref[0]).abs()
            assert (err <= tol[0]).all(), (b, ln, float(err.max()), float((err / tol[0]).max()))

    def error(self):
        return B.np_device_error(self.ws)


GROUPS = [
    [(100, [1, 1])],
    [(1, [1, 2, 3])],
    [(64, [1, 16, 17]), (33, [5]), (0, [4, 9]), (200, [40, 1, 7, 300])],
    [(500, [3, "none", 20]), (15, ["none", 1]), (129, ["none", "none"])],
    [(300, [1] * 40), (17, [2] * 3)],
]


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("groups", range(len(GROUPS)))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 32), (3, 3, 256, 64), (10, 2, 80, 16)])
def test_groups(cache, dtype, groups, Hq, Hkv, D, P):
    s = Setup(GROUPS[groups], Hq, Hkv, D, P, dtype, cache, seed=groups)
    out = s.run()
    s.check(out)
    assert torch.equal(out, s.run()) and s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 16, 50, 130, 1000])
def test_windows(dtype, window):
    s = Setup([(120, [1, 30, 200]), (300, [2, 5])], 4, 2, 64, 16, dtype, seed=7)
    s.check(s.run(window=window), window=window)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_inside_the_prefix(dtype):
    """Rows that end before the prefix does see no more of it."""
    s = Setup([(100, [-1, -60, 3, -99, 0, -37])], 4, 2, 64, 16, dtype, seed=8)
    out = s.run()
    s.check(out)
    assert s.error() == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (16, 1), (24, 1), (40, 8), (64, 2), (128, 1), (200, 1)])
def test_heads(cache, dtype, Hq, Hkv):
    """Groups of heads past a row block's 16 and a tile's 128 rows among them."""
    s = Setup([(90, [4, 1, 30]), (40, [1, 1])], Hq, Hkv, 32, 16, dtype, cache, seed=9)
    s.check(s.run())


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows(dtype):
    """More rows than a wave has lanes, groups across its ends, several tiles a group."""
    groups = [(40, [1 + i % 5 for i in range(70)]), (9, [2]), (70, [3] * 59), (33, [1] * 100), (5, [7, "none", 8])]
    s = Setup(groups, 4, 2, 32, 16, dtype, seed=10)
    s.check(s.run())
    assert s.error() == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_long_prefix_is_split_and_joined(cache, dtype):
    s = Setup([(20001, [1, 300, 5000]), (7000, [9, 1])], 4, 1, 64, 64, dtype, cache, seed=11)
    a = s.run()
    s.check(a)
    assert torch.equal(a, s.run())


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,p,Hq,Hkv,D,P,window", [
    (6, 20001, 16, 4, 64, 64, 0), (8, 20001, 16, 4, 64, 64, 19000), (11, 4200, 32, 16, 80, 16, 0),
    (5, 17000, 16, 4, 128, 32, 0), (3, 8200, 64, 8, 256, 128, 0)])
def test_two_row_blocks_side_by_side(cache, dtype, rows, p, Hq, Hkv, D, P, window):
    """Up to 32 query heads per key-value head behind long prefixes, the second row block partly filled."""
    if dtype == "f32" and D > 128:
        pytest.skip("fp32 has no blocks side by side")
    s = Setup([(p, [1 + 37 * i for i in range(rows)])], Hq, Hkv, D, P, dtype, cache, seed=rows)
    out = s.run(window=window)
    s.check(out, window=window, rows=[0, 1, rows - 1])
    assert torch.equal(out, s.run(window=window)) and s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_agrees_with_decode(dtype):
    """Without groups, and with every row a group of its own, within twice the bound of each."""
    s = Setup(GROUPS[2], 8, 2, 128, 16, dtype, seed=12)
    plain = torch.zeros_like(s.qd)
    B.np_attn_decode(s.shape, 0, s.batch(), s.table.to(DEV), s.qd, s.pool, s.scale, 0, plain, s.ws)
    s.check(plain.cpu())
    assert torch.equal(s.run(s.shared(most=0)), plain.cpu())
    s.check(s.run(s.shared(lead=list(range(s.n)))))
    assert s.error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lead,prefix,bad", [
    ([0, 0, 0, -1, 3], None, [3]),               # outside the batch
    ([0, 0, 0, 4, 4], None, [3]),                # behind the row
    ([0, 0, 1, 3, 3], None, [2]),                # of a row that does not name itself
    ([0, 1, 0, 3, 3], None, [2]),                # not next to each other
    ([0, 0, 0, 3, 1 << 30], None, [4]),
    (None, [-1, 100, 100, 70, 70], [0, 1, 2]),   # a prefix below 0
    (None, [100, 7, 9, 1 << 30, 70], [3, 4]),    # past max_prefix
])
def test_bad_leads(dtype, lead, prefix, bad):
    """Rows with a bad lead are computed by themselves, and the error bit is set."""
    s = Setup([(100, [1, 5, 30]), (70, [2, 9])], 4, 2, 64, 16, dtype, seed=13)
    out = s.run(s.shared(lead, prefix))
    s.check(out)
    assert bad and s.error() == B.NP_DEVERR_STATE


def test_bad_sequences():
    """A lead whose sequence is none: its rows are computed by themselves; it is not served."""
    s = Setup([(100, [1, 5, 30]), (70, [2, 9])], 4, 2, 64, 16, "f16", seed=14)
    out = s.run(batch=s.batch(seqs=i32([99, 1, 2, 3, 4])))
    assert (out[0] == 0).all()
    s.check(out, rows=[1, 2, 3, 4])
    assert s.error() == B.NP_DEVERR_STATE


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_missing_pages(cache, dtype):
    """A page that the lead's table does not name is visible to no row of the group; one of a row's own only to others."""
    s = Setup([(100, [1, 40, 30]), (70, [2, 9])], 4, 2, 64, 16, dtype, cache, seed=15)
    table = s.table.clone()
    table[0, 2] = -1          # positions 32 .. 47 of the first group
    table[2, 7] = s.N + 5     # 112 .. 127 of row 2
    out = s.run(table=table.to(DEV))
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    for b in range(5):
        keep = torch.arange(s.len[b])
        if b < 3:
            keep = keep[(keep < 32) | (keep >= 48)]
        if b == 2:
            keep = keep[(keep < 112) | (keep >= 128)]
        ref, tol = attention(s.q[b:b + 1], s.keys[b][:, keep], s.values[b][:, keep], len(keep) - 1, s.scale, 0, dtype)
        assert ((out[b].double() - ref[0]).abs() <= tol[0]).all(), b


def test_rows_name_their_sequences():
    """A batch of some of the rows, in another order of sequences."""
    s = Setup([(100, [1, 5, 30]), (70, [2, 9])], 4, 2, 64, 16, "bf16", seed=16)
    pick = [4, 3, 1, 2]  # the group of two, led by its second row; two of the three, without their first
    out = torch.zeros(4, 4, 64, dtype=torch.bfloat16, device=DEV)
    batch = B.make_kv_batch(4, 4, 1, s.max_len, i32([s.pos[b] for b in pick]), seqs=i32(pick))
    # row 1 of the first group has its own copy of the prefix's last page
    shared = B.make_kv_shared(i32([0, 0, 2, 2]), i32([70, 0, 100, 0]), 2 * s.bound())
    B.np_attn_decode_shared(s.shape, 0, batch, shared, s.table.to(DEV), s.qd[pick].contiguous(), s.pool, s.scale, 0, out,
                            s.ws)
    whole = torch.zeros_like(s.q)
    whole[pick] = out.cpu()
    s.check(whole, rows=pick)
    assert s.error() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_views_and_in_place(dtype):
    s = Setup(GROUPS[2], 4, 2, 64, 16, dtype, seed=17)
    plain = s.run()
    wide = torch.full((s.n, 9, 64), 3.0, dtype=DT[dtype], device=DEV)
    wide[:, 1:5] = s.qd
    s.run(q=wide[:, 1:5], out=wide[:, 1:5])
    assert torch.equal(wide[:, 1:5].cpu(), plain)
    assert (wide[:, 0] == 3).all() and (wide[:, 5:] == 3).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_values_that_are_not_finite(dtype):
    """A NaN key of the prefix makes its head NaN in every row of the group, an infinite one of a row in that row."""
    s = Setup([(100, [3, 40]), (70, [2, 9])], 2, 2, 64, 16, dtype, seed=18)
    s.pool[0, int(s.table[0, 1]), 0, 1, 5] = math.nan
    s.pool[0, int(s.table[3, 4]), 0, 0, 70 % 16 + 3] = math.inf
    out = s.run()
    assert out[:2, 1].isnan().all() and torch.isfinite(out[:2, 0]).all()
    assert torch.isfinite(out[2]).all() and torch.isfinite(out[3, 1]).all()
    # +-infinity by the query's signs: NaN where the score is +infinity or NaN, else that key has no weight
    assert out[3, 0].isnan().all() or torch.isfinite(out[3, 0]).all()


def test_batches_past_the_parts():
    """More query heads than have rows in the workspace: np_attn_decode's results."""
    s = Setup([(40, [1] * 500), (9, [3] * 20)], 64, 8, 16, 16, "f16", seed=19)
    assert s.n * s.Hq > 32768
    plain = torch.zeros_like(s.qd)
    B.np_attn_decode(s.shape, 0, s.batch(), s.table.to(DEV), s.qd, s.pool, s.scale, 0, plain, s.ws)
    assert torch.equal(s.run(), plain.cpu())


def test_batches_up_to_the_parts():
    """The most query heads whose parts fit: 512 rows of 64 heads."""
    s = Setup([(40, [1] * 300), (90, [3] * 212)], 64, 8, 16, 16, "f16", seed=20)
    s.check(s.run(), rows=[0, 1, 150, 299, 300, 400, 511])
    assert s.error() == 0


@pytest.mark.parametrize("loose", [False, True])
def test_bounds_only_bound(loose):
    """max_len and max_prefix far past what the rows have; as tight as they go, the keys are read row by row."""
    s = Setup(GROUPS[2], 8, 2, 64, 16, "bf16", seed=21)
    s.check(s.run(s.shared(most=1 << 20 if loose else 200), batch=s.batch(max_len=s.M * 16 if loose else s.max_len)))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_graph_replays(cache):
    """Replays with other positions, leads and prefixes than captured, between eager calls on the same workspace."""
    s = Setup([(200, [40, 9, 30]), (70, [20, 9])], 8, 2, 128, 16, "bf16", cache, seed=22)
    pos, lead, prefix, table = i32(s.pos), i32(s.lead), i32(s.prefix), s.table.to(DEV)
    out = torch.zeros_like(s.qd)
    batch, shared = s.batch(pos0=pos), B.make_kv_shared(lead, prefix, s.bound())

    def call(stream=None):
        B.np_attn_decode_shared(s.shape, 0, batch, shared, table, s.qd, s.pool, s.scale, 0, out, s.ws, stream)

    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call(side)
    full = list(s.len)
    for i, (ld, px) in enumerate([([0, 0, 0, 3, 3], [200, 0, 0, 70, 0]), ([0, 1, 1, 3, 4], [1, 150, 9, 8, 7]),
                                  ([0, 0, 0, 3, 3], [33, 1, 1, 70, 1]), ([0, 1, 2, 3, 4], [0] * 5)]):
        s.len = [x - i for x in full]
        s.pos = [x - 1 for x in s.len]
        pos.copy_(i32(s.pos))
        lead.copy_(i32(ld))
        prefix.copy_(i32(px))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        s.check(got.cpu())
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    assert s.error() == 0


def test_shapes_and_graphs_in_turn_on_one_workspace():
    """Shared calls of three shapes and caches, eager and captured, in turn over one workspace: each gives the bits it
    gives with a workspace of its own."""
    runs = [Setup([(3000, [40, 9, 30, 1]), (700, [20, 9])], 8, 2, 128, 16, "bf16", "e4m3", seed=23),
            Setup([(130, [1] * 70)], 32, 8, 64, 64, "f16", "same", seed=24),
            Setup([(500, [7, "none", 3])], 4, 4, 80, 32, "f32", "same", seed=25)]
    alone = [s.run() for s in runs]
    for s, out in zip(runs, alone):
        s.check(out)
    ws = torch.zeros(max(s.ws.numel() for s in runs), dtype=torch.uint8, device=DEV)
    graphs = []
    for s in runs:
        s.ws = ws
        out, table, batch, shared = torch.zeros_like(s.qd), s.table.to(DEV), s.batch(), s.shared()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            B.np_attn_decode_shared(s.shape, 0, batch, shared, table, s.qd, s.pool, s.scale, 0, out, ws, side)
        graphs.append((graph, out, table, batch, shared))
    for turn in range(3):
        for (graph, out, *_), s, want in zip(graphs, runs, alone):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), want)
            for other, w in zip(runs, alone):
                assert torch.equal(other.run(), w)
    assert B.np_device_error(ws) == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 20, 150])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(16, 16, 64, 16), (32, 8, 128, 32), (40, 8, 80, 16), (16, 16, 256, 64),
                                        (24, 24, 16, 16)])
def test_many_rows_with_few_keys_of_their_own(cache, dtype, window, Hq, Hkv, D, P):
    """More blocks of own keys than workgroups: a wave each, up to 256 keys; rows with more, with none and
    not served, and inside the prefix, beside them."""
    owns = [1, 16, 17, 33, 127, 128, 129, 255, 256, 257, 300, "none", 0, -3, 2, 60, 100, 7]
    groups = [(90, owns * 2), (33, [5, "none", 9]), (0, owns[:7]), (17, [1] * 23)]
    s = Setup(groups, Hq, Hkv, D, P, dtype, cache, seed=26)
    assert s.n * Hkv > 512
    out = s.run(window=window)
    s.check(out, window=window, rows=range(30 if D > 128 else s.n))
    assert s.error() == 0
    assert torch.equal(out, s.run(window=window))


def test_a_missing_page_of_own_keys_that_a_wave_has():
    s = Setup([(70, [90, 30] + [40] * 40)], 16, 16, 64, 16, "bf16", seed=27)
    clean = s.run()
    table = s.table.clone()
    table[0, 6] = -1  # positions 96 .. 111 of row 0
    out = s.run(table=table.to(DEV))
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    assert torch.equal(out[1:], clean[1:])
    at = torch.cat((torch.arange(96), torch.arange(112, 160)))
    ref, tol = attention(s.q[:1], s.keys[0][:, at], s.values[0][:, at], len(at) - 1, s.scale, 0, "bf16")
    assert ((out[0].double() - ref[0]).abs() <= tol[0]).all()
