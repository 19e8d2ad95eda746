"""Batches of many ragged rows (more than a wave, more than a workgroup) and
batches with bad rows: append and attention serve the same rows."""
import random

import pytest
import torch

from kv_ref import DT, UNIT, rotate
from paper_2608_22643_amd import binding as B
from test_gpu_attn import DEV, Setup
from test_gpu_attn_tiles import run as run_tiles, widen
from test_gpu_kv import Cache, i32

pytestmark = pytest.mark.gpu


class Append:
    """np_kv_append of random tokens for rows (p0, n) into a pool of 9s."""

    def __init__(self, rows, cu, T, dtype="f16", Hq=3, Hkv=1, D=24, P=16, M=4, R=0):
        g = torch.Generator().manual_seed(len(rows))
        self.rows, self.P, self.Hq, self.Hkv, self.dtype = rows, P, Hq, Hkv, dtype
        S = len(rows)
        N = S * M
        self.table = torch.randperm(N, generator=g).int().view(S, M)
        self.qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(DT[dtype])
        dev = self.qkv.to(DEV)
        self.pool = torch.full((1, N, 2, Hkv, P, D), 9.0, dtype=DT[dtype], device=DEV)
        self.out = torch.full((T, Hq, D), 9.0, dtype=DT[dtype], device=DEV)
        self.cos = self.sin = rot = None
        if R:
            ang = torch.rand(M * P, R // 2, generator=g, dtype=torch.float64) * 6.3
            self.cos, self.sin = ang.cos().float(), ang.sin().float()
            rot = B.make_rotary(self.cos.to(DEV), self.sin.to(DEV), False)
        shape = B.make_kv_shape(1, Hq, Hkv, D, P, N, S, M, dtype)
        ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
        batch = B.make_kv_batch(S, T, 64, M * P, i32(p0 for p0, _ in rows), cu_tokens=i32(cu))
        B.np_kv_append(shape, 0, batch, self.table.to(DEV),
                       B.make_qkv(dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], self.out), rot, self.pool, ws)
        self.error = B.np_device_error(ws)

    def check(self, spans):
        """spans: row -> its first token; all other slots and outputs stay."""
        Hq, Hkv = self.Hq, self.Hkv
        want = torch.full(tuple(self.pool.shape), 9.0, dtype=torch.float64)
        want_out = torch.full(tuple(self.out.shape), 9.0, dtype=torch.float64)
        for b, begin in spans.items():
            p0, n = self.rows[b]
            x, pos = self.qkv[begin:begin + n], torch.arange(p0, p0 + n)
            turn = (lambda y: rotate(y, self.cos, self.sin, pos, False)) if self.cos is not None else torch.Tensor.double
            want_out[begin:begin + n] = turn(x[:, :Hq])
            kk, vv = turn(x[:, Hq:Hq + Hkv]), x[:, Hq + Hkv:].double()
            for i in range(n):
                page, slot = int(self.table[b, (p0 + i) // self.P]), (p0 + i) % self.P
                want[0, page, 0, :, slot], want[0, page, 1, :, slot] = kk[i], vv[i]
        # fp32 products and sums, then one rounding to the type
        big = 2 * float(self.qkv.double().abs().max())
        for got, ref in ((self.out, want_out), (self.pool, want)):
            tol = 0.0 if self.cos is None else 3 * 2.0 ** -24 * big + UNIT[self.dtype] * (ref.abs() + 1e-6) * 1.0001
            assert ((got.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("cu,good", [([0, 1000, 49, 61], {2: 49}), ([0, 40, 61, 1 << 30], {0: 0, 1: 40}),
                                     ([-7, 5, 45, 61], {1: 5, 2: 45}), ([0, 40, 20, 61], {0: 0}),
                                     ([0, 40, 61, 60], {0: 0, 1: 40})])
def test_append_leaves_out_bad_rows_only(cu, good):
    """A row whose cu_tokens are bad has no tokens; the others are appended
    as the attention calls serve them."""
    rows = [(3, b - a) if i in good else (3, 0) for i, (a, b) in enumerate(zip(cu, cu[1:]))]
    if cu == [0, 40, 20, 61]:  # row 2 claims tokens 20 .. 39 too: they are row 0's, 40 .. 60 its own
        a = Append([(3, 40), (3, 0), (0, 41)], cu, 61)
        assert a.error == B.NP_DEVERR_STATE
        shifted = Append([(3, 40), (3, 0), (20, 21)], [0, 40, 40, 61], 61)
        assert torch.equal(a.out, shifted.out) and torch.equal(a.pool, shifted.pool)
        return
    a = Append(rows, cu, 61)
    assert a.error == B.NP_DEVERR_STATE
    a.check(good)


@pytest.mark.parametrize("dtype,R", [("f32", 16), ("bf16", 0), ("f16", 16)])
@pytest.mark.parametrize("n", [64, 65, 130, 1500])
def test_append_of_many_rows(n, dtype, R):
    rng = random.Random(n)
    rows = [(rng.randint(0, 40), rng.choice([0, 0, 1, 1, 2, 7])) for _ in range(n)]
    for i in (0, 63, n - 2):
        rows[i] = (rows[i][0], 0)
    rows[-1] = (5, 3)
    cu = [0]
    for _, k in rows:
        cu.append(cu[-1] + k)
    a = Append(rows, cu, cu[-1], dtype, R=R)
    assert a.error == 0
    a.check({b: cu[b] for b in range(n)})


def many(n, seed):
    rng = random.Random(seed)
    rows = [(rng.choice([0, 0, rng.randint(0, 300)]), rng.choice([0, 1, 2, 5, rng.randint(0, 40)])) for _ in range(n)]
    rows[0], rows[63], rows[n // 2], rows[-1] = (7, 0), (0, 33), (-1, 4), (150, 60)
    return rows


@pytest.mark.parametrize("kernel,dtype", [("rows", "f32"), ("rows", "f16"), ("tiles", "f16"), ("tiles", "bf16")])
@pytest.mark.parametrize("n", [65, 100, 200])
@pytest.mark.parametrize("window", [0, 50])
def test_prompts_of_many_rows(kernel, dtype, n, window):
    s = Setup(many(n, n), 4, 2, 64, 16, dtype, seed=80)
    if kernel == "tiles":
        if window:  # a window bounds the keys of a call: more heads take their place
            heads = 11_000_000 // (s.T * (window + 48)) + 1
            s = Setup(many(n, n), heads + -heads % 2, 2, 64, 16, dtype, seed=80)
            out = run_tiles(s, window=window)
            pick = [b for b in range(n) if b % 9 == 0 or b in (63, 64, n // 2, n - 1)]
            s.check(out, window=window, rows=pick[:14])
        else:
            s.check(run_tiles(widen(s)))
    else:
        s.check(s.run(B.np_attn_prompt, window=window), window=window)
    assert s.error() == 0


@pytest.mark.parametrize("kernel,dtype", [("rows", "f32"), ("tiles", "f16")])
def test_prompts_of_many_rows_with_bad_ones(kernel, dtype):
    """Bad rows among a hundred: reported, the others served."""
    s = Setup(many(100, 5), 4, 2, 64, 16, dtype, seed=81)
    if kernel == "tiles":
        widen(s)
    s.cu[70] = s.T + 9  # rows 69 and 70
    s.pos0[99] = 1 << 29
    out = run_tiles(s) if kernel == "tiles" else s.run(B.np_attn_prompt)
    assert s.error() == B.NP_DEVERR_STATE
    s.check(out, rows=[b for b in range(99) if b not in (69, 70)])
    assert (out[s.cu_host[99]:] == 0).all()


def test_planners_of_more_rows_than_threads():
    """2100 sequences extended, forked and freed in single calls."""
    rng = random.Random(9)
    c = Cache(4096, 9000, 3, 16)
    seqs = rng.sample(range(4096), 2100)
    c.extend(seqs, [rng.choice([0, 1, 15, 16, 17, 40]) for _ in seqs])
    rest = [s for s in range(4096) if s not in set(seqs)]
    src = [rng.choice(seqs) for _ in rest]
    c.fork(src, rest, [rng.randint(0, c.m.len[s]) for s in src])
    c.extend(rng.sample(range(4096), 4096), [1] * 4096)
    c.free(rng.sample(range(4096), 3000))
    c.compact()
    c.extend(rng.sample(range(4096), 1500), [rng.randint(0, 3) for _ in range(1500)])
    assert c.error() in (0, B.NP_DEVERR_OVERFLOW)
