"""np_attn_decode over many rows of few keys, where a wave has a block of a row to
itself: against float64 elementwise, over plain caches and 8-bit elements, at the
borders of the rule that chooses it, with what may go wrong in a row kept to it."""
import pytest
import torch

import test_gpu_attn
import test_gpu_attn8
from kv_ref import DT, attention
from paper_2608_22643_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SETUP = {"same": test_gpu_attn.Setup, "e4m3": test_gpu_attn8.Setup}
DTYPES = ["f32", "f16", "bf16"]
LENGTHS = (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256)


def rows_of(n, most=256):
    """n rows of many lengths up to `most`, the first the longest, some not served."""
    return [(most - 1, 1)] + [(-1 if i % 11 == 5 else min(LENGTHS[i % len(LENGTHS)], most) - 1, 1) for i in range(1, n)]


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,Hq,Hkv,D,P", [(49, 16, 16, 64, 16), (97, 32, 8, 128, 32), (25, 32, 32, 256, 64),
                                          (33, 24, 24, 80, 16), (40, 40, 20, 16, 128), (26, 32, 32, 208, 256),
                                          (100, 136, 8, 48, 16), (400, 20, 1, 96, 16)])
def test_lengths_and_heads(cache, dtype, n, Hq, Hkv, D, P):
    """More than 768 blocks: one head a group, several, and more than the 16 of a block."""
    s = SETUP[cache](rows_of(n), Hq, Hkv, D, P, dtype, seed=90)
    out = s.run(B.np_attn_decode)
    s.check(out, rows=range(min(n, 60)))
    assert all((out[b] == 0).all() for b, (p0, _) in enumerate(s.rows) if p0 < 0)
    assert s.error() == 0
    assert torch.equal(out, s.run(B.np_attn_decode))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("most,n", [(256, 48), (257, 49), (128, 97), (128, 96), (1, 800)])
def test_borders_of_the_rule(cache, dtype, most, n):
    """768 blocks and one row more, 256 keys and one more, the smallest rows."""
    s = SETUP[cache](rows_of(n, most), 16, 16 if most > 128 else 8, 64, 16, dtype, seed=91)
    s.check(s.run(B.np_attn_decode), rows=range(min(n, 50)))
    assert s.error() == 0


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 7, 33, 100, 208, 5000])
def test_windows(cache, dtype, window):
    """Far rows with a window: few keys of each."""
    rows = [(p, 1) for p in (0, 6, 120, 999, 511, 512, 300, 47)] * 13
    s = SETUP[cache](rows, 8, 8, 64, 32, dtype, seed=92)
    s.check(s.run(B.np_attn_decode, window=window), window=window, rows=range(16))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_views_and_in_place(cache, dtype):
    s = SETUP[cache](rows_of(70), 24, 12, 64, 16, dtype, seed=93)
    plain = s.run(B.np_attn_decode)
    wide = torch.full((s.T, 29, 64), 3.0, dtype=DT[dtype], device=DEV)
    wide[:, 1:25] = s.qd
    s.run(B.np_attn_decode, q=wide[:, 1:25], out=wide[:, 1:25])
    assert torch.equal(wide[:, 1:25].cpu(), plain)
    assert (wide[:, 0] == 3).all() and (wide[:, 25:] == 3).all()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [-1, 1 << 20])
def test_missing_pages_and_bad_rows(cache, dtype, bad):
    """A missing page costs its keys; a position past max_len, and a sequence there is none of, their rows."""
    s = SETUP[cache](rows_of(60), 16, 16, 64, 16, dtype, seed=94)
    clean = s.run(B.np_attn_decode)
    s.table[0, 2] = bad  # positions 32 .. 47 of row 0
    out = s.run(B.np_attn_decode)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    assert torch.equal(out[1:], clean[1:])
    at = torch.cat((torch.arange(32), torch.arange(48, 256)))
    ref, tol = attention(s.q[:1], s.keys[0][:, at], s.values[0][:, at], len(at) - 1, s.scale, 0, dtype)
    assert ((out[0].double() - ref[0]).abs() <= tol[0]).all()
    s.ws[:256].zero_()
    seqs = torch.arange(60, dtype=torch.int32, device=DEV)
    seqs[7] = 60
    s.pos0[3] = 256
    out = s.run(B.np_attn_decode, batch=s.batch(cu=False, seqs=seqs))
    assert s.error() & B.NP_DEVERR_STATE
    keep = [b for b in range(60) if b not in (0, 3, 7)]
    assert torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_that_are_not_finite(dtype):
    """A NaN query, key or value, and an infinite score: the heads that see it and no others."""
    s = SETUP["same"](rows_of(60), 32, 16, 64, 16, dtype, seed=95)
    clean = s.run(B.np_attn_decode)
    page = [int(s.table[b, 0]) for b in range(60)]
    s.qd[1, 5] = float("nan")
    s.pool[0, page[2], 0, 3, 1] = float("nan")  # a key that row 2's heads 6 and 7 see
    s.pool[0, page[8], 1, 4, 0, 9] = float("nan")  # one value: a column of heads 8 and 9 of row 8
    s.pool[0, page[9], 0, 0, 0] = float("inf")  # scores of row 9's heads 0 and 1: infinite or NaN
    out = s.run(B.np_attn_decode)
    seen = torch.zeros_like(out, dtype=torch.bool)
    seen[1, 5] = seen[2, 6:8] = True
    seen[8, 8:10, 9] = True
    assert out[seen].isnan().all()
    seen[9, 0:2] = True
    assert torch.equal(out[~seen], clean[~seen])


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_graph_replays(cache):
    s = SETUP[cache](rows_of(50), 16, 16, 128, 16, "bf16", seed=96)
    out = torch.zeros_like(s.qd)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    batch = s.batch(cu=False)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.np_attn_decode(s.shape, 0, batch, s.table, s.qd, s.pool, s.scale, 0, out, s.ws, side)
    g = torch.Generator().manual_seed(97)
    for i in range(4):
        s.qd.copy_(torch.randn(s.q.shape, generator=g).to(s.q.dtype))
        s.pos0.copy_(torch.tensor([max(p - 3 * i, -1) for p, _ in s.rows], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got.cpu(), s.run(B.np_attn_decode, batch=batch))
