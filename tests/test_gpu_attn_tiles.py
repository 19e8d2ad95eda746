"""np_attn_prompt on batches large enough for its tile kernel (16-bit types),
against float64 attention within the bound of kv_ref.attention.  Which kernel
runs follows from host bounds alone, so the small batches here name a max_len
far above their lengths; the long ones reach the kernel by their own size and
have their keys split over workgroups."""
import pytest
import torch

from kv_ref import attention, div_up
from paper_2608_22643_amd import binding as B
from test_gpu_attn import DEV, PROMPTS, Setup

pytestmark = pytest.mark.gpu


def widen(s):
    """Room for as many positions as make the batch a large one."""
    s.max_len = 11_000_000 // (s.T * s.Hq) + 1
    M = max(s.M, div_up(s.max_len, s.P))
    s.table = torch.cat([s.table, torch.full((s.S, M - s.M), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    s.M = M
    s.shape = B.make_kv_shape(1, s.Hq, s.Hkv, s.D, s.P, s.N, s.S, s.M, s.dtype)
    return s


def run(s, **kw):
    return s.run(B.np_attn_prompt, batch=s.batch(max_tokens=s.T + 64), **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", range(len(PROMPTS)))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 32), (3, 3, 256, 64), (10, 2, 80, 16),
                                        (5, 1, 8, 128), (2, 2, 200, 256)])
def test_rows(dtype, rows, Hq, Hkv, D, P):
    s = widen(Setup(PROMPTS[rows], Hq, Hkv, D, P, dtype, seed=40))
    s.check(run(s))
    assert s.error() == 0


LONG = [(6000, 40), (0, 77), (-1, 5), (2991, 9), (0, 0), (130, 1)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(32, 4, 64, 16), (32, 4, 128, 64), (32, 32, 96, 32), (16, 2, 256, 128)])
def test_long_rows_are_split_and_joined(dtype, Hq, Hkv, D, P):
    """The same call again gives the same bits, and leaves no trace in the
    workspace for a third."""
    s = Setup(LONG, Hq, Hkv, D, P, dtype, seed=41)
    a = run(s)
    s.check(a)
    assert s.error() == 0
    assert torch.equal(a, run(s))
    assert torch.equal(a, run(s))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [2500, 3990])
def test_window_of_long_rows(dtype, window):
    s = Setup(LONG, 64, 4, 64, 16, dtype, seed=42)
    s.check(run(s, window=window), window=window)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [1, 33, 64, 150])
def test_small_windows(dtype, window):
    """A window bounds the keys of a call, so it takes many tokens."""
    rows = [(0, 700), (170, 41), (0, 10)]
    Hq = 11_000_000 // (751 * (window + 48)) + 1
    Hq += -Hq % 8
    if Hq > 1024:
        pytest.skip("more heads than a cache can have")
    s = Setup(rows, Hq, 8, 64, 16, dtype, seed=43)
    out = run(s, window=window)
    # every head's arithmetic is the same: a few of them, from each group
    pick = list(range(0, Hq, max(1, Hq // 8)))
    for b, (p0, n) in enumerate(rows):
        t = slice(s.cu_host[b], s.cu_host[b + 1])
        for h in pick:
            kv = h * 8 // Hq
            ref, tol = attention(s.q[t][:, h:h + 1], s.keys[b][kv:kv + 1], s.values[b][kv:kv + 1], p0, s.scale, window,
                                 dtype)
            assert ((out[t][:, h:h + 1].double() - ref).abs() <= tol).all(), (b, h)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales(scale):
    s = widen(Setup([(40, 1), (0, 150)], 2, 1, 64, 16, "bf16", seed=44))
    s.check(run(s, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [[(150, 100), (0, 20)], [(20, 7), (0, 3)]])
def test_a_missing_page_is_not_visible(dtype, rows):
    s = widen(Setup(rows, 4, 2, 64, 16, dtype, seed=45))
    s.table[0, 1] = s.N + 5  # keys 16..31 of row 0
    out = run(s)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    s.check(out, rows=[1])
    keep = [j for j in range(s.keys[0].shape[1]) if not 16 <= j < 32]
    p0, n = rows[0]
    for i in range(n):
        vis = [j for j in keep if j <= p0 + i]
        ref, tol = attention(s.q[i:i + 1], s.keys[0][:, vis], s.values[0][:, vis], len(vis) - 1, s.scale, 0, dtype)
        assert ((out[i:i + 1].double() - ref).abs() <= tol).all(), i


def test_missing_pages_of_a_split_row():
    """Whole parts of a row's keys without a page, their sums empty."""
    s = Setup([(6000, 40), (0, 77)], 32, 4, 64, 16, "f16", seed=46)
    s.table[0, 20:300] = -1  # keys 320..4799 of row 0
    out = run(s)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    s.check(out, rows=[1])
    keep = [j for j in range(6040) if not 320 <= j < 4800]
    for i in (0, 17, 39):
        vis = [j for j in keep if j <= 6000 + i]
        ref, tol = attention(s.q[i:i + 1], s.keys[0][:, vis], s.values[0][:, vis], len(vis) - 1, s.scale, 0, "f16")
        assert ((out[i:i + 1].double() - ref).abs() <= tol).all(), i


def test_bad_rows_are_reported_and_not_served():
    s = widen(Setup([(0, 40), (0, 9), (0, 12)], 4, 2, 64, 16, "f16", seed=47))
    seqs = torch.tensor([0, 77, 2], dtype=torch.int32, device=DEV)
    out = s.run(B.np_attn_prompt, batch=s.batch(max_tokens=1000, seqs=seqs))
    assert s.error() == B.NP_DEVERR_STATE
    assert (out[40:49] == 0).all()
    s.check(out, rows=[0, 2])
    s = widen(Setup([(0, 40), (0, 9), (0, 12)], 4, 2, 64, 16, "f16", seed=47))
    s.cu[1] = 1000
    out = run(s)  # rows 0 and 1 have no tokens then
    assert s.error() == B.NP_DEVERR_STATE
    s.check(out, rows=[2])
    assert (out[:49] == 7).all()


def test_strided_queries_and_outputs():
    s = widen(Setup([(0, 70), (33, 20)], 4, 2, 64, 16, "f16", seed=48))
    wide = torch.full((s.T, 8, 64), 3.0, dtype=torch.float16, device=DEV)
    q, out = wide[:, 2:6], torch.full((s.T, 6, 64), 7.0, dtype=torch.float16, device=DEV)
    q.copy_(s.qd)
    run(s, q=q, out=out[:, 1:5])
    s.check(out[:, 1:5].cpu())
    assert (out[:, 0] == 7).all() and (out[:, 5] == 7).all()
    run(s, q=q, out=q)  # in place
    s.check(q.cpu())
