"""Values that are not finite, in row blocks and in tiles: they reach the
tokens and heads that see them and no others."""
import pytest
import torch

from kv_ref import attention
from paper_2608_22643_amd import binding as B
from test_gpu_attn import Setup
from test_gpu_attn_tiles import run as run_tiles, widen

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def setup(rows, kernel, dtype, seed, Hq=4, Hkv=2):
    s = Setup(rows, Hq, Hkv, 64, 16, dtype, seed=seed)
    return widen(s) if kernel == "tiles" else s


def run(s, kernel, **kw):
    return run_tiles(s, **kw) if kernel == "tiles" else s.run(B.np_attn_prompt, **kw)


KINDS = [("rows", "f32"), ("rows", "bf16"), ("tiles", "f16"), ("tiles", "bf16")]


@pytest.mark.parametrize("kernel,dtype", KINDS)
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_missing_page_beside_queries_that_are_not_finite(kernel, dtype, value, in_place):
    """Head 0 of the row's first token is not finite and a page is missing:
    every other token and head is what it is without that page's keys."""
    s = setup([(150, 100), (0, 20)], kernel, dtype, 70)
    s.table[0, 1] = s.N + 5  # keys 16..31 of row 0
    s.qd[0, 0] = value
    out = run(s, kernel, out=s.qd if in_place else None)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
    s.check(out, rows=[1])
    keep = [j for j in range(250) if not 16 <= j < 32]
    for i in range(100):
        vis = [j for j in keep if j <= 150 + i]
        ref, tol = attention(s.q[i:i + 1], s.keys[0][:, vis], s.values[0][:, vis], len(vis) - 1, s.scale, 0, dtype)
        ok = (out[i:i + 1].double() - ref).abs() <= tol
        assert ok[:, 1 if i == 0 else 0:].all(), i
    assert out[0, 0].isnan().all()


@pytest.mark.parametrize("kernel,dtype", KINDS)
@pytest.mark.parametrize("rows", [[(0, 90), (200, 7)], [(5000, 33), (0, 3)]])
def test_scores_that_are_not_finite(kernel, dtype, rows):
    """A NaN query: its head of its token.  A NaN key: the tokens that see it,
    in the heads of its group.  An infinite score: NaN, as inf - inf is."""
    s = setup(rows, kernel, dtype, 71)
    p0, n = rows[0]
    clean = run(s, kernel)
    s.check(clean)
    q = s.qd.clone()
    q[2, 1] = NAN
    out = run(s, kernel, q=q)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    bad[2, 1] = True
    assert torch.equal(out.isnan().all(-1), bad) and torch.equal(out.isnan().any(-1), bad)
    assert torch.equal(out[~bad], clean[~bad])
    # key p0 + 20 of row 0, head 1
    key = p0 + 20
    page = int(s.table[0, key // s.P])
    s.pool[0, page, 1 - 1, 1, key % s.P, 3] = NAN
    out = run(s, kernel)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    bad[20:n, 2:] = True
    assert torch.equal(out.isnan().all(-1), bad) and torch.equal(out.isnan().any(-1), bad)
    assert torch.equal(out[~bad], clean[~bad])
    # the same key with one infinite element and queries of both signs there
    s.pool[0, page, 0, 1, key % s.P, 3] = INF
    q = s.qd.clone()
    q[:, :, 3] = q[:, :, 3].abs() + 0.5
    plus = run(s, kernel, q=q)
    assert torch.equal(plus.isnan().any(-1), bad) and torch.equal(plus.isnan().all(-1), bad)
    q[:, :, 3] *= -1
    minus = run(s, kernel, q=q)  # weight 0, and so is its value's share
    assert not minus.isnan().any()
    for h in (2, 3):
        for i in (20, n - 1):
            vis = [j for j in range(p0 + i + 1) if j != key]
            ref, tol = attention(q[i:i + 1, h:h + 1].cpu(), s.keys[0][1:, vis], s.values[0][1:, vis], len(vis) - 1,
                                 s.scale, 0, dtype)
            assert ((minus[i:i + 1, h:h + 1].double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("kernel,dtype", KINDS)
def test_scores_of_minus_infinity_alone(kernel, dtype):
    """Nothing left to weigh: zeros, for those tokens only."""
    s = setup([(0, 40), (30, 5)], kernel, dtype, 72)
    clean = run(s, kernel)
    for j in range(10):
        s.pool[0, int(s.table[0, j // s.P]), 0, :, j % s.P, 7] = -INF
    q = s.qd.clone()
    q[:, :, 7] = 1.0
    out = run(s, kernel, q=q)
    assert (out[:10] == 0).all()
    assert not out.isnan().any() and (out[10:40] != 0).any()
    same = s.run(B.np_attn_prompt, q=q) if kernel == "rows" else run(s, kernel, q=q)
    assert torch.equal(out, same)
    assert out.shape == clean.shape
