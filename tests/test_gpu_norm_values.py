"""Norms of query and key heads that hold what is not finite, in plain caches and in
8-bit elements: x_d weight_d / sqrt(mean + eps) with a NaN among the x_d is NaN in all
of the head; with an infinity it is NaN there (infinity by infinity) and 0 elsewhere."""
import math

import pytest
import torch

from kv_ref import DT, rotate
from paper_2608_22643_amd import binding as B
from paper_2608_22643_amd.kvcache import rotary_tables
from test_gpu_kv_norm import Setup

pytestmark = pytest.mark.gpu

NAN, INF = math.nan, math.inf
# heads by what they hold beside zeros (or beside other numbers: rest)
HEADS = [dict(rest=True, at={3: NAN}), dict(rest=False, at={7: NAN}), dict(rest=True, at={5: INF}),
         dict(rest=False, at={0: -INF}), dict(rest=True, at={2: INF, 9: NAN}), dict(rest=True, at={1: INF, 15: -INF}),
         dict(rest=True, at={i: NAN for i in range(16)}), dict(rest=False, at={})]


def expected(x, weight, eps, cos, sin, pos, inter):
    x = x.double()
    mean = x.square().mean(-1, keepdim=True) + eps
    y = torch.where(mean == 0, torch.zeros_like(x), x / mean.sqrt())
    if weight is not None:
        y = y * weight.double()
    return y if cos is None else rotate(y, cos, sin, pos, inter)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,R,inter", [(64, 0, False), (64, 64, False), (128, 32, True), (256, 256, False), (16, 16, False)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("weights", [True, False])
def test_heads_that_are_not_finite(cache, dtype, D, R, inter, eps, weights):
    n = len(HEADS)
    s = Setup([(0, n), (3, 5)], 4, 2, D, 16, dtype, cache, seed=D + R)
    x = s.qkv.clone()
    for t, head in enumerate(HEADS):
        if not head["rest"]:
            x[t, :6] = 0
        for i, v in head["at"].items():
            x[t, :6, i] = v
    s.dev.copy_(x)
    cos, sin = rotary_tables(R, s.longest) if R else (None, None)
    s.append(eps, weights=weights, rotary=B.make_rotary(cos, sin, inter) if R else None)
    c, z = (cos.cpu(), sin.cpu()) if R else (None, None)
    keys, _ = s.read()
    for got, heads, w in ((s.q_out.cpu(), x[:, :4], s.wq), (keys, x[:, 4:6], s.wk)):
        want = expected(heads, w if weights else None, eps, c, z, s.pos, inter)
        bad = want.isnan()
        assert torch.equal(got.isnan(), bad), (got.isnan() != bad).nonzero()[:5]
        # what is finite beside an infinity is 0, and so is a head of zeros
        assert (got[:n][~bad[:n]] == 0).all() and (want[:n][~bad[:n]] == 0).all()
        # The heads of other tokens are what they are.  Of their largest value: 28 units of 2^-24 of |a c| + |b s| (as in
        # kv8_ref.norm_rotate), which is at most twice it, and the rounding to the type, at most eps / 2; of elements
        # 2^-4 of the rounded value besides, or 2^-10 of the scale, which is below 1/224 of it.
        off = (got[n:].double() - want[n:]).abs()
        size = want[n:].abs().amax(-1, keepdim=True)
        tol = (torch.finfo(DT[dtype]).eps / 2 + 64 * 2.0 ** -24) * size
        if cache == "e4m3" and heads.shape[1] == 2:
            tol = tol * (1 + 2.0 ** -4) + 2.0 ** -4 * want[n:].abs() + 2.0 ** -17 * size
        assert (off <= tol).all()
    assert B.np_device_error(s.ws) == 0
