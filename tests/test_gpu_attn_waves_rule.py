"""np_attn_decode over many rows of few keys, on both sides of the numbers of blocks at
which even shares take over from a wave for each block: the same results within the
bound, the same bits from run to run."""
import pytest
import torch

import test_gpu_attn
import test_gpu_attn8
from paper_2608_22643_amd import binding as B
from test_gpu_attn_waves import rows_of

pytestmark = pytest.mark.gpu
SETUP = {"same": test_gpu_attn.Setup, "e4m3": test_gpu_attn8.Setup}


@pytest.mark.parametrize("dtype,cache,D", [("f32", "same", 64), ("f32", "same", 128), ("f32", "e4m3", 64), ("f16", "same", 128),
                                           ("bf16", "same", 112)])
@pytest.mark.parametrize("n", [64, 65, 83, 84, 102, 103, 116, 129])
def test_borders_by_blocks(dtype, cache, D, n):
    """16 blocks a row: 1024 to 2064 of them, between which 65, 80 and 90 in 100 of a round lie."""
    s = SETUP[cache](rows_of(n), 16, 16, D, 32, dtype, seed=98)
    out = s.run(B.np_attn_decode)
    s.check(out, rows=range(12))
    assert all((out[b] == 0).all() for b, (p0, _) in enumerate(s.rows) if p0 < 0)
    assert s.error() == 0 and torch.equal(out, s.run(B.np_attn_decode))


@pytest.mark.parametrize("most", [64, 65, 128, 192, 193])
def test_borders_by_keys(most):
    s = SETUP["same"](rows_of(70, most), 16, 16, 64, 16, "f32", seed=99)
    s.check(s.run(B.np_attn_decode), rows=range(20))
    assert s.error() == 0
