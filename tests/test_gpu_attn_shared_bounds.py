"""np_attn_decode_shared where what the host or the device says bounds nothing: prefixes
up to the largest number, past max_len and the table."""
import pytest
import torch

from paper_2608_22643_amd import binding as B
from test_gpu_attn_shared import Setup

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("dtype,cache", [("f32", "same"), ("f16", "same"), ("bf16", "e4m3")])
@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (8, 1, 128), (40, 1, 64), (2, 2, 256)])
@pytest.mark.parametrize("prefix", [300, 1 << 20, 1 << 30, MOST - 127, MOST - 126, MOST - 63, MOST])
def test_prefixes_past_all_positions(dtype, cache, Hq, Hkv, D, prefix):
    """Rows that all end inside a prefix of up to 2^31 - 1 positions see their own keys of it; a group with a true
    prefix beside them."""
    s = Setup([(300, [0, -5, -100, -299]), (70, [2, 9])], Hq, Hkv, D, 16, dtype, cache, seed=30)
    out = s.run(s.shared(prefix=[prefix, 0, 0, 0, 70, 0], most=MOST))
    s.check(out)
    assert s.error() == 0
    assert torch.equal(out, s.run(s.shared(prefix=[prefix, 0, 0, 0, 70, 0], most=MOST)))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("max_len", [0, 1, 40, 170])
def test_prefixes_past_max_len(dtype, max_len):
    """Rows at or past max_len are not served (and set the error bit); the others see what they saw."""
    s = Setup([(150, [-149, -111, 20, 21]), (33, [7])], 4, 2, 64, 16, dtype, seed=31)
    out = s.run(s.shared(prefix=[MOST, 0, 0, 0, 33], lead=[0, 0, 2, 2, 4], most=MOST), batch=s.batch(max_len=max_len))
    for b in range(s.n):
        if s.len[b] > max_len:
            s.pos[b] = -1
    s.check(out)
    assert s.error() == (B.NP_DEVERR_STATE if -1 in s.pos else 0)


def test_a_workspace_that_served_others():
    """The same after another shape's shared call has filled the plan and the parts."""
    a = Setup([(3000, [40, 9, 30, 1]), (700, [20, 9])], 32, 8, 128, 16, "bf16", seed=32)
    s = Setup([(300, [0, -5])], 2, 1, 64, 16, "f16", seed=33)
    ws = torch.zeros(max(a.ws.numel(), s.ws.numel()), dtype=torch.uint8, device="cuda:0")
    a.ws = s.ws = ws
    want = a.run()
    for prefix in (MOST, MOST - 100, 1 << 30):
        s.check(s.run(s.shared(prefix=[prefix, 0], most=MOST)))
        assert torch.equal(a.run(), want)
    assert s.error() == 0
