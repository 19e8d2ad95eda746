"""np_attn_decode_shared with a window: shared keys that no row of a group sees are left
out, whatever the lengths of the groups and rows; batches large enough to take its
kernels (sharing saves at most a window of the prefix)."""
import pytest
import torch

from paper_2608_22643_amd import binding as B
from test_gpu_attn_shared import Setup

pytestmark = pytest.mark.gpu


def shares(s, window):
    """Whether the bytes that sharing can save reach what the call asks for."""
    row = s.D * (1 if s.shape.dtype & B.NP_KV_E4M3 else s.q.element_size())
    return (s.n - 1) * min(max(s.prefix), window) * s.Hkv * 2 * row >= (32 + s.n) * 1500000


CASES = [
    # groups, Hq, Hkv, D, P, windows
    ([(700, [1, 30, 200, "none", 9, 350] * 5), (90, [3, 40]), (1500, [2, 9, 900, 1400])], 64, 64, 64, 16, (150, 333, 1000)),
    ([(1100, [1 + 7 * (i % 40) for i in range(70)]), (500, [5, 600, -100, -499])], 64, 16, 128, 64, (130, 1024, 1300)),
    ([(640, [64] * 9), (640, [1, 2, 3, 400])], 512, 128, 64, 16, (200, 640, 641)),
    ([(900, ["none", 10, 20, "none"] * 8), (50, ["none"] * 3)], 64, 64, 80, 32, (200, 900)),
]


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_windows_of_groups(cache, dtype, case):
    groups, Hq, Hkv, D, P, windows = CASES[case]
    s = Setup(groups, Hq, Hkv, D, P, dtype, cache, seed=40 + case)
    rows = sorted({0, 1, 2, 3, 5, s.n - 4, s.n - 3, s.n - 2, s.n - 1, min(63, s.n - 1), min(64, s.n - 1)})
    for window in windows:
        out = s.run(window=window)
        s.check(out, window=window, rows=rows)
        assert torch.equal(out, s.run(window=window)) and s.error() == 0
        s.check(out, window=window, rows=[b for b in range(s.n) if s.pos[b] < 0])
    assert any(shares(s, w) for w in windows)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_window_as_long_as_everything(dtype):
    """The same bits as without one: nothing is left out."""
    s = Setup([(1200, [1, 300, 20] * 4), (700, [9, 2])], 32, 32, 64, 16, dtype, seed=50)
    assert shares(s, s.max_len)
    assert torch.equal(s.run(window=s.max_len), s.run())


def test_what_is_left_out_may_be_anything():
    """NaN in keys and values of the prefix before all windows reaches nothing; 200 rows of one group, past the lanes
    of a wave."""
    s = Setup([(600, [1 + i % 50 for i in range(200)])], 32, 32, 64, 16, "bf16", seed=51)
    window = 300
    assert shares(s, window)
    want = s.run(window=window)
    s.check(want, window=window, rows=[0, 63, 64, 127, 199])
    first = min(s.len) - window  # the first key that a row sees; steps of 128 and pages of 16 before it
    for page in range(first // 128 * 128 // 16):
        s.pool[0, int(s.table[0, page])] = float("nan")
    assert torch.equal(s.run(window=window), want) and s.error() == 0
