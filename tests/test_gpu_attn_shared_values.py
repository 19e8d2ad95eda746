"""np_attn_decode_shared over keys and values that are not finite: infinite keys by the
sign of their scores, keys that only some rows of a group see, and values of a prefix,
which stay with the group."""
import math

import pytest
import torch

from kv_ref import attention
from test_gpu_attn_shared import Setup

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "f16", "bf16"]


def place(s, b, pos):
    """(page, slot) of a position of row b."""
    return int(s.table[b, pos // s.P]), pos % s.P


def sharing(dtype, groups, seed):
    """Two key-value heads of 64, one query head each; every query's first element 1."""
    s = Setup(groups, 2, 2, 64, 16, dtype, seed=seed)
    s.q[:, :, 0] = 1
    s.qd[:, :, 0] = 1
    return s


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("sign", [1, -1])
def test_infinite_scores(dtype, where, sign):
    """One infinite element of a key, met by a query's 1: a score of +infinity makes the head NaN in the rows that see it,
    one of -infinity costs that key only."""
    s = sharing(dtype, [(100, [3, 40]), (70, [2, 9])], 60)
    clean = s.run()
    b, pos = (2, 13) if where == "prefix" else (3, 74)
    page, slot = place(s, b, pos)
    s.pool[0, page, 0, 0, slot, 0] = sign * math.inf
    out = s.run()
    rows = [2, 3] if where == "prefix" else [3]
    others = [r for r in range(4) if r not in rows]
    assert torch.equal(out[others], clean[others]) and torch.equal(out[:, 1], clean[:, 1])
    if sign > 0:
        assert out[rows, 0].isnan().all()
        return
    for r in rows:
        keep = torch.tensor([j for j in range(s.len[r]) if j != pos])
        ref, tol = attention(s.q[r:r + 1], s.keys[r][:, keep], s.values[r][:, keep], len(keep) - 1, s.scale, 0, dtype)
        assert ((out[r].double() - ref[0]).abs() <= tol[0])[0].all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_keys_that_some_rows_see(dtype, value):
    """A key of the prefix that is not finite, behind the end of one row: that row does not meet it."""
    s = sharing(dtype, [(100, [3, -60, 40]), (70, [2, 9])], 61)
    clean = s.run()
    page, slot = place(s, 0, 50)
    s.pool[0, page, 0, 0, slot] = value
    out = s.run()
    assert out[[0, 2], 0].isnan().all()
    assert torch.equal(out[[1, 3, 4]], clean[[1, 3, 4]]) and torch.equal(out[:, 1], clean[:, 1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_keys_behind_some_windows(dtype):
    """A NaN key that the window of one row of a group has passed; a batch that takes the shared kernels with a window."""
    s = Setup([(400, [1, 260] * 10), (300, [2, 9])], 64, 64, 64, 16, dtype, seed=62)
    window = 300
    assert (s.n - 1) * window * 64 * 2 * 128 >= (32 + s.n) * 1500000
    clean = s.run(window=window)
    pos = 320  # rows 0, 2, ...: positions 101 .. 400; rows 1, 3, ...: 360 .. 659
    page, slot = place(s, 0, pos)
    s.pool[0, page, 0, 5, slot] = math.nan
    out = s.run(window=window)
    see = list(range(0, 20, 2))
    rest = [r for r in range(s.n) if r not in see]
    assert out[see, 5].isnan().all()
    assert torch.equal(out[rest], clean[rest])
    out[:, 5] = clean[:, 5]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [2, 40])
def test_values_stay_with_the_group(cache, dtype, rows):
    """A NaN among the prefix's values: its column in every row of the group, and nothing else anywhere."""
    s = Setup([(60, [4, 1]), (100, [3 + i for i in range(rows)]), (70, [2, 9])], 4, 2, 64, 16, dtype, cache, seed=63)
    clean = s.run()
    page, slot = place(s, 2, 20)
    if cache == "e4m3":
        s.pool[0, page, 1, 1, slot * 64 + 7] = 127
    else:
        s.pool[0, page, 1, 1, slot, 7] = math.nan
    out = s.run()
    seen = torch.zeros_like(out, dtype=torch.bool)
    seen[2:2 + rows, 2:4, 7] = True
    assert out[seen].isnan().all() and torch.equal(out[~seen], clean[~seen])


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_that_some_rows_see(dtype):
    """Behind the end of one row of the group: NaN where it is seen; in the row that ends before, that column alone may
    have it; other groups do not."""
    s = Setup([(100, [3, -60, 40]), (70, [2, 9])], 2, 2, 64, 16, dtype, seed=64)
    clean = s.run()
    page, slot = place(s, 0, 50)
    s.pool[0, page, 1, 0, slot, 7] = math.nan
    out = s.run()
    assert out[[0, 2], 0, 7].isnan().all()
    touched = torch.zeros_like(out, dtype=torch.bool)
    touched[:3, 0, 7] = True
    assert torch.equal(out[~touched], clean[~touched])
