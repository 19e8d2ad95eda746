"""One workspace for caches of several shapes: what has to last from call to
call (arrival counts, the zeros that stand in for missing pages) lies where no
call of any shape writes its scratch."""
import pytest
import torch

from paper_2608_22643_amd import binding as B
from test_gpu_attn import DEV, Setup

pytestmark = pytest.mark.gpu


class Planner:
    """A cache whose planners fill their scratch: thousands of pages given
    out, freed and moved."""

    def __init__(self, n_pages, ws):
        self.n = n_pages
        self.shape = B.make_kv_shape(1, 1, 1, 8, 16, n_pages, 4, n_pages, "f16")
        i32 = dict(dtype=torch.int32, device=DEV)
        self.t = [torch.empty(4, n_pages, **i32), torch.empty(4, **i32), torch.empty(n_pages, **i32)]
        self.kv = B.make_kv_state(*self.t)
        self.pool = torch.zeros(1, n_pages, 2, 1, 16, 8, dtype=torch.float16, device=DEV)
        self.ws = ws
        B.np_kv_reset(self.shape, self.kv, ws)

    def work(self):
        half = self.n // 2 - 8
        ids = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
        new = torch.tensor([16 * half, 16 * half - 3], dtype=torch.int32, device=DEV)
        pos0 = torch.empty(2, dtype=torch.int32, device=DEV)
        B.np_kv_extend(self.shape, self.kv, self.pool, 2, ids, new, pos0, self.ws)
        B.np_kv_fork(self.shape, self.kv, 1, ids[1:], ids[2:], None, self.ws)
        B.np_kv_extend(self.shape, self.kv, self.pool, 1, ids[2:], None, pos0, self.ws)
        B.np_kv_free(self.shape, self.kv, 1, ids, self.ws)
        moved = torch.empty(1, dtype=torch.int32, device=DEV)
        B.np_kv_compact(self.shape, self.kv, self.pool, moved, self.ws)
        assert int(moved) > 0
        B.np_kv_free(self.shape, self.kv, 2, ids[1:], self.ws)
        assert int((self.t[2] != 0).sum()) == 0


def setups(dtype):
    """Caches of different page counts, all with rows that are split: row
    blocks with a fixed split, even shares, tiles."""
    return [(Setup([(16000, 1)], 8, 1, 64, 16, dtype, seed=60, pages=1100), B.np_attn_decode),
            (Setup([(3000, 1), (20, 1), (6000, 1), (-1, 1)] * 8, 8, 4, 64, 16, dtype, seed=61, pages=9000),
             B.np_attn_decode),
            (Setup([(6000, 40), (0, 77)], 32, 4, 128, 64, dtype, seed=62, pages=300), B.np_attn_prompt)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_split_calls_of_several_shapes_in_turn(dtype):
    """Each call in turn with the others and with planners over one workspace
    gives the bits it gives with a workspace of its own."""
    runs = setups(dtype)
    alone = [s.run(call) for s, call in runs]
    for (s, call), out in zip(runs, alone):
        if s.T < 100:  # the row blocks; the others have tests of their own
            s.check(out)
    ws = torch.full((max(s.ws.numel() for s, _ in runs) + 4096 * 64,), 0x5A, dtype=torch.uint8, device=DEV)
    small, large = Planner(700, ws), Planner(7001, ws)  # the resets initialise it for every shape
    for s, _ in runs:
        s.ws = ws
    for turn in range(2):
        for (s, call), want in zip(runs, alone):
            assert torch.equal(s.run(call), want)
            large.work()
            assert torch.equal(s.run(call), want)
            small.work()
        for (s, call), want in zip(runs, alone):
            assert torch.equal(s.run(call), want)
    assert B.np_device_error(ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_missing_pages_read_zeros_whatever_ran_before(dtype):
    """The stand-in for a missing page is still zero after another shape's
    planners and partial sums."""
    s = Setup([(200, 1), (90, 1)], 4, 2, 64, 16, dtype, seed=63)
    s.table[0, 1] = -1
    want = s.run(B.np_attn_prompt)
    other = Setup([(16000, 1)], 8, 1, 64, 16, dtype, seed=64, pages=1100)
    s.ws = other.ws = torch.zeros(max(s.ws.numel(), other.ws.numel()) + 4096 * 64, dtype=torch.uint8, device=DEV)
    other.run(B.np_attn_decode)
    Planner(7001, s.ws).work()
    assert torch.equal(s.run(B.np_attn_prompt), want)
    assert s.error() == B.NP_DEVERR_NOT_RESIDENT
