"""The ends of the ranges the interface names: positions up to 2^30, groups of
1024 heads, 2^24 tokens, more than 2^28 query heads in row blocks."""
import pytest
import torch

from kv_ref import DT, attention
from paper_2608_22643_amd import binding as B
from test_gpu_kv import DEV, i32

pytestmark = pytest.mark.gpu
LAST = 1 << 30  # positions a sequence can have


class Far:
    """Rows (p0, n) at far positions behind a window: only the pages that the
    window reaches are there, the table's others name none."""

    def __init__(self, rows, window, Hq, Hkv, D, dtype, P=256):
        g = torch.Generator().manual_seed(len(rows))
        S, M = len(rows), LAST // P
        self.rows, self.window, self.dtype, self.Hq = rows, window, dtype, Hq
        table = torch.full((S, M), -1, dtype=torch.int32, device=DEV)
        self.first, self.k, self.v, used = [], [], [], 0
        blocks = []
        for b, (p0, n) in enumerate(rows):
            j0, j1 = max(0, p0 - window + 1) // P, (p0 + n - 1) // P + 1
            x = torch.randn(j1 - j0, 2, Hkv, P, D, generator=g).to(DT[dtype])
            table[b, j0:j1] = torch.arange(used, used + j1 - j0, dtype=torch.int32)
            used += j1 - j0
            blocks.append(x)
            self.first.append(j0 * P)
            kv = x.permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, D)
            self.k.append(kv[0])
            self.v.append(kv[1])
        self.pool = torch.cat(blocks)[None].contiguous().to(DEV)
        self.table = table
        self.shape = B.make_kv_shape(1, Hq, Hkv, D, P, used, S, M, dtype)
        self.ws = torch.zeros(B.np_kv_workspace_size(self.shape), dtype=torch.uint8, device=DEV)
        self.T = sum(n for _, n in rows)
        self.q = torch.randn(self.T, Hq, D, generator=g).to(DT[dtype])
        self.cu = [0]
        for _, n in rows:
            self.cu.append(self.cu[-1] + n)
        self.scale = D ** -0.5

    def run(self, call):
        cu = i32(self.cu) if call is B.np_attn_prompt else None
        batch = B.make_kv_batch(len(self.rows), self.T, max(n for _, n in self.rows), LAST,
                                i32(p0 for p0, _ in self.rows), cu_tokens=cu)
        out = torch.full(tuple(self.q.shape), 7.0, dtype=self.q.dtype, device=DEV)
        call(self.shape, 0, batch, self.table, self.q.to(DEV), self.pool, self.scale, self.window, out, self.ws)
        assert B.np_device_error(self.ws) == 0
        return out.cpu()

    def check(self, out, heads, tokens=None):
        for b, (p0, n) in enumerate(self.rows):
            for i in range(n) if tokens is None else sorted({0, n // 2, n - 1}):
                t, p = self.cu[b] + i, p0 + i - self.first[b]
                per = self.Hq // self.k[b].shape[0]
                for h in heads:
                    ref, tol = attention(self.q[t:t + 1, h:h + 1], self.k[b][h // per:h // per + 1],
                                         self.v[b][h // per:h // per + 1], p, self.scale, self.window, self.dtype)
                    assert ((out[t:t + 1, h:h + 1].double() - ref).abs() <= tol).all(), (b, i, h)
        assert not (out == 7.0).all(-1).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [[(LAST - 40, 40)], [(1 << 28, 40)], [(0, 60), (LAST - 300, 33), (LAST // 2, 1)],
                                  [((1 << 27) - 20, 40), (LAST - 40, 40), ((1 << 28) + 5, 7)]])
def test_tiles_at_far_positions_of_large_groups(dtype, rows):
    """1024 heads over one: a block of 128 rows is an eighth of a token, so
    blocks counted from position 0 pass 2^31 from 2^28 tokens on."""
    s = Far(rows, 256, 1024, 1, 64, dtype)
    assert s.T * 1024 * (256 + 48) > 10_000_000  # enough for the tiles
    s.check(s.run(B.np_attn_prompt), (0, 1, 127, 128, 500, 1023), tokens=3)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows", [[(LAST - 1, 1)], [(LAST - 1, 1), (0, 1), (LAST // 2 + 7, 1)] * 3])
@pytest.mark.parametrize("window", [100, 5000])
def test_decode_at_far_positions(dtype, rows, window):
    s = Far(rows, window, 8, 2, 64, dtype)
    s.check(s.run(B.np_attn_decode), (0, 3, 4, 7))


def test_small_prompts_at_far_positions():
    s = Far([(LAST - 9, 9), (1 << 29, 3), (0, 5)], 70, 8, 2, 64, "f32")
    s.check(s.run(B.np_attn_prompt), (0, 7))


def test_append_of_the_most_tokens():
    """2^24 tokens of one sequence, every slot."""
    T, P = 1 << 24, 256
    pages = T // P
    shape = B.make_kv_shape(1, 1, 1, 8, P, pages, 1, pages, "f16")
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    qkv = torch.randint(-30000, 30000, (T, 3, 8), dtype=torch.int16, device=DEV, generator=g).view(torch.float16)
    pool = torch.zeros(1, pages, 2, 1, P, 8, dtype=torch.float16, device=DEV)
    out = torch.zeros(T, 1, 8, dtype=torch.float16, device=DEV)
    batch = B.make_kv_batch(1, T, T, T, i32([0]), cu_tokens=i32([0, T]))
    B.np_kv_append(shape, 0, batch, i32(range(pages)), B.make_qkv(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], out), None, pool,
                   ws)
    assert B.np_device_error(ws) == 0
    bits = lambda x: x.reshape(T, 8).view(torch.int16)
    assert torch.equal(bits(out), bits(qkv[:, 0]))
    for kind in (0, 1):
        assert torch.equal(bits(pool[0, :, kind, 0]), bits(qkv[:, 1 + kind]))


def test_row_blocks_of_more_than_2_28_query_heads():
    """A window of one key: every head of a token gives the token's own value
    vector, exactly."""
    n, S, Hq, P = 4100, 64, 1024, 256
    T, M = n * S, 17
    assert T * Hq // 16 * 256 > 1 << 32  # threads of the launch
    shape = B.make_kv_shape(1, Hq, 1, 8, P, S * M, S, M, "f32")
    ws = torch.zeros(B.np_kv_workspace_size(shape), dtype=torch.uint8, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    pool = torch.randn(1, S * M, 2, 1, P, 8, device=DEV, generator=g)
    q = torch.zeros(T, Hq, 8, device=DEV)
    q[:, ::7] = 0.5
    out = torch.full((T, Hq, 8), 7.0, device=DEV)
    batch = B.make_kv_batch(S, T, n, n, i32([0] * S), cu_tokens=i32(range(0, T + 1, n)))
    B.np_attn_prompt(shape, 0, batch, i32(range(S * M)), q, pool, 0.3, 1, out, ws)
    assert B.np_device_error(ws) == 0
    values = pool[0, :, 1, 0].reshape(S, M * P, 8)[:, :n].reshape(T, 1, 8)
    for t in range(0, T, 16384):
        assert (out[t:t + 16384] == values[t:t + 16384]).all(), t
    del q, out, pool
    torch.cuda.empty_cache()
