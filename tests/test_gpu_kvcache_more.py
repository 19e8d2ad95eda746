"""Whole decoder layers with normed heads, caches of 8-bit elements and shared
prefixes: prompts, forks and decoding against float64 layers on the CPU; the
cache's calls on streams of their own; refusals of KVCache."""
import math

import pytest
import torch

from kv8_ref import quantise
from kv_ref import rotate
from paper_2608_22643_amd import binding as B
from paper_2608_22643_amd import kvcache
from paper_2608_22643_amd import workload as W

pytestmark = pytest.mark.gpu
LOOSE = 60000  # a bound on prefixes from which sharing looks worth while, whatever the prefixes


def reference(net, x, e4m3):
    """The layers over one sequence x [n][d], everything in float64 but the cache's elements."""
    cfg, hq, hk, hd = net.cfg, net.heads, net.kv_heads, net.head_dim
    dt = kvcache.TORCH_DT[cfg.adtype]
    x = x.double()
    n = x.shape[0]
    f = 10000.0 ** (-torch.arange(0, hd // 16 * 16, 2, dtype=torch.float64) / (hd // 16 * 16))
    ang = torch.arange(n, dtype=torch.float64)[:, None] * f[None]
    cos, sin = ang.cos().float(), ang.sin().float()
    norm = lambda y, w=None: y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * (1 if w is None else w.cpu().double())
    pos = torch.arange(n)
    for layer in range(cfg.layers):
        qkv = (norm(x) @ net.wqkv[layer].cpu().double()).view(n, hq + 2 * hk, hd)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        if net.qk_norm[layer] is not None:
            wq, wk = net.qk_norm[layer]._kept
            q, k = norm(q, wq), norm(k, wk)
        q, k = rotate(q, cos, sin, pos, False), rotate(k, cos, sin, pos, False)
        if e4m3:
            k, v = (quantise(y.to(dt).double(), cfg.adtype)[2] for y in (k, v))
        k, v = k.repeat_interleave(hq // hk, 1), v.repeat_interleave(hq // hk, 1)
        s = (torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(hd)).masked_fill((pos[None] > pos[:, None])[None], -math.inf)
        x = x + torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v).reshape(n, hq * hd) @ net.wo[layer].cpu().double()
        rec, d = net.records[layer].cpu().double(), cfg.d_model
        g, u = norm(x) @ rec[:, :d].T, norm(x) @ rec[:, d:2 * d].T
        x = x + (g.clamp(min=0) * u) @ rec[:, 2 * d:]
    return x


# float32 layers: a few hundred roundings of 2^-24; 16-bit activations: about ten
# roundings a layer.  8-bit elements: a key or value next to the border of two
# elements may fall to either; that is one in (2^-4 / its error) values, a step is up
# to 2^-3 of a value, and a value is one of D in a score or one of many weights: a few
# such steps (f32), or three in a hundred values off by a step (bf16: an error of 2^-9)
TOL = {("f32", None): 2e-5, ("bf16", None): 8e-2, ("f32", "e4m3"): 5e-3, ("bf16", "e4m3"): 1.2e-1}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cache", [None, "e4m3"])
@pytest.mark.parametrize("qk_norm", [False, True])
def test_prompts_forks_and_shared_decoding(dtype, cache, qk_norm):
    cfg = W.get("tiny").with_(layers=2, wdtype=dtype, adtype=dtype)
    net = kvcache.DecoderLayers(cfg, 4, 2, max_seqs=6, max_len=160, page_size=16, cache=cache, qk_norm=qk_norm)
    kv, dt = net.cache, kvcache.TORCH_DT[dtype]
    g = torch.Generator().manual_seed(1)
    tokens = {s: torch.randn(150, cfg.d_model, generator=g).to(dt) for s in range(2)}
    shared_at = {2: (0, 45), 3: (0, 70), 4: (1, 33)}  # forks: of which sequence, how much of it
    for s, (a, n) in shared_at.items():
        tokens[s] = torch.cat((tokens[a][:n], torch.randn(60, cfg.d_model, generator=g).to(dt)))
    done, got = {s: 0 for s in tokens}, {s: [] for s in tokens}

    def run(seqs, n_new, shared=None):
        x = torch.cat([tokens[s][done[s]:done[s] + n] for s, n in zip(seqs, n_new)]).to(net.device)
        y = net.step(x, kv.extend(seqs, None if all(n == 1 for n in n_new) else n_new), shared).cpu()
        for s, n in zip(seqs, n_new):
            got[s].append(y[:n])
            y, done[s] = y[n:], done[s] + n

    run([0, 1], [70, 33])
    kv.fork([0, 0, 1], [2, 3, 4], [45, 70, 33])
    for s, (a, n) in shared_at.items():
        got[s].append(got[a][0][:n])
        done[s] = n
    # rows 0 .. 2: sequences 0, 2 and 3, 45 positions in common; then 4 and 1
    shared = kv.share([0, 0, 0, 3, 3], [45, 0, 0, 33, 0], LOOSE)
    for _ in range(6):
        run([0, 2, 3, 4, 1], [1] * 5, shared)
    kv.free([0])
    kv.compact()
    for _ in range(3):  # the first sequence is gone, its pages are still the others'
        run([3, 2, 4], [1] * 3, kv.share([0, 0, 2], [45, 0, 0], LOOSE))
    run([2, 3], [1, 1], kv.share([0, 0], [45, 45]))  # a tight bound: row by row
    assert kv.device_error() == 0
    for s in tokens:
        y, ref = torch.cat(got[s]), reference(net, tokens[s][:done[s]], cache == "e4m3")
        err = (y.double() - ref).abs().max() / ref.abs().max()
        assert y.shape == ref.shape and err <= TOL[dtype, cache], (s, float(err))


@pytest.mark.parametrize("cache", [None, "e4m3"])
def test_calls_from_another_stream(cache):
    """append, read and shared attention in order with the caller's stream, whose tensors may be dropped at once."""
    dev = "cuda:0"
    a = kvcache.KVCache(1, 4, 2, 64, "bf16", 3, 200, 16, rotary_dim=64, cache=cache, stream=torch.cuda.Stream())
    b = kvcache.KVCache(1, 4, 2, 64, "bf16", 3, 200, 16, rotary_dim=64, cache=cache)
    outs = []
    for kv, here in ((a, torch.cuda.Stream()), (b, torch.cuda.default_stream())):
        g = torch.Generator(device=dev).manual_seed(3)
        with torch.cuda.stream(here):
            def new(n, heads):
                return torch.randn(n, heads, 64, generator=g, device=dev).bfloat16()

            def step(batch, n, shared=None):
                norm = B.make_qk_norm(new(1, 1)[0, 0], new(1, 1)[0, 0], 1e-5)
                q = new(n, 4)
                kv.append(0, batch, q, new(n, 2), new(n, 2), q, norm)
                out = torch.zeros_like(q)
                kv.attend(0, batch, q, out, shared=shared)
                k, v = torch.zeros(n, 2, 64, dtype=q.dtype, device=dev), torch.zeros(n, 2, 64, dtype=q.dtype, device=dev)
                kv.read(0, batch, k, v)
                return torch.cat((out, k, v), 1)

            res = [step(kv.extend([0], [90]), 90)]
            kv.fork([0, 0], [1, 2])
            for i in range(4):
                shared = kv.share([0, 0, 0], torch.full((3,), 90, dtype=torch.int32, device=dev), LOOSE)
                res.append(step(kv.extend([0, 1, 2]), 3, shared))
                del shared
            outs.append(torch.cat(res).cpu())
        torch.cuda.synchronize()
        assert kv.device_error() == 0
    assert torch.equal(*outs)


def test_refusals():
    kv = kvcache.KVCache(1, 4, 2, 64, "f16", 3, 64, 16, cache="e4m3")
    assert kv.pool.dtype == torch.uint8 and kv.pool.shape == (1, 12, 2, 2, 16 * 65)
    with pytest.raises(ValueError):
        kvcache.KVCache(1, 4, 2, 64, "f16", 3, 64, 16, cache="int8")
    with pytest.raises(B.NPError):
        kvcache.KVCache(1, 4, 2, 72, "f16", 3, 64, 16, cache="e4m3")  # 72 is no multiple of 16
    with pytest.raises(ValueError):
        kv.share([0, 0], [5])
    q = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda:0")
    batch = kv.extend([0, 1])
    with pytest.raises(ValueError):
        kv.attend(0, batch, q, q, shared=kv.share([0], [5]))
    with pytest.raises(ValueError):
        kv.attend(0, kv.extend([0], [2]), q, q, shared=kv.share([0], [5]))
    assert kv.share([0, 0], [5, 9]).max_prefix == 9
    assert kv.share([], []).max_prefix == 0


@pytest.mark.parametrize("args", [[], ["--cache", "e4m3", "--qk-norm"]])
def test_the_example_runs(capsys, args):
    kvcache.main(["--config", "tiny", "--prompt", "70", "--samples", "3", "--tokens", "4", *args])
    assert "samples x 4 tokens" in capsys.readouterr().out
