"""Whole decoder layers over the paged cache: prompts packed, forked, extended
and decoded against float64 layers on the CPU."""
import math

import numpy as np
import pytest
import torch

from kv_ref import rotate
from paper_2608_22643_amd import kvcache
from paper_2608_22643_amd import workload as W

pytestmark = pytest.mark.gpu


def reference(net, x):
    """The layers over one sequence x [n][d], everything in float64."""
    cfg, hq, hk, hd = net.cfg, net.heads, net.kv_heads, net.head_dim
    x = x.double()
    n = x.shape[0]
    R = hd // 16 * 16
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    ang = torch.arange(n, dtype=torch.float64)[:, None] * f[None]
    cos, sin = ang.cos().float(), ang.sin().float()
    norm = lambda y: y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6)
    pos = torch.arange(n)
    hide = pos[None] > pos[:, None]
    if net.window:
        hide |= pos[None] <= pos[:, None] - net.window
    for layer in range(cfg.layers):
        qkv = (norm(x) @ net.wqkv[layer].cpu().double()).view(n, hq + 2 * hk, hd)
        q = rotate(qkv[:, :hq], cos, sin, pos, False)
        k = rotate(qkv[:, hq:hq + hk], cos, sin, pos, False).repeat_interleave(hq // hk, 1)
        v = qkv[:, hq + hk:].repeat_interleave(hq // hk, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(hd)
        p = torch.softmax(s.masked_fill(hide[None], -math.inf), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(n, hq * hd) @ net.wo[layer].cpu().double()
        rec = net.records[layer].cpu().double()
        d = cfg.d_model
        g, u = norm(x) @ rec[:, :d].T, norm(x) @ rec[:, d:2 * d].T
        a = torch.nn.functional.silu(g) * u if cfg.act == "swiglu" else g.clamp(min=0) * u
        x = x + a @ rec[:, 2 * d:]
    return x


# what float32 layers may be off by: a few hundred roundings of 2^-24 through
# sums of up to 1024 terms and two layers; 16-bit activations are rounded about
# ten times a layer, 2^-9 (bf16) or 2^-12 (fp16) each on average
TOL = {"f32": 2e-5, "f16": 1e-2, "bf16": 8e-2}


@pytest.mark.parametrize("dtype,act", [("f32", "relu"), ("f32", "swiglu"), ("f16", "relu"), ("bf16", "swiglu")])
@pytest.mark.parametrize("window", [0, 40])
def test_prompts_forks_and_decoding(dtype, act, window):
    cfg = W.get("tiny").with_(layers=2, wdtype=dtype, adtype=dtype, act=act)
    net = kvcache.DecoderLayers(cfg, 4, 2, max_seqs=5, max_len=160, page_size=16, window=window)
    cache = net.cache
    dt = kvcache.TORCH_DT[dtype]
    g = torch.Generator().manual_seed(1)
    tokens = {s: torch.randn(150, cfg.d_model, generator=g).to(dt) for s in range(3)}
    # the forks go their own way after 45 tokens of sequence 0 and all of 1
    tokens[3] = torch.cat((tokens[0][:45], torch.randn(60, cfg.d_model, generator=g).to(dt)))
    tokens[4] = torch.cat((tokens[1][:33], torch.randn(60, cfg.d_model, generator=g).to(dt)))
    done = {s: 0 for s in tokens}
    got = {s: [] for s in tokens}

    def run(seqs, n_new):
        x = torch.cat([tokens[s][done[s]:done[s] + n] for s, n in zip(seqs, n_new)]).to(net.device)
        batch = cache.extend(seqs, None if all(n == 1 for n in n_new) else n_new)
        y = net.step(x, batch).cpu()
        for s, n in zip(seqs, n_new):
            got[s].append(y[:n])
            y, done[s] = y[n:], done[s] + n

    run([0, 1, 2], [70, 33, 1])
    cache.fork([0, 1], [3, 4], [45, 33])
    for s, n in ((3, 45), (4, 33)):
        got[s].append(got[s - 3][0][:n])
        done[s] = n
    for _ in range(5):
        run([0, 1, 2, 3, 4], [1] * 5)
    run([3, 2], [30, 50])  # a prompt behind a cached one
    cache.free([0])
    cache.compact()
    for _ in range(3):
        run([4, 2, 3], [1, 1, 1])
    assert cache.device_error() == 0
    for s in tokens:
        y = torch.cat(got[s])
        ref = reference(net, tokens[s][:done[s]])
        assert y.shape == ref.shape
        err = (y.double() - ref).abs().max() / ref.abs().max()
        assert err <= TOL[dtype], (s, float(err))


def test_the_example_runs(capsys):
    kvcache.main(["--config", "tiny", "--prompt", "70", "--samples", "3", "--tokens", "5"])
    assert "samples x 5 tokens" in capsys.readouterr().out
