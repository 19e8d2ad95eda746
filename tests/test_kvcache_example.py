"""The example's own check that samples of the same tokens agree, and the example with a
prompt long enough that it is read once for all samples."""
from types import SimpleNamespace

import pytest
import torch

from paper_2608_22643_amd import kvcache


def net(dtype="f32", heads=4, kv_heads=2, head_dim=64, cache=None):
    pool = torch.zeros(1, dtype=torch.uint8 if cache else kvcache.TORCH_DT[dtype])
    return SimpleNamespace(cfg=SimpleNamespace(adtype=dtype), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                           cache=SimpleNamespace(pool=pool))


@pytest.mark.parametrize("cache", [None, "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_samples_that_differ_are_seen(dtype, cache):
    """By one bit where their keys are cut alike, by more than roundings where they may not be."""
    dt = kvcache.TORCH_DT[dtype]
    x = torch.linspace(-1, 1, 256).to(dt).repeat(3, 1)
    kvcache.check_samples(net(dtype, cache=cache), x, 100, 116)
    one = x.clone()
    one[2, 7] = torch.nextafter(one[2, 7].float(), torch.tensor(2.0)).to(dt) if dtype == "f32" else one[2, 8]
    with pytest.raises(AssertionError):
        kvcache.check_samples(net(dtype, cache=cache), one, 100, 116)
    kvcache.check_samples(net(dtype, cache=cache), one, 100_000, 100_016)
    far = x.clone()
    far[1, 0] += 0.07
    with pytest.raises(AssertionError):
        kvcache.check_samples(net(dtype, cache=cache), far, 100_000, 100_016)


def test_fp32_samples_behind_long_prompts():
    x = torch.linspace(-1, 1, 256).repeat(3, 1)
    x[1, 0] += 2e-4
    with pytest.raises(AssertionError):
        kvcache.check_samples(net(), x, 100_000, 100_016)


@pytest.mark.gpu
@pytest.mark.parametrize("args", [[], ["--cache", "e4m3", "--qk-norm"]])
def test_the_example_shares_long_prompts(capsys, args):
    """40 samples behind 9000 tokens: more than sharing asks for, in both caches."""
    n = 9000
    assert 39 * n * 2 * 2 * 64 >= (32 + 40) * 1_000_000
    kvcache.main(["--config", "tiny", "--prompt", str(n), "--samples", "40", "--tokens", "2", *args])
    assert "samples x 2 tokens" in capsys.readouterr().out
