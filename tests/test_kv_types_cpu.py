"""Weights and read tokens of another type than the heads are refused, also where an
element of it has as many bytes."""
import pytest
import torch

from paper_2608_22643_amd import binding as B
from test_kv_more_abi_cpu import batch, rows, shape

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("heads", TYPES)
@pytest.mark.parametrize("given", [torch.float32, torch.float16, torch.bfloat16, torch.int16, torch.int32, torch.float64])
def test_types(cache, heads, given):
    s, b = shape(dtype=heads, cache=cache), batch()
    if given == TYPES[heads]:
        return  # what the other tests give
    w, x = torch.ones(s.head_dim).to(given), torch.zeros(b.n_tokens, s.kv_heads, s.head_dim).to(given)
    for norm in (B.make_qk_norm(w), B.make_qk_norm(None, w)):
        with pytest.raises(ValueError):
            B.np_kv_append_norm(s, 0, b, 16, rows(), norm, None, 16, 16)
    for k, v in ((x, None), (None, x)):
        with pytest.raises(ValueError):
            B.np_kv_read(s, 0, b, 16, 16, k, v, 16)
