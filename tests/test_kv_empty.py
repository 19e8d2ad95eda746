"""Batches without rows or without tokens: accepted, nothing enqueued (so the
C calls answer on the CPU too), whatever the token arrays are."""
import ctypes

import pytest
import torch

from paper_2608_22643_amd import binding as B
from paper_2608_22643_amd import kvcache
from paper_2608_22643_amd import workload as W
from test_kv_abi_cpu import refused, shape


@pytest.mark.parametrize("n_seq,cu", [(0, None), (0, 16), (3, 16)])
def test_calls_without_tokens(n_seq, cu):
    s = shape()
    b = B.np_kv_batch(n_seq, 0, 0, 100, None, cu, 16 if n_seq else None)
    x = torch.empty(0, 32, 128, dtype=torch.float16)
    assert x.data_ptr() == 0
    kv = torch.empty(0, 8, 128, dtype=torch.float16)
    B.np_kv_append(s, 0, b, 16, B.make_qkv(x, kv, kv, x), None, 16, 16)
    B.np_attn_prompt(s, 0, b, 16, x, 16, 0.1, 0, x, 16)
    if cu is None:
        B.np_attn_decode(s, 0, b, 16, x, 16, 0.1, 0, x, 16)
    # everything else is still checked
    refused(lambda: B.np_attn_prompt(s, 99, b, 16, x, 16, 0.1, 0, x, 16))
    refused(lambda: B.np_attn_prompt(s, 0, b, 16, x, 16, 0.1, -1, x, 16))
    refused(lambda: B.np_attn_prompt(s, 0, b, None, x, 16, 0.1, 0, x, 16))
    refused(lambda: B.np_kv_append(s, 0, b, 16, B.make_qkv(x, kv, kv, x), None, None, 16))


def test_arrays_of_a_token_are_checked():
    s = shape()
    b = B.np_kv_batch(1, 1, 1, 100, None, None, 16)
    for q, out in ((None, 32), (16, None), (24, 32)):
        assert B.lib().np_attn_decode(ctypes.byref(s), 0, ctypes.byref(b), 16, q, 4096, 16, 0.1, 0, out, 4096, 16,
                                      None) == B.NP_ERR_INVALID_ARG


@pytest.mark.gpu
def test_the_cache_without_rows_or_tokens():
    cfg = W.get("tiny").with_(layers=2)
    net = kvcache.DecoderLayers(cfg, 4, 2, 3, 64, 16)
    cache = net.cache
    x = torch.zeros(0, cfg.d_model, dtype=kvcache.TORCH_DT[cfg.adtype], device="cuda:0")
    for seqs, new in (([], None), ([], []), ([0, 2], [0, 0])):
        assert net.step(x, cache.extend(seqs, new)).shape == x.shape
    cache.fork([], [])
    cache.free([])
    assert cache.kv_len.tolist() == [0, 0, 0] and cache.pages_used() == 0
    assert cache.device_error() == 0
