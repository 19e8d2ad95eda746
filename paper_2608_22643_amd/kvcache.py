"""The paged key-value cache and whole decoder layers over the C ABI (the
runtime around the cache and attention kernels).

KVCache owns the device buffers of a cache (torch allocations) and forwards to
the np_kv_* and np_attn_* calls on one stream, in order with the stream its
caller is on; sequences are rows of its page table.  A step is

    extend (pages for the new tokens) -> per layer: append -> attention

DecoderLayers runs whole layers with synthetic weights: attention over the
cache and the gated MLP of the configuration's records.  Prompts of several
sequences are packed into one pass (np_attn_prompt; the MLP's activations by
np_act_batch); decoding brings one token per sequence (np_attn_decode, or
np_attn_decode_shared where sequences share a prefix, and np_dense_mlp per row).
The cache holds elements of the layers' type, or 8-bit ones (cache="e4m3"), and
the query and key heads may be normed.  Run as a program it prefills a prompt,
forks it into samples that share its pages, decodes them, frees them and compacts
the pool:

    python -m paper_2608_22643_amd.kvcache --config tiny --prompt 100 --samples 3
    python -m paper_2608_22643_amd.kvcache --config tiny --cache e4m3 --qk-norm
"""
from __future__ import annotations

import contextlib
import math

import numpy as np
import torch

from . import binding as B
from . import workload as W

TORCH_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def rotary_tables(dim: int, max_pos: int, theta: float = 10000.0, device="cuda:0"):
    """cos and sin [max_pos][dim / 2] float32 of angles pos * theta^(-2 i / dim)."""
    f = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * f[None]
    return ang.cos().float().to(device), ang.sin().float().to(device)


class KVCache:
    """Pages, page table, lengths and reference counts of up to max_seqs
    sequences of at most max_len tokens, n_pages pages of page_size tokens in
    every layer.

    All calls are enqueued on `stream` (a torch stream or a handle; default: the
    device's default stream), which every buffer of the cache and of its
    batches belongs to.  Called while another stream is current, a call starts
    after what that one holds, and it goes on after the call: inputs and
    outputs need no events, and may be dropped as soon as the call returns.

    cache: None (elements of dtype) or "e4m3" (8-bit elements, a scale for each
    token and key-value head: half the memory of 16-bit ones).

    Sequences, prefix lengths: Python lists (uploaded from pageable memory, which
    waits for the stream) or contiguous int32 tensors on the device."""

    def __init__(self, layers: int, heads: int, kv_heads: int, head_dim: int, dtype: str, max_seqs: int, max_len: int,
                 page_size: int = 64, n_pages: int | None = None, device: str = "cuda:0", stream=None,
                 rotary_dim: int | None = None, cache: str | None = None):
        seq_pages = -(-max_len // page_size)
        n_pages = max_seqs * seq_pages if n_pages is None else n_pages
        self.shape = B.make_kv_shape(layers, heads, kv_heads, head_dim, page_size, n_pages, max_seqs, seq_pages, dtype,
                                     cache)
        B.np_kv_shape_check(self.shape)
        self.device = torch.device(device)
        if stream is None or stream == 0:
            stream = torch.cuda.default_stream(self.device)
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, self.device)
        self.stream = stream
        self.max_len = seq_pages * page_size
        self.scale = 1.0 / math.sqrt(head_dim)
        self.rotary = None
        with self.on_stream():
            i32 = dict(dtype=torch.int32, device=self.device)
            self.page_table = torch.empty(max_seqs, seq_pages, **i32)
            self.kv_len, self.refs = torch.empty(max_seqs, **i32), torch.empty(n_pages, **i32)
            self.state = B.make_kv_state(self.page_table, self.kv_len, self.refs)
            self.pool = torch.empty(B.kv_pool_shape(self.shape),
                                    dtype=torch.uint8 if cache == "e4m3" else TORCH_DT[dtype], device=self.device)
            self.ws = torch.zeros(B.np_kv_workspace_size(self.shape), dtype=torch.uint8, device=self.device)
            if rotary_dim:
                self.rotary = B.make_rotary(*rotary_tables(rotary_dim, self.max_len, device=self.device))
            self.reset()

    @contextlib.contextmanager
    def on_stream(self):
        """Makes the cache's stream the current one, after what the caller's
        stream holds; on leaving, the caller's stream goes on after it.  So a
        block that either stream's allocator hands out again is written after
        the other's last use of it."""
        here = torch.cuda.current_stream(self.device)
        if here.cuda_stream == self.stream.cuda_stream:
            yield
            return
        self.stream.wait_stream(here)
        try:
            with torch.cuda.stream(self.stream):
                yield
        finally:
            here.wait_stream(self.stream)

    def _ids(self, x):
        if x is None:
            return None
        if isinstance(x, torch.Tensor):
            if x.dtype != torch.int32 or not x.is_cuda or not x.is_contiguous():
                raise ValueError("need a list or a contiguous int32 tensor on the device")
            x.record_stream(self.stream)  # a batch may be read after calls from other streams
            return x
        return torch.tensor(list(x), dtype=torch.int32, device=self.device)

    def reset(self) -> None:
        with self.on_stream():
            B.np_kv_reset(self.shape, self.state, self.ws, self.stream)

    def extend(self, seqs, n_new: list[int] | None = None, max_len: int | None = None) -> B.np_kv_batch:
        """Pages for n_new[b] tokens of sequence seqs[b] (default: one each; a
        list, since the host needs their sum); returns the step's batch for
        append, prompt and decode.  max_len: a bound on the lengths after the
        step, if the caller knows one."""
        if n_new is not None:
            n_new = [int(k) for k in n_new]
            if any(k < 0 for k in n_new):
                raise ValueError(f"negative token counts in {n_new}")
        with self.on_stream():
            seqs = self._ids(seqs)
            n = seqs.numel()
            if n_new is not None and len(n_new) != n:
                raise ValueError(f"{len(n_new)} token counts for {n} sequences")
            pos0 = torch.empty(n, dtype=torch.int32, device=self.device)
            B.np_kv_extend(self.shape, self.state, self.pool, n, seqs, self._ids(n_new), pos0, self.ws, self.stream)
            most = self.max_len if max_len is None else max_len
            if n_new is None:
                return B.make_kv_batch(n, n, 1, most, pos0, seqs=seqs)
            cu = self._ids(np.concatenate([[0], np.cumsum(n_new)]).tolist())
            return B.make_kv_batch(n, sum(n_new), max(n_new, default=0), most, pos0, seqs=seqs, cu_tokens=cu)

    def fork(self, src, dst, lens=None) -> None:
        with self.on_stream():
            src, dst, lens = self._ids(src), self._ids(dst), self._ids(lens)
            if dst.numel() != src.numel() or (lens is not None and lens.numel() != src.numel()):
                raise ValueError("src, dst and lens differ in length")
            B.np_kv_fork(self.shape, self.state, src.numel(), src, dst, lens, self.ws, self.stream)

    def free(self, seqs) -> None:
        with self.on_stream():
            seqs = self._ids(seqs)
            B.np_kv_free(self.shape, self.state, seqs.numel(), seqs, self.ws, self.stream)

    def compact(self) -> None:
        with self.on_stream():
            B.np_kv_compact(self.shape, self.state, self.pool, None, self.ws, self.stream)

    def append(self, layer: int, batch, q, k, v, q_out, norm: B.np_qk_norm | None = None) -> None:
        """norm (binding.make_qk_norm): the query and key heads are normed first."""
        with self.on_stream():
            rows = B.make_qkv(q, k, v, q_out)
            if norm is None:
                B.np_kv_append(self.shape, layer, batch, self.page_table, rows, self.rotary, self.pool, self.ws,
                               self.stream)
            else:
                B.np_kv_append_norm(self.shape, layer, batch, self.page_table, rows, norm, self.rotary, self.pool,
                                    self.ws, self.stream)

    def read(self, layer: int, batch, k_out, v_out) -> None:
        """The batch's tokens' keys and values ([tokens][kv_heads][head_dim] tensors of dtype, either None)."""
        with self.on_stream():
            B.np_kv_read(self.shape, layer, batch, self.page_table, self.pool, k_out, v_out, self.ws, self.stream)

    def share(self, lead, prefix, max_prefix: int | None = None) -> B.np_kv_shared:
        """Groups of a batch's rows that share a prefix, for attend: lead[b] the first row of row b's group (its rows
        next to each other), prefix[lead] the positions that the group's sequences have in common, as fork left them.
        max_prefix: a bound on them (of lists, the largest; of tensors, max_len)."""
        if max_prefix is None:
            max_prefix = self.max_len if isinstance(prefix, torch.Tensor) else max((int(p) for p in prefix), default=0)
        with self.on_stream():
            lead, prefix = self._ids(lead), self._ids(prefix)
            if lead.numel() != prefix.numel():
                raise ValueError(f"{lead.numel()} leads and {prefix.numel()} prefixes")
            return B.make_kv_shared(lead, prefix, max_prefix)

    def attend(self, layer: int, batch, q, out, window: int = 0, shared: B.np_kv_shared | None = None) -> None:
        """Attention of the batch's tokens; the keys and values of its new
        tokens have been appended.  shared (share): of one token a row, whose
        groups' prefixes are read once."""
        if shared is not None:
            if batch.cu_tokens:
                raise ValueError("shared prefixes are for batches of one token a row")
            for x in getattr(shared, "_kept", ()):
                if x.numel() != batch.n_seq:
                    raise ValueError(f"{x.numel()} leads for {batch.n_seq} rows")
            with self.on_stream():
                B.np_attn_decode_shared(self.shape, layer, batch, shared, self.page_table, q, self.pool, self.scale,
                                        window, out, self.ws, self.stream)
            return
        call = B.np_attn_prompt if batch.cu_tokens else B.np_attn_decode
        with self.on_stream():
            call(self.shape, layer, batch, self.page_table, q, self.pool, self.scale, window, out, self.ws,
                 self.stream)

    def pages_used(self) -> int:
        with self.on_stream():
            return int((self.refs > 0).sum())

    def device_error(self) -> int:
        return B.np_device_error(self.ws, self.stream)


class DecoderLayers:
    """cfg.layers whole decoder layers with synthetic weights: x += Wo attention(
    norm(x)), x += MLP(norm(x)), norm(x) = x / rms(x); the MLP from the
    configuration's neuron records.  Everything runs on the cache's stream, in
    order with the caller's as KVCache's calls are."""

    def __init__(self, cfg: W.Config, heads: int, kv_heads: int, max_seqs: int, max_len: int, page_size: int = 64,
                 window: int = 0, device: str = "cuda:0", n_pages: int | None = None, stream=None,
                 cache: str | None = None, qk_norm: bool = False):
        d, dt = cfg.d_model, TORCH_DT[cfg.adtype]
        self.cfg, self.heads, self.kv_heads, self.head_dim, self.window = cfg, heads, kv_heads, d // heads, window
        self.device = torch.device(device)
        self.cache = KVCache(cfg.layers, heads, kv_heads, self.head_dim, cfg.adtype, max_seqs, max_len, page_size,
                             n_pages, device, stream, rotary_dim=self.head_dim // 16 * 16, cache=cache)
        g = torch.Generator().manual_seed(cfg.seed + 17)
        width = (heads + 2 * kv_heads) * self.head_dim

        def normal(rows, cols):
            return (torch.randn(rows, cols, generator=g) / math.sqrt(rows)).to(dt).to(self.device)

        with self.cache.on_stream():
            self.wqkv = [normal(d, width) for _ in range(cfg.layers)]
            self.wo = [normal(d, d) for _ in range(cfg.layers)]
            # per layer, the weights of the query and key heads' norms
            self.qk_norm = [B.make_qk_norm(*((1 + 0.1 * torch.randn(self.head_dim, generator=g)).to(dt).to(self.device)
                                             for _ in range(2)), 1e-6)
                            for _ in range(cfg.layers)] if qk_norm else [None] * cfg.layers
            self.records = []  # per layer [F][3d], resident
            for layer in range(cfg.layers):
                r = W.storage(cfg, layer, 1)[0]
                t = torch.from_numpy(r.view(np.int16) if cfg.wdtype != "f32" else r).to(self.device)
                self.records.append(t.view(dt) if cfg.wdtype != "f32" else t)
            self.mlp_shape = B.make_shape(cfg.layers, d, cfg.d_ffn, cfg.rank, cfg.k, cfg.capacity, cfg.wdtype,
                                          cfg.adtype, cfg.act)
            self.mlp_ws = torch.zeros(B.np_workspace_size(self.mlp_shape), dtype=torch.uint8, device=self.device)

    def _norm(self, x):
        f = x.float()
        return (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def _mlp(self, layer: int, x):
        rec, d, n = self.records[layer], self.cfg.d_model, x.shape[0]
        if n > 16:  # a prompt: the activations on the matrix cores, then the down rows
            acts = torch.empty(n, self.cfg.d_ffn, dtype=torch.float32, device=self.device)
            B.np_act_batch(self.mlp_shape, rec, x, n, acts, None, self.cache.stream)
            return (acts @ rec[:, 2 * d:].float()).to(x.dtype)
        y = torch.empty_like(x)
        for i in range(n):
            B.np_dense_mlp(self.mlp_shape, rec, x[i], y[i], self.mlp_ws, self.cache.stream)
        return y

    def step(self, x, batch, shared=None):
        """The layers over x [tokens][d_model] for a batch of KVCache.extend (shared: KVCache.share)."""
        here = torch.cuda.current_stream(self.device)
        with self.cache.on_stream():
            x = self._layers(x, batch, shared)
        if here.cuda_stream != self.cache.stream.cuda_stream:
            x.record_stream(here)
        return x

    def _layers(self, x, batch, shared=None):
        hq, hk, hd = self.heads, self.kv_heads, self.head_dim
        for layer in range(self.cfg.layers):
            qkv = (self._norm(x) @ self.wqkv[layer]).view(x.shape[0], hq + 2 * hk, hd)
            q = torch.empty(x.shape[0], hq, hd, dtype=x.dtype, device=self.device)
            out = torch.empty_like(q)
            self.cache.append(layer, batch, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], q,
                              self.qk_norm[layer])
            self.cache.attend(layer, batch, q, out, self.window, shared)
            x = x + out.view(x.shape[0], hq * hd) @ self.wo[layer]
            x = x + self._mlp(layer, self._norm(x))
        return x


def check_samples(net: DecoderLayers, x, prompt: int, total: int) -> None:
    """x [samples][d_model] of samples that had the same `total` tokens, `prompt` of them shared.  Bit for bit the same
    where np_attn_decode cuts their keys alike: up to 768 groups of 128 keys, and less than 32 MB that sharing the prompt
    could save.  Beyond that their attention may differ by roundings, which the layers pass on."""
    n, dt = x.shape[0], net.cfg.adtype
    groups = n * net.kv_heads * -(-net.heads // net.kv_heads // 16) * -(-total // 128)
    row = net.head_dim * (1 if net.cache.pool.dtype == torch.uint8 else x.element_size())
    if groups <= 768 and (n - 1) * prompt * net.kv_heads * 2 * row < 32_000_000:
        assert all(torch.equal(x[0], x[i]) for i in range(n)), "samples of the same tokens agree"
        return
    off = (x.float() - x[:1].float()).abs().max() / x.float().abs().max()
    # (a key or value that falls to the other side of a border of 8-bit elements is off by a sixteenth)
    most = 0.05 if net.cache.pool.dtype == torch.uint8 else {"f32": 1e-4, "f16": 0.02, "bf16": 0.05}[dt]
    assert off <= most, f"samples of the same tokens agree: off by {float(off):.2g} of the largest output"


def main(argv=None) -> None:
    import argparse
    import time

    ap = argparse.ArgumentParser(description="prefill a prompt, fork it, decode the samples")
    ap.add_argument("--config", default="tiny")
    ap.add_argument("--layers", type=int, default=2, help="layers of the configuration to run")
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=100)
    ap.add_argument("--samples", type=int, default=3)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--cache", choices=["same", "e4m3"], default="same", help="elements of the cache")
    ap.add_argument("--qk-norm", action="store_true", help="norms of the query and key heads")
    args = ap.parse_args(argv)
    cfg = W.get(args.config).with_(layers=args.layers)
    n, total = args.samples, args.prompt + args.tokens
    net = DecoderLayers(cfg, args.heads, args.kv_heads, n + 1, total, cache=args.cache, qk_norm=args.qk_norm)
    cache = net.cache
    h = torch.from_numpy(W.hidden(cfg, total).view(np.uint8)).to(net.device).view(TORCH_DT[cfg.adtype])
    prompt_out = net.step(h[:args.prompt], cache.extend([0], [args.prompt], args.prompt))
    cache.fork([0] * n, range(1, n + 1))
    pages = cache.pages_used()
    # the prompt is read once for all samples, where that is worth a second kernel
    shared = cache.share([0] * n, [args.prompt] * n)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for t in range(args.prompt, total):
        x = net.step(h[t:t + 1].repeat(n, 1), cache.extend(range(1, n + 1), max_len=t + 1), shared)
    torch.cuda.synchronize()
    dt = time.perf_counter() - t0
    assert torch.isfinite(prompt_out.float()).all() and torch.isfinite(x.float()).all()
    check_samples(net, x, args.prompt, total)
    used = cache.pages_used()
    cache.free([0])
    cache.compact()
    print(f"prompt of {args.prompt} tokens, {n} samples x {args.tokens} tokens: {n * args.tokens / dt:.0f} tokens/s; "
          f"pages: {pages} shared after the fork, {used} after decoding, {cache.pages_used()} after freeing the prompt")
    assert cache.device_error() == 0


if __name__ == "__main__":
    main()
