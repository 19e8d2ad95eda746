// np_attn.hip -- np_attn_decode and np_attn_prompt: their arguments, and the
// kernels over plain caches.
#include "np_attn.hpp"

namespace np {

AttnArgs attn_args(const np_kv_shape& s, int layer, const np_kv_batch& b, const int32_t* table,
                   const void* q, int64_t q_stride, const void* pool, float scale, int window,
                   void* out, int64_t out_stride, void* ws) {
  const int64_t w = dtype_size(kv_dtype(s));
  AttnArgs a;
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  a.b = {b.seqs, b.cu_tokens, b.pos0, b.n_seq, b.n_tokens, s.max_seqs,
         (int)std::min<int64_t>(b.max_len, (int64_t)s.seq_pages * s.page_size)};
  a.table = table;
  a.q = (const char*)q;
  a.out = (char*)out;
  a.q_stride = q_stride * w;
  a.out_stride = out_stride * w;
  a.page_bytes = kv_page_bytes(s);
  a.pool = (const char*)pool + (size_t)layer * s.n_pages * a.page_bytes;
  a.Hkv = s.kv_heads;
  a.G = s.heads / s.kv_heads;
  a.D = s.head_dim;
  a.M = s.seq_pages;
  a.N = s.n_pages;
  a.pshift = __builtin_ctz((unsigned)s.page_size);
  a.scale = scale * LOG2E;
  a.window = window;
  a.part = k.part;
  a.zeros = k.zeros;
  a.count = k.count;
  a.ml = k.ml;
  a.err = (int32_t*)((char*)ws + WS_ERR);
  // row blocks: at most one partly filled per row of the batch
  a.tiles = b.cu_tokens ? (int)((int64_t)b.n_tokens * a.G / RB) + b.n_seq
                        : b.n_seq * ((a.G + RB - 1) / RB);
  return a;
}

hipError_t launch_attn(const np_kv_shape& s, int layer, const np_kv_batch& b,
                       const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                       float scale, int window, void* out, int64_t out_stride, void* ws,
                       hipStream_t stream) {
  AttnArgs a = attn_args(s, layer, b, table, q, q_stride, pool, scale, window, out, out_stride, ws);
  // keys a block can see
  int64_t keys = a.b.lim;
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + RB + 32);
  keys = std::max<int64_t>(keys, 1);
  const int dtype = kv_dtype(s);
  if (kv_e4m3(s)) return launch_attn_e4m3(dtype, a, keys, b.max_tokens, stream);
  if (dtype == NP_F32) return launch_attn_t<TF32, false>(a, keys, b.max_tokens, stream);
  if (dtype == NP_F16) return launch_attn_t<TF16, false>(a, keys, b.max_tokens, stream);
  return launch_attn_t<TBF16, false>(a, keys, b.max_tokens, stream);
}

}  // namespace np
