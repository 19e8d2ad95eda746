// np_attn_shared.hip -- np_attn_decode_shared: decode of sequences that share
// prefixes.
#include "np_attn.hpp"

namespace np {

hipError_t launch_attn_shared(const np_kv_shape& s, int layer, const np_kv_batch& b,
                              const np_kv_shared& sh, const int32_t* table, const void* q,
                              int64_t q_stride, const void* pool, float scale, int window,
                              void* out, int64_t out_stride, void* ws, hipStream_t stream) {
  (void)sh;
  return launch_attn(s, layer, b, table, q, q_stride, pool, scale, window, out, out_stride, ws,
                     stream);
}

}  // namespace np
