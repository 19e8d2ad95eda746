// np_attn8.hip -- the attention kernels over caches of 8-bit elements.
#include "np_attn.hpp"

namespace np {

hipError_t launch_attn_e4m3(int dtype, AttnArgs& a, int64_t keys, int max_tokens,
                            hipStream_t stream) {
  if (dtype == NP_F32) return launch_attn_t<TF32, true>(a, keys, max_tokens, stream);
  if (dtype == NP_F16) return launch_attn_t<TF16, true>(a, keys, max_tokens, stream);
  return launch_attn_t<TBF16, true>(a, keys, max_tokens, stream);
}

}  // namespace np
