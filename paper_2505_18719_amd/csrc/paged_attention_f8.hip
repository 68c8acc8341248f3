// Attention of one new token per environment over a paged KV cache of 8-bit numbers (vla_paged_attention_f8): paged_dev.h with
// 8-bit pages.
#include "paged_dev.h"

namespace vla {

hipError_t launch_paged_attn_f8(const PagedAttnArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16F8>(a, s) : launch_type<kF16F8>(a, s);
}

}  // namespace vla
