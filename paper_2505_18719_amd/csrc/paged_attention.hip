// Attention of one new token per environment over a paged KV cache (vla_paged_attention): paged_dev.h with 16-bit pages.
#include "paged_dev.h"

namespace vla {

size_t paged_attn_bytes(int n_env, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const int group = n_heads / n_kv_heads, tiles = query_tiles(group, head_dim), rows = query_rows(group, tiles);
  const int blocks = (tiles == 1 ? head_blocks<1>(group) : head_blocks<2>(group)) * n_kv_heads;
  if (!split_keys((long long)n_env * blocks, max_pages)) return 256;
  if (head_dim == 64) return tiles == 1 ? split_bytes<64, 1>(rows) : split_bytes<64, 2>(rows);
  if (head_dim == 128) return tiles == 1 ? split_bytes<128, 1>(rows) : split_bytes<128, 2>(rows);
  return split_bytes<256, 1>(rows);
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16>(a, s) : launch_type<kF16>(a, s);
}

}  // namespace vla
