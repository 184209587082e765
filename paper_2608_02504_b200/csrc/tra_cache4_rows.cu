// Attention of few rows over a cache of 4 bits: both head dimensions and types.
#include "tra_cache4_rows.cuh"

int tra_cache4_rows(const tra_packed_ctx& c, const tra_cache4_launch& a, int chunk, bool clustered) {
  const bool bf = c.h->cfg.dtype == TRA_BF16;
  if (c.h->cfg.head_dim == 128) return bf ? launch_cache4<__nv_bfloat16, 128>(c, a, chunk, clustered) : launch_cache4<__half, 128>(c, a, chunk, clustered);
  return bf ? launch_cache4<__nv_bfloat16, 64>(c, a, chunk, clustered) : launch_cache4<__half, 64>(c, a, chunk, clustered);
}
