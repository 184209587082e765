// Packed attention of few rows over many keys: both head dimensions and types.
#include "tra_packed_rows.cuh"

int tra_packed_rows(const tra_packed_ctx& c, const tra_packed_launch& a, int chunk, bool clustered) {
  const bool bf = c.h->cfg.dtype == TRA_BF16;
  if (c.h->cfg.head_dim == 128)
    return bf ? launch_rows<__nv_bfloat16, 128>(c, a, chunk, clustered) : launch_rows<__half, 128>(c, a, chunk, clustered);
  return bf ? launch_rows<__nv_bfloat16, 64>(c, a, chunk, clustered) : launch_rows<__half, 64>(c, a, chunk, clustered);
}
