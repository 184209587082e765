// Packed attention with a window, gradients, head_dim 64, key tiles of a few steps.
#include "tra_packed_bwd.cuh"

int tra_packed_bwd_few_d64(const tra_packed_ctx& c, const tra_packed_launch& a) {
  return a.stream_rows == 64 ? launch_bwd_window<64, 1, true>(c, a) : launch_bwd_window<64, 2, true>(c, a);
}
