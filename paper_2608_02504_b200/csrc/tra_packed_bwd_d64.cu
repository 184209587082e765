// Packed attention, gradients, head_dim 64.
#include "tra_packed_bwd.cuh"

int tra_packed_bwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a) {
  return a.stream_rows == 64 ? launch_bwd_shape<64, 1>(c, a) : launch_bwd_shape<64, 2>(c, a);
}
