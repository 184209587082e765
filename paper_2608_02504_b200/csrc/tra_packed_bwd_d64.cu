// Packed attention, gradients, head_dim 64.
#include "tra_packed_bwd.cuh"

int tra_packed_bwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_bwd_shape<64>(c, a); }
