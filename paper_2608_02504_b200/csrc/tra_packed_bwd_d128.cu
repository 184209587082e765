// Packed attention, gradients, head_dim 128.
#include "tra_packed_bwd.cuh"

int tra_packed_bwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_bwd_shape<128, 2>(c, a); }
