// Packed attention, forward, head_dim 128.
#include "tra_packed_fwd.cuh"

int tra_packed_fwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_fwd_shape<128>(c, a); }
