// Packed attention with a window, gradients, head_dim 128.
#include "tra_packed_bwd.cuh"

int tra_packed_bwd_window_d128(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_bwd_window<128, 2, false>(c, a); }
