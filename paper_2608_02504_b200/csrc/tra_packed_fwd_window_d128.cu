// Packed attention with a window, forward, head_dim 128.
#include "tra_packed_fwd.cuh"

int tra_packed_fwd_window_d128(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_fwd_window<128>(c, a); }
