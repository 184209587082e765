// Packed attention over keys and values in two pieces, head_dim 64.
#include "tra_packed_fwd.cuh"

int tra_packed_fwd_pieces_d64(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_fwd_pieces<64>(c, a); }
