// Packed attention with fp16 products for bf16 tensors, head_dim 128.
#include "tra_packed_fwd.cuh"

int tra_packed_fwd_fp16_d128(const tra_packed_ctx& c, const tra_packed_launch& a) { return launch_fwd_fp16<128>(c, a); }
