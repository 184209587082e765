// What the packed-attention kernels add to the PTX wrappers: both 16-bit types, and zeroed rows of a swizzled tile.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "tra_tcgen05.cuh"

namespace {

// Instruction descriptor, kind::f16: fp32 accumulate, both operands of type T, M = 128.
template <typename T>
__host__ __device__ constexpr uint32_t make_idesc_t(int n, bool b_mn_major) {
  return sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value
             ? make_idesc(n, b_mn_major)
             : make_idesc(n, b_mn_major) & ~((1u << 7) | (1u << 10));      // operand formats 0: fp16
}

// two values rounded to T, `lo` in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi) {
  return pack_bf16(lo, hi);
}
template <>
__device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// acc_lo += low half, acc_hi += high half, widened by the mixed-precision add
template <typename T>
__device__ __forceinline__ void add_pair(float& acc_lo, float& acc_hi, uint32_t packed);
template <>
__device__ __forceinline__ void add_pair<__nv_bfloat16>(float& acc_lo, float& acc_hi, uint32_t packed) {
  add_bf16_pair(acc_lo, acc_hi, packed);
}
template <>
__device__ __forceinline__ void add_pair<__half>(float& acc_lo, float& acc_hi, uint32_t packed) {
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "add.rn.f32.f16 %0, lo, %0;\n\t"
      "add.rn.f32.f16 %1, hi, %1;\n\t}"
      : "+f"(acc_lo), "+f"(acc_hi)
      : "r"(packed));
}

template <typename T>
__device__ __forceinline__ void unpack_pair(uint32_t packed, float& lo, float& hi);
template <>
__device__ __forceinline__ void unpack_pair<__nv_bfloat16>(uint32_t packed, float& lo, float& hi) {
  lo = __uint_as_float(packed << 16);
  hi = __uint_as_float(packed & 0xffff0000u);
}
template <>
__device__ __forceinline__ void unpack_pair<__half>(uint32_t packed, float& lo, float& hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  lo = f.x;
  hi = f.y;
}

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// A launch that follows another one in the stream starts while it ends: the first one allows it (once all its blocks run),
// the second waits where it needs the first one's results.
__device__ __forceinline__ void allow_next_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_last_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void tmem_alloc_all(uint32_t* base) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(base)) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_all(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// Zeroes rows [row0, row1) of `atoms` 64-column pieces of a tile, rows 128 bytes apart (the 128-byte swizzle moves
// 16-byte chunks inside a row only).
__device__ __forceinline__ void zero_tile_rows(uint8_t* tile, int row0, int row1, int atoms, int atom_bytes, int tid,
                                               int n_threads) {
  const int per_atom = (row1 - row0) * 8;
  for (int a = 0; a < atoms; ++a)
    for (int i = tid; i < per_atom; i += n_threads)
      *reinterpret_cast<uint4*>(tile + (size_t)a * atom_bytes + row0 * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
}

}  // namespace
