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
// what rounding to the pair took from two values, rounded itself
template <typename T>
__device__ __forceinline__ uint32_t rest_pair(float lo, float hi, uint32_t packed) {
  float a, b;
  unpack_pair<T>(packed, a, b);
  return pack_pair<T>(lo - a, hi - b);
}


__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// A value that all lanes hold, in a form that the compiler knows to be the same in all of them (a warp reduction's or a vote's
// result).  tcgen05.mma takes its descriptors from uniform registers; where the compiler cannot tell that they are uniform (values
// read from shared memory, or computed under a condition that a lane's own wait decided) every product spends 70 to 85 cycles on
// moving them there, more than a product of 64 columns takes.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_or_sync(0xffffffffu, x); }
__device__ __forceinline__ int uniform(int x) { return (int)__reduce_or_sync(0xffffffffu, (unsigned)x); }
__device__ __forceinline__ bool uniform(bool x) { return __any_sync(0xffffffffu, x) != 0; }

// A launch that follows another one in the stream starts while it ends: the first one allows it (once all its blocks run),
// the second waits where it needs the first one's results.
__device__ __forceinline__ void allow_next_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_last_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Cluster launch control: asks for a block of this grid that has not been started yet; the 16-byte answer arrives on `bar`.
// true: `block` is its blockIdx.x and the block will not be started; false: none left (no further request is made then).
__device__ __forceinline__ void ask_for_launch(uint32_t answer, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar)
               : "memory");
}
__device__ __forceinline__ bool launch_answer(uint32_t answer, int& block) {
  uint32_t yes, x = 0;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\t"
      "ld.shared.b128 a, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, a;\n\t}"
      : "=r"(yes), "=r"(x)
      : "r"(answer)
      : "memory");
  if (yes) block = (int)x;
  return yes != 0;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
template <int kColumns>
__device__ __forceinline__ void tmem_alloc(uint32_t* base) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(base)), "n"(kColumns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int kColumns>
__device__ __forceinline__ void tmem_free(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns) : "memory");
}

// Rows to memory.  A thread holds 64 bytes of its own row (tensor memory gives every lane a row); stored like that, each of a
// warp's 16-byte stores touches 32 lines.  Groups of four lanes exchange 16-byte pieces first, v[4 u ..] = piece u of the own row ->
// v[4 i ..] = piece (lane % 4) of the group's row i, and a store touches eight.  (Groups of eight and whole lines take three
// times the instructions, and this code runs once per tile, out of a cold instruction cache: 7,600 cycles for two tiles
// against 4,500 without any exchange.)
struct RowAddresses {
  uint64_t row[4];             // of the group's rows (0: not stored)
  __device__ __forceinline__ explicit RowAddresses(const void* own) {
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = __shfl_sync(0xffffffffu, (unsigned long long)own, (threadIdx.x & 28) + i);
  }
  // 64 bytes of every row, `offset` bytes from its start; all lanes of the warp call it
  __device__ __forceinline__ void store64(uint32_t* v, int offset) const {
    const int l = threadIdx.x & 3;
#pragma unroll
    for (int b = 1; b < 4; b <<= 1) {
      const bool up = (l & b) != 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (u & b) continue;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t& lo = v[u * 4 + w];
          uint32_t& hi = v[(u | b) * 4 + w];
          const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? lo : hi, b);
          if (up)
            lo = got;
          else
            hi = got;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row[i]) *reinterpret_cast<uint4*>(row[i] + offset + l * 16) = make_uint4(v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]);
  }
};

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
