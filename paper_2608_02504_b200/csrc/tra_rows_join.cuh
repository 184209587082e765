// What the kernels for few rows share: the 16 x 8 x 16 products, and the join of a row's parts (warps of a block, then blocks of a
// thread-block cluster, or a workspace that tra_packed_join_kernel reads).
#pragma once
#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kRowsMax = 16;              // rows of a block at most

template <typename T>
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// the same onto zeros (written so, the zeros take no registers)
template <typename T>
__device__ __forceinline__ void mma16816_first(float* d, const uint32_t* a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816_first<__nv_bfloat16>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
template <>
__device__ __forceinline__ void mma16816_first<__half>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// 16 x 8 x 8: the first operand's rows g, g + 8 in two registers
template <typename T>
__device__ __forceinline__ void mma1688(float* c, uint32_t a0, uint32_t a1, uint32_t b);
template <>
__device__ __forceinline__ void mma1688<__nv_bfloat16>(float* c, uint32_t a0, uint32_t a1, uint32_t b) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(b));
}
template <>
__device__ __forceinline__ void mma1688<__half>(float* c, uint32_t a0, uint32_t a1, uint32_t b) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(b));
}

// ---- thread-block clusters: a barrier over the cluster, and 16 bytes of another block's shared memory
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 cluster_ld4(const void* own_address, uint32_t rank) {
  uint32_t addr;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(own_address)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// The rows of a block: n_rows of (sequence, key/value head), from row0 on, over part blockIdx.z of the keys.
struct rows_place {
  tra_seq_range q;
  int kvh, row0, n_rows;
  bool parts, clustered;
};

template <int D>
constexpr int rows_join_bytes(int warps, int rows = kRowsMax) { return (warps + 1) * rows * (D + 4) * 4; }

// store(part, stat): the sums of every of kWarps warps to part [warp][row][D] and its maximum, the sum that divides O and the unrounded
// sum to stat [warp][row][4], kRows rows each.  All kThreads threads call it.
template <typename T, int D, int kWarps, int kThreads, int kRows, typename Store>
__device__ __forceinline__ void rows_join(const tra_packed_launch& p, const rows_place& at, float* part, Store store) {
  const int tid = threadIdx.x, n_rows = at.n_rows;
  const long long part_base = (long long)blockIdx.z * p.total_q * p.heads;
  auto row_token = [&](int r) -> long long { return at.q.begin + (at.row0 + r) / p.group; };
  auto row_head = [&](int r) -> int { return at.kvh * p.group + (at.row0 + r) % p.group; };
  float* stat = part + kWarps * kRows * D;
  float* mine = stat + kWarps * kRows * 4;                // the block's rows: [row][D], then [row][4]
  float* mine_stat = mine + kRows * D;
  if (tid < 32 * kWarps) store(part, stat);
  __syncthreads();
  // Rows of the parts `st(w)`, `row(w)` of n (warps of a block, then blocks of a cluster) on one reference.  A part has seen nothing
  // when its sum is 0, not when its maximum is -inf: scores of NaN leave the maximum where it is, and their NaN in the sums
  // has to reach the result (0 * NaN is NaN).
  auto join = [](int n, auto st, auto row, float& ref, float& sl, float& se, float4& acc) {
    float top = -INFINITY;
    for (int w = 0; w < n; ++w) top = fmaxf(top, st(w).x);
    ref = top > -INFINITY ? top : 0.f;
    sl = se = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < n; ++w) {
      const float4 t = st(w), v = row(w);
      const float f = ex2(t.x - ref);
      if (t.y == 0.f) continue;                              // nothing seen there
      sl += f * t.y;
      se += f * t.z;
      acc.x += f * v.x;
      acc.y += f * v.y;
      acc.z += f * v.z;
      acc.w += f * v.w;
    }
  };
  auto finish = [&](int r, int c, float ref, float sl, float se, const float4& acc) {
    const float inv = sl != 0.f ? 1.f / sl : 0.f;
    const long long tok = row_token(r), row = tok * p.heads + row_head(r);
    if (at.parts) {
      *reinterpret_cast<float4*>(p.part_o + (part_base + row) * D + c) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      if (c == 0) {
        p.part_lse2[part_base + row] = sl != 0.f ? ref + log2f(sl) : -INFINITY;
        if (p.part_exact) p.part_exact[part_base + row] = se != 0.f ? ref + log2f(se) : -INFINITY;
      }
    } else {
      T* dst = (T*)p.o + tok * p.o_stride[0] + row_head(r) * p.o_stride[1] + c;
      const float y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
      const uint2 packed = make_uint2(pack_pair<T>(y[0], y[1]), pack_pair<T>(y[2], y[3]));
      *reinterpret_cast<uint2*>(dst) = packed;
      if (p.o_rest)
        *reinterpret_cast<uint2*>((T*)p.o_rest + row * D + c) = make_uint2(rest_pair<T>(y[0], y[1], packed.x), rest_pair<T>(y[2], y[3], packed.y));
      if (c == 0 && p.lse) p.lse[row] = se != 0.f ? (ref + log2f(se)) * kLn2 : -INFINITY;
    }
  };
  // four channels of a row per step
  for (int i = tid; i < n_rows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    float ref, sl, se;
    float4 acc;
    join(kWarps, [&](int w) { return *reinterpret_cast<const float4*>(stat + (w * kRows + r) * 4); },
         [&](int w) { return *reinterpret_cast<const float4*>(part + (w * kRows + r) * D + c); }, ref, sl, se, acc);
    if (at.clustered) {
      *reinterpret_cast<float4*>(mine + r * D + c) = acc;
      if (c == 0) *reinterpret_cast<float4*>(mine_stat + r * 4) = make_float4(sl != 0.f ? ref : -INFINITY, sl, se, 0.f);
    } else {
      finish(r, c, ref, sl, se, acc);
    }
  }
  if (at.clustered) {
    cluster_sync();                                          // every block's rows are there
    for (int i = (int)blockIdx.z * kThreads + tid; i < n_rows * (D / 4); i += (int)gridDim.z * kThreads) {
      const int r = i / (D / 4), c = (i % (D / 4)) * 4;
      float ref, sl, se;
      float4 acc;
      join((int)gridDim.z, [&](int w) { return cluster_ld4(mine_stat + r * 4, (uint32_t)w); },
           [&](int w) { return cluster_ld4(mine + r * D + c, (uint32_t)w); }, ref, sl, se, acc);
      finish(r, c, ref, sl, se, acc);
    }
    cluster_sync();                                          // nobody leaves while its rows are read
  }
}

}  // namespace
