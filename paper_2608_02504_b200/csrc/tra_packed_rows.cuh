// Attention of few rows over many keys: one new token of every sequence (or a few), over a key/value cache split along
// its length.  At most 16 rows (tokens times the heads of a group) per sequence and key/value head.
//
// Bound: HBM, every key and value is read once and used for at most 16 rows.  A thread block takes `chunk` keys of one
// (sequence, key/value head): a producer warp streams 64-key tiles of K and V through a ring of TMA
// loads (96 KB in flight per block, two blocks per SM), and four warps take sixteen keys of every tile each, with a running
// maximum and sum of their own, joined at the end through shared memory.  The products are 16 x 16 x 16 mma.sync steps:
// a 128-row tcgen05 tile would spend its softmax on 112 rows that are not there (128 threads walk 128 score columns per key
// block whatever the rows hold), and the tensor pipe is idle either way.
//
// 64 caches of 700 to 32,768 keys, 40 / 8 heads, d 128: 686 us, 6.4 TB/s (98 % of the copy rate).  One cache of 777 keys, 12 heads, d 64:
// 5.5 us on the GPU.
//
// The parts of a sequence: up to eight are one thread-block cluster and are joined through distributed shared memory, without
// a workspace or a second launch; more go through a workspace and tra_packed_join_kernel.
#pragma once
#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kRowsMax = 16;
constexpr int kRowsTile = 64;             // keys per ring slot
constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = 32 * (kRowsWarps + 1);

template <int D>
struct RowsCfg {
  static constexpr int kAtoms = D / 64;
  static constexpr int kAtomBytes = kRowsTile * 128;
  static constexpr int kTileBytes = kAtoms * kAtomBytes;
  static constexpr int kStages = D == 128 ? 3 : 6;            // of one K and one V tile: 96 KB
  static constexpr int kSmemData = kStages * 2 * kTileBytes;
  static constexpr int kSmemBytes = kSmemData + 1024 + 256;
};
// the join of the warps' parts reuses the ring
static_assert((kRowsWarps + 1) * kRowsMax * (128 + 4) * 4 <= RowsCfg<128>::kSmemData, "join area");
static_assert((kRowsWarps + 1) * kRowsMax * (64 + 4) * 4 <= RowsCfg<64>::kSmemData, "join area");

struct RowsCtl {
  uint64_t full[6], empty[6];
  int abort_flag;
};
static_assert(sizeof(RowsCtl) <= 256, "control block");

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
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

// sequence = blockIdx.x, key/value head = blockIdx.y, part = blockIdx.z (keys [part * chunk, ...)); chunk is a multiple of 64
template <typename T, int D>
__global__ void __launch_bounds__(kRowsThreads, 2) tra_packed_rows_kernel(const __grid_constant__ tra_packed_launch p, int chunk, int clustered) {
  using C = RowsCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  RowsCtl* ctl = (RowsCtl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int seq = blockIdx.x, kvh = blockIdx.y;
  const tra_seq_range qr = tra_clamp_range(p.cu_q[seq], p.cu_q[seq + 1], p.total_q, p.max_q, p.status);
  const tra_seq_range kr = tra_clamp_range(p.k_begin[seq], p.k_end[seq], p.total_k, p.max_k, p.status);
  const bool parts = gridDim.z > 1 && !clustered;
  if (parts) allow_next_launch();                            // the join of the parts
  const int n_rows = qr.len * p.group;                       // <= 16
  if (n_rows == 0) return;
  const int ahead = kr.len - qr.len;
  const int key0 = (int)blockIdx.z * chunk, key1 = min(key0 + chunk, kr.len);     // chunk * parts fits an int
  const int n_tiles = key1 > key0 ? (key1 - key0 + kRowsTile - 1) / kRowsTile : 0;
  const long long part_base = (long long)blockIdx.z * p.total_q * p.heads;
  auto row_token = [&](int r) -> long long { return qr.begin + r / p.group; };
  auto row_head = [&](int r) -> int { return kvh * p.group + r % p.group; };

  if (n_tiles == 0 && parts) {                               // nothing here: the join skips the part
    if (tid < n_rows) {
      const long long row = part_base + row_token(tid) * p.heads + row_head(tid);
      p.part_lse2[row] = -INFINITY;
      if (p.part_exact) p.part_exact[row] = -INFINITY;
    }
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(smem_u32(&ctl->full[i]), 1);
      mbar_init(smem_u32(&ctl->empty[i]), kRowsWarps);
    }
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  volatile int* abort_flag = &ctl->abort_flag;

  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, le[2] = {0.f, 0.f};      // rows lane / 4 and lane / 4 + 8
  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[i][j] = 0.f;

  if (warp == kRowsWarps) {
    if (lane == 0) {
      int slot = 0;
      uint32_t phase = 1u;                                   // the first pass over the ring finds every slot free
      for (int t = 0; t < n_tiles; ++t) {
        if (!mbar_wait(smem_u32(&ctl->empty[slot]), phase, abort_flag, p.status)) break;
        const uint32_t bar = smem_u32(&ctl->full[slot]);
        mbar_expect_tx(bar, 2 * C::kTileBytes);
        for (int kv = 0; kv < 2; ++kv)
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(smem + (2 * slot + kv) * C::kTileBytes + a * C::kAtomBytes), kv == 0 ? &p.map_k : &p.map_v,
                        bar, a * 64, kvh, kr.begin + key0 + t * kRowsTile);
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
      }
    }
  } else {
    const int g = lane >> 2, tig = lane & 3;
    const float scale_log2 = p.sm_scale * kLog2e;
    // Q rows as the A operand, straight from global memory; rows that are not there are zero
    uint32_t qa[D / 16][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = g + 8 * half;
      const T* qrow = (const T*)p.q + row_token(r < n_rows ? r : 0) * p.q_stride[0] + row_head(r < n_rows ? r : 0) * p.q_stride[1];
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          qa[kk][half + 2 * c] = r < n_rows ? *reinterpret_cast<const uint32_t*>(qrow + kk * 16 + c * 8 + tig * 2) : 0u;
    }
    int seen[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int t = min((g + 8 * half) / p.group, qr.len - 1);
      seen[half] = p.causal ? min(max(t + 1 + ahead, 0), kr.len) : kr.len;
    }
    const int seen_min = p.causal ? min(max(1 + ahead, 0), kr.len) : kr.len;       // of the first token
    const int row_in_tile = warp * 16;
    int slot = 0;
    uint32_t phase = 0u;
    bool alive = true;
    for (int t = 0; t < n_tiles; ++t) {
      if (!mbar_wait_warp(smem_u32(&ctl->full[slot]), phase, abort_flag, p.status)) {
        alive = false;
        break;
      }
      const int k0 = key0 + t * kRowsTile + row_in_tile;     // first key of this warp, inside the sequence
      if (k0 < key1) {
        uint8_t* kt = smem + 2 * slot * C::kTileBytes;
        uint8_t* vt = kt + C::kTileBytes;
        if (k0 + 16 > key1)                                  // the sequence ends here: rows that are not its own may hold
          zero_tile_rows(vt, row_in_tile + (key1 - k0), row_in_tile + 16, C::kAtoms, C::kAtomBytes, lane, 32);   // anything
        __syncwarp();
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        {
          const int row = row_in_tile + ((lane >> 4) << 3) + (lane & 7);
          const uint32_t base = smem_u32(kt) + row * 128;
          const int sw = row & 7, c0 = (lane >> 3) & 1;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            uint32_t b[4];
            ldsm4(base + (kk >> 2) * C::kAtomBytes + ((((kk & 3) * 2 + c0) ^ sw) << 4), b);
            mma16816<T>(s[0], qa[kk], b[0], b[1]);
            mma16816<T>(s[1], qa[kk], b[2], b[3]);
          }
        }
        if (k0 + 16 > min(seen_min, key1)) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int lim = min(seen[half], key1) - k0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if ((j >> 1) * 8 + tig * 2 + (j & 1) >= lim) s[j >> 1][half * 2 + (j & 1)] = -INFINITY;
          }
        }
        uint32_t pa[4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float t4[4] = {s[0][half * 2] * scale_log2, s[0][half * 2 + 1] * scale_log2, s[1][half * 2] * scale_log2,
                         s[1][half * 2 + 1] * scale_log2};
          float mx = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          // exact whatever the reference is, as long as all terms share it: raised only when it is 8 (2^8) behind
          if (mx > m[half] + kRescaleThreshold) {
            const float alpha = ex2(m[half] - mx);
            l[half] *= alpha;
            le[half] *= alpha;
            m[half] = mx;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
              o[i][half * 2] *= alpha;
              o[i][half * 2 + 1] *= alpha;
            }
          }
          const float ref = m[half] > -INFINITY ? m[half] : 0.f;
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = ex2(t4[j] - ref);
          le[half] += (x[0] + x[1]) + (x[2] + x[3]);
          pa[half] = pack_pair<T>(x[0], x[1]);
          pa[half + 2] = pack_pair<T>(x[2], x[3]);
          float s0 = 0.f, s1 = 0.f;                          // the sum that divides O: of the rounded probabilities
          add_pair<T>(s0, s1, pa[half]);
          add_pair<T>(s0, s1, pa[half + 2]);
          l[half] += s0 + s1;
        }
        {
          const int row = row_in_tile + (lane & 15);
          const uint32_t base = smem_u32(vt) + row * 128;
          const int sw = row & 7, c0 = lane >> 4;
#pragma unroll
          for (int nn = 0; nn < D / 16; ++nn) {
            uint32_t b[4];
            ldsm4_trans(base + (nn >> 2) * C::kAtomBytes + ((((nn & 3) * 2 + c0) ^ sw) << 4), b);
            mma16816<T>(o[2 * nn], pa, b[0], b[1]);
            mma16816<T>(o[2 * nn + 1], pa, b[2], b[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->empty[slot]));
      if (++slot == C::kStages) {
        slot = 0;
        phase ^= 1u;
      }
    }
    (void)alive;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
      le[half] += __shfl_xor_sync(0xffffffffu, le[half], 1);
      le[half] += __shfl_xor_sync(0xffffffffu, le[half], 2);
    }
  }
  __syncthreads();                                           // every tile has been read: the ring becomes the join area
  const bool gave_up = ctl->abort_flag != 0;
  if (gave_up) {
    // a wait ran out: copies in flight land before the block ends; nothing is written (and nothing added to a cluster's rows)
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    if (!clustered) return;
  }
  float* part = (float*)smem;                                // [warp][row][D], then [warp][row][4]: m, l, le
  float* stat = part + kRowsWarps * kRowsMax * D;
  float* mine = stat + kRowsWarps * kRowsMax * 4;            // the block's rows: [row][D], then [row][4]
  float* mine_stat = mine + kRowsMax * D;
  if (warp < kRowsWarps) {
    const int g = lane >> 2, tig = lane & 3;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = g + 8 * half;
      float* dst = part + (warp * kRowsMax + r) * D;
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        *reinterpret_cast<float2*>(dst + i * 8 + tig * 2) = make_float2(o[i][half * 2], o[i][half * 2 + 1]);
      if (tig == 0) {
        float* st = stat + (warp * kRowsMax + r) * 4;
        st[0] = m[half];
        st[1] = gave_up ? 0.f : l[half];
        st[2] = le[half];
      }
    }
  }
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
    if (parts) {
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
  for (int i = tid; i < n_rows * (D / 4); i += kRowsThreads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    float ref, sl, se;
    float4 acc;
    join(kRowsWarps, [&](int w) { return *reinterpret_cast<const float4*>(stat + (w * kRowsMax + r) * 4); },
         [&](int w) { return *reinterpret_cast<const float4*>(part + (w * kRowsMax + r) * D + c); }, ref, sl, se, acc);
    if (clustered) {
      *reinterpret_cast<float4*>(mine + r * D + c) = acc;
      if (c == 0) *reinterpret_cast<float4*>(mine_stat + r * 4) = make_float4(sl != 0.f ? ref : -INFINITY, sl, se, 0.f);
    } else {
      finish(r, c, ref, sl, se, acc);
    }
  }
  if (clustered) {
    cluster_sync();                                          // every block's rows are there
    for (int i = (int)blockIdx.z * kRowsThreads + tid; i < n_rows * (D / 4); i += (int)gridDim.z * kRowsThreads) {
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

template <typename T, int D>
int launch_rows(const tra_packed_ctx& c, const tra_packed_launch& a, int chunk, bool clustered) {
  constexpr auto kern = tra_packed_rows_kernel<T, D>;
  const int rc = tra_allow_smem<kern>(RowsCfg<D>::kSmemBytes);
  if (rc != TRA_OK) return rc;
  return tra_launch(kern, dim3((unsigned)a.n_seq, (unsigned)a.kv_heads, (unsigned)a.splits), kRowsThreads, RowsCfg<D>::kSmemBytes, c.stream,
                    false, clustered ? a.splits : 1, a, chunk, clustered ? 1 : 0);
}

}  // namespace
