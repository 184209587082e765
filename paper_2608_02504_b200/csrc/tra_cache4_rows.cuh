// Attention of few rows over a cache of 4 bits: one new token of every sequence (or a few), the codes turned into operands of the
// products in registers.  At most 16 rows (tokens times the heads of a group) per block; more rows take more blocks.
//
// Mathematics.  A key is k_c = m_j + s_j n_c for the channels c of group j, n = 0 .. 15, so
//   q k = sum_j (s_j sum_(c in j) q_c n_c + m_j sum_(c in j) q_c):
// the products run over the codes themselves, and steps and lowest values come in fp32 behind them (the second sum is one more product, of
// the lowest values with the queries' group sums in two or three pieces).  Likewise o_c = sum_i (p_i s_ij) n_ic + sum_i p_i m_ij: a step is
// multiplied into the probability.  Nothing is rounded to the type of the tensors on the way.
//
// A code in the low bits of a 16-bit half is the fp16 number n 2^-24, exactly (a subnormal), and one in the next four bits is 16 times
// that: so one mask takes two codes to two halves, and the factor 16 goes to the other operand (keys: channels of q) or to the
// result (values: channels of o).  All products are fp16 with fp32 sums, whatever the type of the tensors: q is scaled by a power of two per
// row that brings its largest element to 2^10, and steps and lowest values of the values by one, 2^-e, that follows the largest of them so
// far, so that fp16's range is not an issue: elements 2^-24 times the largest lose precision, which no 16-bit tensor shows.  The probabilities are
// held times 2^6 for the same reason.
//
// Bound: HBM (0.625 bytes a channel, against 2), with about 1.4 instructions per code between them.  A producer warp streams 128-key tiles
// through a ring of bulk copies (a tile is four runs of bytes); four warps take 32 keys of every tile each.
#pragma once
#include "tra_cache4.h"
#include "tra_rows_join.cuh"

namespace {

constexpr int kC4Tile = 128;              // keys per ring slot
constexpr int kC4Warps = 4;
constexpr int kC4Threads = 32 * (kC4Warps + 1);
constexpr int kC4ProbLog2 = 6;            // probabilities are held times 2^6
constexpr int kC4QLog2 = 10;              // rows of q: largest element in [2^9, 2^10)

template <int D>
struct C4Cfg {
  static constexpr int kGroups = D / kCacheGroup;
  static constexpr int kRow = D / 2, kStepRow = D / 8;                    // bytes
  static constexpr int kCodes = kC4Tile * kRow;
  static constexpr int kSteps = (kC4Tile * kStepRow + 16 + 15) / 16 * 16;   // a tile may start in the middle of 16 bytes (d 64)
  static constexpr int kStageBytes = 2 * (kCodes + kSteps);
  static constexpr int kStages = D == 128 ? 3 : 6;
  static constexpr int kSmemData = kStages * kStageBytes;
  static constexpr int kScratch = kC4Warps * 2 * kGroups * 32 * 2;        // scaled steps and lowest values of a warp's 32 values
  static constexpr int kSmemBytes = kSmemData + kScratch + 256;
};
static_assert(rows_join_bytes<128>(kC4Warps) <= C4Cfg<128>::kSmemData, "join area");
static_assert(rows_join_bytes<64>(kC4Warps) <= C4Cfg<64>::kSmemData, "join area");

struct C4Ctl {
  uint64_t full[6], empty[6];
  int abort_flag;
};
static_assert(sizeof(C4Ctl) <= 256, "control block");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Physical row, of eight, that takes part in a product as its row x: neighbours x, x + 1 then lie in rows of different parity, and so do
// 0, 2 and 4, 6, which spreads both kinds of reads over the banks (rows of 64 bytes).  Its own inverse.
__device__ __forceinline__ int c4_row(int x) { return x ^ ((x >> 1) & 1); }

// sequence = blockIdx.x, (row tile, key/value head) = blockIdx.y, part = blockIdx.z (keys [part * chunk, ...) of the key axis); chunk is a
// multiple of 128.  NT: groups of eight rows.
template <typename T, int D, int NT, bool kWindow>
__global__ void __launch_bounds__(kC4Threads, NT == 1 ? 3 : 2)
    tra_cache4_rows_kernel(const __grid_constant__ tra_cache4_launch args, int chunk, int clustered) {
  using C = C4Cfg<D>;
  constexpr int G = C::kGroups;
  const tra_packed_launch& p = args.a;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* scratch = smem + C::kSmemData;
  C4Ctl* ctl = (C4Ctl*)(smem + C::kSmemData + C::kScratch);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int seq = blockIdx.x, kvh = blockIdx.y / args.row_tiles, row0 = (blockIdx.y % args.row_tiles) * kRowsMax;
  const tra_seq_range qr = tra_clamp_range(p.cu_q[seq], p.cu_q[seq + 1], p.total_q, p.max_q, p.status);
  const tra_seq_range kr = tra_clamp_range(p.k_begin[seq], p.k_end[seq], p.total_k, p.max_k, p.status);
  const bool parts = gridDim.z > 1 && !clustered;
  if (parts) allow_next_launch();                            // the join of the parts
  const int n_rows = min(qr.len * p.group - row0, kRowsMax);
  if (n_rows <= 0) return;
  const int ahead = kr.len - qr.len;
  const int tok0 = row0 / p.group, tok1 = (row0 + n_rows - 1) / p.group;        // tokens of this tile
  // (sink_rows is a multiple of the tile here: a tile holds first tokens or the window's)
  const tra_key_axis<kWindow ? kOrderWindow : kOrderCausal> axis(p, ahead + tok0, kr.len);
  const int walk = p.order ? min(max(tok1 + 1 + ahead - axis.gap, 0), axis.len) : kr.len;       // keys that the last token sees
  const int key0 = (int)blockIdx.z * chunk, key1 = min(key0 + chunk, walk);
  const int n_tiles = key1 > key0 ? (key1 - key0 + kC4Tile - 1) / kC4Tile : 0;
  auto row_token = [&](int r) -> long long { return qr.begin + (row0 + r) / p.group; };
  auto row_head = [&](int r) -> int { return kvh * p.group + (row0 + r) % p.group; };

  if (n_tiles == 0 && parts) {                               // nothing here: the join skips the part
    if (tid < n_rows) {
      const long long row = (long long)blockIdx.z * p.total_q * p.heads + row_token(tid) * p.heads + row_head(tid);
      p.part_lse2[row] = -INFINITY;
      if (p.part_exact) p.part_exact[row] = -INFINITY;
    }
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(smem_u32(&ctl->full[i]), 1);
      mbar_init(smem_u32(&ctl->empty[i]), kC4Warps);
    }
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  volatile int* abort_flag = &ctl->abort_flag;
  // Tile from axis position v on: its first row of the cache and how many rows are loaded.  Of the first tokens' tiles only those are (where
  // a gap follows, nobody sees the rows behind them).
  auto tile_row = [&](int v) -> int { return kr.begin + (kWindow && v >= p.sink_rows ? v + axis.gap : v); };
  auto tile_count = [&](int v) -> int {
    const int n = min(kC4Tile, key1 - v);
    return kWindow && axis.gap > 0 && v < p.sink_rows ? max(min(n, p.sinks - v), 0) : n;
  };

  float m[NT][2], l[NT][2], le[NT][2];                       // rows nt * 8 + 2 tig, + 1
  float o[D / 16][NT][4], om[NT][4];                         // channels 16 i + g, + 8 (times 16); groups' lowest values
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < 2; ++c) m[nt][c] = -INFINITY, l[nt][c] = le[nt][c] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      om[nt][c] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i][nt][c] = 0.f;
    }
  }
  int e_run = -120;                                          // values are held times 2^-e_run
  const int g = lane >> 2, tig = lane & 3;

  if (warp == kC4Warps) {
    if (lane == 0) {
      const long long head = (long long)kvh * p.total_k;
      int slot = 0;
      uint32_t phase = 1u;                                   // the first pass over the ring finds every slot free
      for (int t = 0; t < n_tiles; ++t) {
        if (!mbar_wait(smem_u32(&ctl->empty[slot]), phase, abort_flag, p.status)) break;
        const int v = key0 + t * kC4Tile, row = tile_row(v), n = tile_count(v);
        // d 64: rows of 8 bytes of steps, two of them per 16 (the cache holds an even number of rows)
        const int first = D == 64 ? row & ~1 : row, last = D == 64 ? (row + n + 1) & ~1 : row + n;
        const uint32_t codes = (uint32_t)n * C::kRow, steps = (uint32_t)(last - first) * C::kStepRow;
        const uint32_t bar = smem_u32(&ctl->full[slot]), dst = smem_u32(smem + slot * C::kStageBytes);
        if (n > 0) {
          mbar_expect_tx(bar, 2 * (codes + steps));
          bulk_load(dst, args.k + (head + row) * C::kRow, codes, bar);
          bulk_load(dst + 2 * C::kCodes, (const uint8_t*)args.k_step + (head + first) * C::kStepRow, steps, bar);
          bulk_load(dst + C::kCodes, args.v + (head + row) * C::kRow, codes, bar);
          bulk_load(dst + 2 * C::kCodes + C::kSteps, (const uint8_t*)args.v_step + (head + first) * C::kStepRow, steps, bar);
        } else {
          mbar_arrive(bar);
        }
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
      }
    }
  } else {
    // ---- queries as the second operand: column g of a product is row nt * 8 + g
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr int kPieces = kBf16 ? 3 : 2;                   // of the group sums, in T
    uint32_t qb[D / 16][NT][2], qs[NT][2];
    float col_mul[NT][2];
    int hi[NT][2];                                           // keys in front of it are seen by the row
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 8 + g;
      const bool there = r < n_rows;
      const T* qrow = (const T*)p.q + row_token(there ? r : 0) * p.q_stride[0] + row_head(there ? r : 0) * p.q_stride[1];
      uint32_t raw[D / 8];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        raw[i] = there ? *reinterpret_cast<const uint32_t*>(qrow + i * 8 + tig * 2) : 0u;
        float a, b;
        unpack_pair<T>(raw[i], a, b);
        top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -100), 128);       // |q| < 2^e
      const float mul = pow2i(kC4QLog2 - e);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        float sum = 0.f;
#pragma unroll
        for (int i = 4 * j; i < 4 * j + 4; ++i) {
          float a, b;
          unpack_pair<T>(raw[i], a, b);
          a *= mul, b *= mul;
          sum += a + b;
          const float f = i & 1 ? 0.0625f : 1.f;             // its codes are held times 16
          qb[i >> 1][nt][i & 1] = pack_pair<__half>(a * f, b * f);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        // piece x of group j is row x G + j of the operand: rows 2 tig, 2 tig + 1 in register 0, 8 more in register 1
        float left = sum;
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
          const int at = x * G + j;
          const uint32_t piece = pack_pair<T>(left, 0.f) & 0xffffu;
          float a, b;
          unpack_pair<T>(piece, a, b);
          left -= a;
          if (at == 0) qs[nt][0] = qs[nt][1] = 0u;
          if (((at & 7) >> 1) == tig) qs[nt][at >> 3] |= piece << ((at & 1) * 16);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        col_mul[nt][c] = p.sm_scale * kLog2e * pow2i(__shfl_sync(0xffffffffu, e, (2 * tig + c) * 4) - kC4QLog2);
        const int t = min((row0 + nt * 8 + 2 * tig + c) / p.group, tok1);
        hi[nt][c] = p.order ? min(max(t + 1 + ahead - axis.gap, 0), axis.len) : kr.len;
      }
    }
    const int hi_min = p.order ? min(max(tok0 + 1 + ahead - axis.gap, 0), axis.len) : kr.len;
    const int old_max = kWindow ? walk - p.window : 0;       // keys that have left the last token's window
    uint8_t* warp_scratch = scratch + warp * (C::kScratch / kC4Warps);
    int slot = 0;
    uint32_t phase = 0u;
    for (int t = 0; t < n_tiles; ++t) {
      if (!mbar_wait_warp(smem_u32(&ctl->full[slot]), phase, abort_flag, p.status)) break;
      const int v0 = key0 + t * kC4Tile, there = tile_count(v0), in_tile = warp * 32;
      const int k0 = v0 + in_tile;                           // axis position of this warp's first key
      if (in_tile < there) {
        const uint8_t* stage = smem + slot * C::kStageBytes;
        const int shift = D == 64 ? tile_row(v0) & 1 : 0;
        const uint8_t *kc = stage + in_tile * C::kRow, *vc = kc + C::kCodes;
        const uint8_t* ks = stage + 2 * C::kCodes + (in_tile + shift) * C::kStepRow;
        const uint8_t* vs = ks + C::kSteps;
        // ---- steps and lowest values of the values: lane = key
        {
          float x[2 * G];
          uint32_t raw[G];
          const uint8_t* at = vs + lane * C::kStepRow;
          if constexpr (G == 4) {
            const uint4 w = *reinterpret_cast<const uint4*>(at);
            raw[0] = w.x, raw[1] = w.y, raw[2] = w.z, raw[3] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(at);
            raw[0] = w.x, raw[1] = w.y;
          }
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < G; ++i) {
            if (in_tile + lane >= there) raw[i] = 0u;        // behind the sequence's end: anything
            unpack_pair<T>(raw[i], x[2 * i], x[2 * i + 1]);
            const float f = i < G / 2 ? 16.f : 1.f;
            top = fmaxf(top, f * fmaxf(fabsf(x[2 * i]), fabsf(x[2 * i + 1])));
          }
          const int e = min((int)(__reduce_max_sync(0xffffffffu, __float_as_uint(top)) >> 23) - 126, 126);     // all below 2^e
          if (e > e_run) {
            const float f = ex2((float)(e_run - e));
            e_run = e;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                om[nt][c] *= f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[i][nt][c] *= f;
              }
          }
          const float mul = pow2i(-e_run);
          const int r = lane & 7, logical = c4_row(r), half = (lane >> 3) & 1, sub = lane >> 4;
          __half* dst = (__half*)warp_scratch + (sub * 4 + (logical >> 1)) * 4 + half * 2 + (logical & 1);
#pragma unroll
          for (int i = 0; i < 2 * G; ++i) dst[i * 32] = __float2half_rn(x[i] * (i < G ? 16.f * mul : mul));
          __syncwarp();
        }
        uint32_t pb[2][NT][2];                               // probabilities as the second operand: [16 keys][rows]
        float s[2][NT][4];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int r0 = sub * 16 + c4_row(g), r1 = r0 + 8;
          // the lowest values' share
          uint32_t am[4];
          {
            constexpr int kPairs = G / 2;
            const int pair = tig % kPairs;
            am[0] = *reinterpret_cast<const uint32_t*>(ks + r0 * C::kStepRow + G * 2 + pair * 4);
            am[1] = *reinterpret_cast<const uint32_t*>(ks + r1 * C::kStepRow + G * 2 + pair * 4);
            am[2] = am[0], am[3] = am[1];
          }
          float st[2][G];
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < G / 2; ++i)
              unpack_pair<T>(*reinterpret_cast<const uint32_t*>(ks + (half ? r1 : r0) * C::kStepRow + i * 4), st[half][2 * i], st[half][2 * i + 1]);
          uint32_t w[2][G];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint8_t* at = kc + (half ? r1 : r0) * C::kRow + tig * (G * 4);
            if constexpr (G == 4) {
              const uint4 x = *reinterpret_cast<const uint4*>(at);
              w[half][0] = x.x, w[half][1] = x.y, w[half][2] = x.z, w[half][3] = x.w;
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(at);
              w[half][0] = x.x, w[half][1] = x.y;
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816<T>(c, am, qs[nt][0], qs[nt][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[sub][nt][i] = c[i] * 0x1p-24f;
          }
#pragma unroll
          for (int j = 0; j < G; ++j) {
            const uint32_t a0[4] = {w[0][j] & 0x000f000fu, w[1][j] & 0x000f000fu, w[0][j] & 0x00f000f0u, w[1][j] & 0x00f000f0u};
            const uint32_t h0 = w[0][j] >> 8, h1 = w[1][j] >> 8;
            const uint32_t a1[4] = {h0 & 0x000f000fu, h1 & 0x000f000fu, h0 & 0x00f000f0u, h1 & 0x00f000f0u};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float c[4] = {0.f, 0.f, 0.f, 0.f};
              mma16816<__half>(c, a0, qb[2 * j][nt][0], qb[2 * j][nt][1]);
              mma16816<__half>(c, a1, qb[2 * j + 1][nt][0], qb[2 * j + 1][nt][1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[sub][nt][i] = fmaf(st[i >> 1][j], c[i], s[sub][nt][i]);
            }
          }
          // scores in base 2: the codes' factor 2^24 and the row's own
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[sub][nt][i] *= 0x1p24f * col_mul[nt][i & 1];
          const int v = k0 + sub * 16 + c4_row(g);
          if (k0 + 32 > min(hi_min, key1) || in_tile + 32 > there) {
            const int end = min(key1, v0 + there);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (v + (i >> 1) * 8 >= min(hi[nt][i & 1], end)) s[sub][nt][i] = -INFINITY;
          }
          if (kWindow && k0 < old_max && k0 + 32 > p.sinks) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int x = v + (i >> 1) * 8;
                if (x < hi[nt][i & 1] - p.window && x >= p.sinks) s[sub][nt][i] = -INFINITY;
              }
          }
        }
        // ---- probabilities
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mx = fmaxf(fmaxf(s[0][nt][c], s[0][nt][c + 2]), fmaxf(s[1][nt][c], s[1][nt][c + 2]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            // exact whatever the reference is, as long as all terms share it: raised only when it is 8 (2^8) behind
            if (mx > m[nt][c] + kRescaleThreshold) {
              const float alpha = ex2(m[nt][c] - mx);
              l[nt][c] *= alpha;
              le[nt][c] *= alpha;
              m[nt][c] = mx;
#pragma unroll
              for (int i = 0; i < D / 16; ++i) {
                o[i][nt][c] *= alpha;
                o[i][nt][c + 2] *= alpha;
              }
              om[nt][c] *= alpha;
            }
          }
          const float ref[2] = {m[nt][0] > -INFINITY ? m[nt][0] - kC4ProbLog2 : 0.f, m[nt][1] > -INFINITY ? m[nt][1] - kC4ProbLog2 : 0.f};
#pragma unroll
          for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float x0 = ex2(s[sub][nt][2 * half] - ref[0]), x1 = ex2(s[sub][nt][2 * half + 1] - ref[1]);
              le[nt][0] += x0;
              le[nt][1] += x1;
              const uint32_t packed = pack_pair<__half>(x0, x1);
              add_pair<__half>(l[nt][0], l[nt][1], packed);  // the sum that divides O: of the rounded probabilities
              pb[sub][nt][half] = transpose8x8(packed);
            }
        }
        // ---- values
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int r0 = sub * 16 + c4_row(2 * tig), r1 = sub * 16 + c4_row(2 * tig + 1);
          const uint8_t* sc = warp_scratch + (sub * 4 + tig) * 8;
          {
            uint2 x = make_uint2(0u, 0u);
            if (g < G) x = *reinterpret_cast<const uint2*>(sc + (G + g) * 64);
            const uint32_t a[4] = {x.x, 0u, x.y, 0u};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816<__half>(om[nt], a, pb[sub][nt][0], pb[sub][nt][1]);
          }
          uint32_t w[4][G / 2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint8_t* at = vc + ((i & 1 ? r1 : r0) + (i >> 1) * 8) * C::kRow + g * (G * 2);
            if constexpr (G == 4) {
              const uint2 x = *reinterpret_cast<const uint2*>(at);
              w[i][0] = x.x, w[i][1] = x.y;
            } else {
              w[i][0] = *reinterpret_cast<const uint32_t*>(at);
            }
          }
#pragma unroll
          for (int j = 0; j < G; ++j) {
            // the four codes of group j in two neighbouring keys, side by side
            const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
            const uint32_t x = __byte_perm(w[0][j >> 1], w[1][j >> 1], sel), y = __byte_perm(w[2][j >> 1], w[3][j >> 1], sel);
            const uint32_t xh = x >> 8, yh = y >> 8;
            const uint32_t a0[4] = {x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
            const uint32_t a1[4] = {xh & 0x000f000fu, xh & 0x00f000f0u, yh & 0x000f000fu, yh & 0x00f000f0u};
            const uint2 step = *reinterpret_cast<const uint2*>(sc + j * 64);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint32_t b0 = mul_half2(pb[sub][nt][0], step.x), b1 = mul_half2(pb[sub][nt][1], step.y);
              mma16816<__half>(o[2 * j][nt], a0, b0, b1);
              mma16816<__half>(o[2 * j + 1][nt], a1, b0, b1);
            }
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
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 4; i < 32; i <<= 1) {
          l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], i);
          le[nt][c] += __shfl_xor_sync(0xffffffffu, le[nt][c], i);
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
  rows_join<T, D, kC4Warps>(p, {qr, kvh, row0, n_rows, parts, clustered != 0}, (float*)smem, [&](float* part, float* stat) {
    const float f = pow2i(e_run);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = nt * 8 + 2 * tig + c;
        float* dst = part + (warp * kRowsMax + r) * D;
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const float low = __shfl_sync(0xffffffffu, om[nt][c], j * 4 + tig) * f;      // of group j
#pragma unroll
          for (int i = 2 * j; i < 2 * j + 2; ++i) {
            dst[i * 16 + g] = fmaf(o[i][nt][c] * 0x1p20f, f, low);      // codes 2^24, steps 2^-4
            dst[i * 16 + g + 8] = fmaf(o[i][nt][c + 2] * 0x1p16f, f, low);
          }
        }
        if (g == 0) {
          float* st = stat + (warp * kRowsMax + r) * 4;
          st[0] = m[nt][c] - kC4ProbLog2;
          st[1] = gave_up ? 0.f : l[nt][c];
          st[2] = le[nt][c];
        }
      }
  });
}

template <typename T, int D, int NT, bool kWindow>
int launch_cache4_kernel(const tra_packed_ctx& c, const tra_cache4_launch& a, int chunk, bool clustered) {
  constexpr auto kern = tra_cache4_rows_kernel<T, D, NT, kWindow>;
  const int rc = tra_allow_smem<kern>(C4Cfg<D>::kSmemBytes);
  if (rc != TRA_OK) return rc;
  return tra_launch(kern, dim3((unsigned)a.a.n_seq, (unsigned)(a.a.kv_heads * a.row_tiles), (unsigned)a.a.splits), kC4Threads, C4Cfg<D>::kSmemBytes,
                    c.stream, false, clustered ? a.a.splits : 1, a, chunk, clustered ? 1 : 0);
}

template <typename T, int D>
int launch_cache4(const tra_packed_ctx& c, const tra_cache4_launch& a, int chunk, bool clustered) {
  const bool narrow = (long long)a.a.max_q * a.a.group <= 8, window = a.a.order == kOrderWindow;
  if (window)
    return narrow ? launch_cache4_kernel<T, D, 1, true>(c, a, chunk, clustered) : launch_cache4_kernel<T, D, 2, true>(c, a, chunk, clustered);
  return narrow ? launch_cache4_kernel<T, D, 1, false>(c, a, chunk, clustered) : launch_cache4_kernel<T, D, 2, false>(c, a, chunk, clustered);
}

}  // namespace
