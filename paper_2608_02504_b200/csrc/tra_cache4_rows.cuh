// Attention of few rows over a cache of 4 bits: one new token of every sequence (or a few), the codes turned into operands of the
// products in registers.  At most 16 rows (tokens times the heads of a group) per block; more rows take more blocks.
//
// Mathematics.  A key is k_c = low_j + step_j n_c for the channels c of group j, n = 0 .. 15, so
//   q k = sum_j (step_j sum_(c in j) q_c n_c + low_j sum_(c in j) q_c):
// the products run over the codes themselves, and the steps come in fp32 behind them (the second sum is one more product, of the lowest
// values with the queries' group sums in two or three pieces).  A value is mid_j + step_j (n_c - 8), mid = low + 8 step, so
//   o_c = sum_i (p_i step_ij) n_ic - 8 sum_i (p_i step_ij) + sum_i p_i mid_ij:
// the steps go to the probabilities, the second sum is a product with a constant, into the first one's registers every 16 keys, and the last, the same
// for the channels of a group, is one product for all groups.
//
// Rounding.  p step is rounded to fp16, once, and meets n - 8, which is as large as what a value differs from its group's middle: that is
// the rounding of the probabilities of any attention kernel.  (Probabilities rounded first and multiplied by the steps in fp16, against n and
// low: 4.5e-4 off on a cache of 777 fp16 keys, where rounding the result alone makes 2.0e-4; so: 2.8e-4.)  p mid has p rounded to fp16.  Everything
// else is exact or fp32.  The sums of n and of 8 are taken off each other as they grow: of two sums of their own over 20,000 keys the difference
// is a hundredth, and the tensor pipe's truncated additions show in it (4.0e-4 against 2.8e-4).
//
// A code in the low bits of a 16-bit half is the fp16 number n 2^-24, exactly (a subnormal), and one in the next four bits is 16 times
// that: so one mask takes two codes to two halves, and the factor 16 goes to the other operand (keys: channels of q) or to the
// result (values: channels of o).  All products are fp16 with fp32 sums, whatever the type of the tensors: q is scaled by a power of two per
// row that brings its largest element to 2^15 (bf16 elements keep their 8 bits down to 2^-28 of it, fp16 ones their 11 down to 2^-25; from 2^10 a group of
// fp16 queries 2^-20 of another, on keys as much larger, took o 1.1e-3 off, from 2^15 2.5e-4, as if all were alike), and steps and middles of the values by one that follows the largest value so far (of a
// warp's keys, all groups), 2^e above it: the range 15 step is below 2 2^e, so that 8 steps are held below 16 / 15, for their products with
// probabilities of up to 2^15, and middles below 2^15.  So middles keep 11 bits down to 2^-29 of 2^e, which covers fp16's normal numbers beside values of up
// to 2^15; bf16 values further apart than that lose bits.  (Middles held below 1.5: values of 0.01 were 0.08 to 0.25 of their norm off beside one of 6e4 that the
// order hides; so: 2.8e-4, where the result's rounding alone makes 2.0e-4.)
//
// Bound: instruction issue and latency beside HBM (0.625 bytes a channel, against 2): 702 instructions per 32 keys of a head, of which a third
// turns codes into operands; at the rate at which HBM delivers them, an SM would have to issue 3.3 of its 4 per cycle, and issues 2.3.  A
// block is four warps that each walk pieces of 32 keys, every fourth one, through a ring of bulk copies of their own (a piece is four runs
// of bytes): no warp waits for another before the join.  64 caches of 700 to 32,768 keys, 40 / 8 heads, d 128: 333 us, 4.1 TB/s (63 % of the copy rate; the cache
// in 16 bits: 646 us).  History: codes as operands with P multiplied in fp16, a producer warp, two clustered parts 424; the rounding above, a ring per warp
// 561; parts without clusters 334; queries in shared memory 326; the sums of 8 in the others' registers 338.  Four blocks an SM in 128 registers (748 instructions) or the ring's slots unrolled
// (745): 1 to 2 % less, and 10 to 15 % more for short caches.
#pragma once
#include "tra_cache4.h"
#include "tra_rows_join.cuh"

namespace {

constexpr int kC4Piece = 32;              // keys of a ring slot: one per lane
constexpr int kC4Warps = 4;
constexpr int kC4Threads = 32 * kC4Warps;
constexpr int kC4Tile = kC4Piece * kC4Warps;
// Probabilities are at most 2^kC4Above and held times 2^kC4ProbLog2: below 2^15, and in full precision down to 2^-27 for the largest steps.  (2^8 and
// 2^6: 4.2e-4 off over 20,000 fp16 keys, most of whose probabilities were subnormal; so: 2.8e-4.)
constexpr int kC4ProbLog2 = 13;
constexpr float kC4Above = 2.f;
constexpr int kC4MidLog2 = 15, kC4StepLog2 = 3;        // middles and steps of the values: see above
constexpr int kC4QLog2 = 15;              // rows of q: largest element in [2^14, 2^15)

template <int D>
struct C4Cfg {
  static constexpr int kGroups = D / kCacheGroup;
  static constexpr int kRow = D / 2, kStepRow = D / 8;                    // bytes
  static constexpr int kCodes = kC4Piece * kRow;
  static constexpr int kSteps = kC4Piece * kStepRow + 16;                 // a piece may start in the middle of 16 bytes (d 64)
  static constexpr int kStageBytes = 2 * (kCodes + kSteps);
  static constexpr int kStages = D == 128 ? 3 : 4;
  static constexpr int kRing = kStages * kStageBytes;                     // of a warp
  // a warp's steps in fp32, [32 keys][groups] of the keys and of the values, and middles in fp16, [groups][32 keys]
  static constexpr int kScratch = kC4Piece * kGroups * (4 + 4 + 2);
  static constexpr int kQueries = D / 16 * 8 * 32;                        // of eight rows: two registers per 16 channels and lane
  static constexpr int kSmemData = kC4Warps * (kRing + kScratch) + 2 * kQueries;
  static constexpr int kSmemBytes = kSmemData + 256;
};
static_assert(rows_join_bytes<128>(kC4Warps) <= C4Cfg<128>::kSmemData, "join area");
static_assert(rows_join_bytes<64>(kC4Warps) <= C4Cfg<64>::kSmemData, "join area");

struct C4Ctl {
  uint64_t full[kC4Warps][4];
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
__device__ __forceinline__ uint32_t sub_half2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Codes to operands: of the four codes in either half of x, those of bits 0 and 4 and those of bits 8 and 12 (the second of a pair times
// 16).  The low code of the upper byte is what is left of the byte, an fp16 number itself: a subtraction on the pipe that has less to do.
__device__ __forceinline__ void low_codes(uint32_t x, uint32_t& c0, uint32_t& c1) {
  c0 = x & 0x000f000fu;
  c1 = x & 0x00f000f0u;
}
__device__ __forceinline__ void high_codes(uint32_t x, uint32_t& c0, uint32_t& c1) {
  const uint32_t bytes = __byte_perm(x, 0u, 0x4341);
  c1 = bytes & 0x00f000f0u;
  c0 = sub_half2(bytes, c1);
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Physical row, of eight, that takes part in a product as its row x: neighbours x, x + 1 then lie in rows of different parity, and so do
// 0, 2 and 4, 6, which spreads both kinds of reads over the banks (rows of 64 bytes).  Its own inverse.
__device__ __forceinline__ int c4_row(int x) { return x ^ ((x >> 1) & 1); }

// sequence = blockIdx.x, (row tile, key/value head) = blockIdx.y, part = blockIdx.z (keys [part * chunk, ...) of the key axis); chunk is a
// multiple of 128.  NB: groups of eight rows.
template <typename T, int D, int NB, bool kWindow>
__global__ void __launch_bounds__(kC4Threads, NB == 1 ? 3 : 2)
    tra_cache4_rows_kernel(const __grid_constant__ tra_cache4_launch args, int chunk, int clustered) {
  using C = C4Cfg<D>;
  constexpr int G = C::kGroups;
  const tra_packed_launch& p = args.a;
  extern __shared__ __align__(128) uint8_t smem[];
  C4Ctl* ctl = (C4Ctl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* ring = smem + warp * C::kRing;
  float* k_step = (float*)(smem + kC4Warps * C::kRing + warp * C::kScratch);
  float* v_step = k_step + kC4Piece * G;
  __half* v_mid = (__half*)(v_step + kC4Piece * G);
  uint4* queries = (uint4*)(smem + kC4Warps * (C::kRing + C::kScratch));      // [rows / 8][32 channels][lane]
  const int seq = blockIdx.x, kvh = blockIdx.y / args.row_tiles, row0 = (blockIdx.y % args.row_tiles) * kRowsMax;
  const tra_seq_range qr = tra_clamp_range(p.cu_q[seq], p.cu_q[seq + 1], p.total_q, p.max_q, p.status);
  const tra_seq_range kr = tra_clamp_range(p.k_begin[seq], p.k_end[seq], p.total_k, p.max_k, p.status);
  const bool parts = gridDim.z > 1 && !clustered;
  if (parts) allow_next_launch();                            // the join of the parts
  const int n_rows = min(qr.len * p.group - row0, kRowsMax);
  if (n_rows <= 0) return;
  const int ahead = kr.len - qr.len;
  const int tok0 = row0 / p.group, tok1 = (row0 + n_rows - 1) / p.group;        // tokens of this tile
  // (sink_rows is a multiple of a piece here: a piece holds first tokens or the window's)
  const tra_key_axis<kWindow ? kOrderWindow : kOrderCausal> axis(p, ahead + tok0, kr.len);
  const int walk = p.order ? min(max(tok1 + 1 + ahead - axis.gap, 0), axis.len) : kr.len;       // keys that the last token sees
  const int key0 = (int)blockIdx.z * chunk, key1 = min(key0 + chunk, walk);
  auto row_token = [&](int r) -> long long { return qr.begin + (row0 + r) / p.group; };
  auto row_head = [&](int r) -> int { return kvh * p.group + (row0 + r) % p.group; };

  if (key1 <= key0 && parts) {                               // nothing here: the join skips the part
    if (tid < n_rows) {
      const long long row = (long long)blockIdx.z * p.total_q * p.heads + row_token(tid) * p.heads + row_head(tid);
      p.part_lse2[row] = -INFINITY;
      if (p.part_exact) p.part_exact[row] = -INFINITY;
    }
    return;
  }
  if (tid == 0) ctl->abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(smem_u32(&ctl->full[warp][i]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  volatile int* abort_flag = &ctl->abort_flag;
  // Piece from axis position v on: its first row of the cache and how many rows are loaded.  Of the first tokens' pieces only those are (where
  // a gap follows, nobody sees the rows behind them).
  auto piece_row = [&](int v) -> int { return kr.begin + (kWindow && v >= p.sink_rows ? v + axis.gap : v); };
  auto piece_count = [&](int v) -> int {
    const int n = min(kC4Piece, key1 - v);
    return kWindow && axis.gap > 0 && v < p.sink_rows ? min(n, p.sinks - v) : n;
  };
  const int first_piece = key0 + warp * kC4Piece;
  const int n_pieces = key1 > first_piece ? (key1 - first_piece + kC4Tile - 1) / kC4Tile : 0;
  // Lanes 0 .. 3 issue a copy each: codes of keys, of values, steps of keys, of values.
  const bool of_steps = lane & 2;
  const uint8_t* src = (lane & 1) ? (of_steps ? (const uint8_t*)args.v_step : args.v) : (of_steps ? (const uint8_t*)args.k_step : args.k);
  src += (long long)kvh * p.total_k * (of_steps ? C::kStepRow : C::kRow);
  const uint32_t dst = smem_u32(ring) + (of_steps ? 2 * C::kCodes + (lane & 1) * C::kSteps : (lane & 1) * C::kCodes);
  const uint32_t row_bytes = of_steps ? C::kStepRow : C::kRow;
  const uint32_t bars = smem_u32(&ctl->full[warp][0]);
  auto load_piece = [&](int i, int slot) {
    const int v = first_piece + i * kC4Tile, n = piece_count(v);
    int row = piece_row(v), count = n;
    uint32_t bytes = (uint32_t)n * (2 * (C::kRow + C::kStepRow));
    if (D == 64) {                                           // rows of 8 bytes of steps, two of them per 16 (the cache holds an even number of rows)
      const int first = row & ~1, more = ((row + n + 1) & ~1) - first;
      bytes += (uint32_t)(more - n) * (2 * C::kStepRow);
      if (of_steps) row = first, count = more;
    }
    const uint32_t bar = bars + slot * 8;
    if (n <= 0) {
      if (lane == 0) mbar_arrive(bar);
    } else {
      if (lane == 0) mbar_expect_tx(bar, bytes);
      __syncwarp();
      if (lane < 4) bulk_load(dst + slot * C::kStageBytes, src + (long long)row * row_bytes, count * row_bytes, bar);
    }
  };
  for (int i = 0; i < C::kStages && i < n_pieces; ++i) load_piece(i, i);

  const int g = lane >> 2, tig = lane & 3;
  float m[NB][2], l[NB][2];                                  // rows 8 nb + 2 tig, + 1
  float o[D / 16][NB][4], om[NB][4];                         // [channels 16 i + g, + 8 (times 16)][rows 8 nb + 2 tig, + 1]; groups' share
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
    for (int c = 0; c < 2; ++c) m[nb][c] = -INFINITY, l[nb][c] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      om[nb][c] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i][nb][c] = 0.f;
    }
  }
  int e_run = -111;                                          // middles are held times 2^(15 - e_run), steps times 2^(3 - e_run)

  // ---- queries as the second operand: column g of a product is row 8 nb + g
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  constexpr int kPieces = kBf16 ? 3 : 2;                     // of the group sums, in T
  // Their products with the lowest values join those with the codes, which are held times 2^-24.  fp16: sums of up to 2^20 are brought into its range.  bf16:
  // times 2^-23 no lowest value takes a product past fp32 (times 2^-24 the loop has one factor less and the compiler lays it out worse: 335 us for 333).
  constexpr float kSumMul = kBf16 ? 0x1p-23f : 0x1p-5f, kLowMul = 0x1p-24f / kSumMul;
  // (in shared memory: registers are what limits the blocks of an SM)
  uint32_t qs[NB][2];
  float row_mul[NB][2];                                      // to scores in base 2, codes' factor 2^24 included
  int hi[NB][2];                                             // keys in front of it are seen by the row
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = nb * 8 + g;
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
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -110), 128);       // |q| < 2^e
    const float mul = pow2i(kC4QLog2 - e);
    qs[nb][0] = qs[nb][1] = 0u;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      float sum = 0.f;
      uint32_t qb[4];
#pragma unroll
      for (int i = 4 * j; i < 4 * j + 4; ++i) {
        float a, b;
        unpack_pair<T>(raw[i], a, b);
        a *= mul, b *= mul;
        sum += a + b;
        const float f = i & 1 ? 0.0625f : 1.f;               // its codes are held times 16
        qb[i & 3] = pack_pair<__half>(a * f, b * f);
      }
      if (warp == 0) queries[(nb * G + j) * 32 + lane] = make_uint4(qb[0], qb[1], qb[2], qb[3]);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      // piece x of group j is row x G + j of the operand: rows 2 tig, 2 tig + 1 in one register, 8 more in the other
      float left = sum * kSumMul;
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        const int at = x * G + j;
        const uint32_t piece = pack_pair<T>(left, 0.f) & 0xffffu;
        float a, b;
        unpack_pair<T>(piece, a, b);
        left -= a;
        if (((at & 7) >> 1) == tig) qs[nb][at >> 3] |= piece << ((at & 1) * 16);
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      // (never 0, which would make NaN of masked keys: products are below 2^128; nor infinite, which would of scores of 0)
      const float mul_c = p.sm_scale * kLog2e * 0x1p24f * pow2i(__shfl_sync(0xffffffffu, e, (2 * tig + c) * 4) - kC4QLog2);
      row_mul[nb][c] = fminf(fmaxf(mul_c, 0x1p-149f), 0x1.fffffep127f);
      const int tok = min((row0 + nb * 8 + 2 * tig + c) / p.group, tok1);
      hi[nb][c] = p.order ? min(max(tok + 1 + ahead - axis.gap, 0), axis.len) : kr.len;
    }
  }
  const int hi_min = p.order ? min(max(tok0 + 1 + ahead - axis.gap, 0), axis.len) : kr.len;
  const int old_max = kWindow ? walk - p.window : 0;         // keys that have left the last token's window
  const uint32_t eight[4] = {0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u};        // -8 2^-24, and 16 times that
  auto scale_sums = [&](float f0, float f1, int nb) {
    om[nb][0] *= f0, om[nb][1] *= f1;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i][nb][0] *= f0, o[i][nb][1] *= f1, o[i][nb][2] *= f0, o[i][nb][3] *= f1;
  };

  __syncthreads();                                           // the queries are there
  int slot = 0;
  uint32_t phase = 0u;
#pragma unroll 1
  for (int piece = 0; piece < n_pieces; ++piece) {
    if (!mbar_wait_warp(smem_u32(&ctl->full[warp][slot]), phase, abort_flag, p.status)) break;
    const int k0 = first_piece + piece * kC4Tile, there = piece_count(k0);        // axis position of the first key; keys
    if (there > 0) {
      const uint8_t* kc = ring + slot * C::kStageBytes;
      const uint8_t* vc = kc + C::kCodes;
      const uint8_t* ks = kc + 2 * C::kCodes + (D == 64 ? (piece_row(k0) & 1) * C::kStepRow : 0);
      const uint8_t* vs = ks + C::kSteps;
      // ---- steps and lowest values, lane = key: what the lanes need of each other's keys goes through scratch
      {
        uint32_t kw[G / 2], vw[G];
        if constexpr (G == 4) {
          const uint2 a = *reinterpret_cast<const uint2*>(ks + lane * 16);
          const uint4 b = *reinterpret_cast<const uint4*>(vs + lane * 16);
          kw[0] = a.x, kw[1] = a.y;
          vw[0] = b.x, vw[1] = b.y, vw[2] = b.z, vw[3] = b.w;
        } else {
          const uint2 b = *reinterpret_cast<const uint2*>(vs + lane * 8);
          kw[0] = *reinterpret_cast<const uint32_t*>(ks + lane * 8);
          vw[0] = b.x, vw[1] = b.y;
        }
        float kf[G], st[G], mid[G], top = 0.f;
#pragma unroll
        for (int i = 0; i < G / 2; ++i) {
          unpack_pair<T>(kw[i], kf[2 * i], kf[2 * i + 1]);
          const bool in = lane < there;                      // behind the last key: anything
          unpack_pair<T>(in ? vw[i] : 0u, st[2 * i], st[2 * i + 1]);
          unpack_pair<T>(in ? vw[G / 2 + i] : 0u, mid[2 * i], mid[2 * i + 1]);
        }
#pragma unroll
        for (int j = 0; j < G; ++j) {
          top = fmax3(top, fabsf(mid[j]), fabsf(fmaf(st[j], 15.f, mid[j])));        // lowest and largest value (infinite: 2^128)
          mid[j] = fmaf(st[j], 8.f, mid[j]);                 // low + 8 step
          st[j] = fmaxf(st[j], 0.f);                         // NaN (a group that is not finite) stays in the middle alone
        }
        const int e = min((int)(__reduce_max_sync(0xffffffffu, __float_as_uint(top)) >> 23) - 126, 128);       // all below 2^e
        if (e > e_run) {
          const float f = ex2((float)(e_run - e));
          e_run = e;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) scale_sums(f, f, nb);
        }
        const float mul = pow2i(kC4StepLog2 - e_run), mul_mid = pow2i(kC4MidLog2 - e_run);
        const int r = lane & 7, logical = c4_row(r), half = (lane >> 3) & 1, sub = lane >> 4;
        __half* mid_at = v_mid + (sub * 4 + (logical >> 1)) * 4 + half * 2 + (logical & 1);
#pragma unroll
        for (int j = 0; j < G; ++j) {
          st[j] *= mul;
          mid_at[j * kC4Piece] = __float2half_rn(mid[j] * mul_mid);
        }
        // in the order of the products' rows
        const int at = ((lane & ~7) + logical) * G;
        if constexpr (G == 4) {
          *reinterpret_cast<float4*>(k_step + at) = make_float4(kf[0], kf[1], kf[2], kf[3]);
          *reinterpret_cast<float4*>(v_step + at) = make_float4(st[0], st[1], st[2], st[3]);
        } else {
          *reinterpret_cast<float2*>(k_step + at) = make_float2(kf[0], kf[1]);
          *reinterpret_cast<float2*>(v_step + at) = make_float2(st[0], st[1]);
        }
        __syncwarp();
      }
      // ---- scores: s[sub][nb][i] = key 16 sub + g + 8 (i / 2) (of the products' order), row 8 nb + 2 tig + i % 2
      float s[2][NB][4];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int r0 = sub * 16 + c4_row(g), r1 = r0 + 8;
        uint32_t w[2][G];
        float st[2][G];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint8_t* at = kc + (half ? r1 : r0) * C::kRow + tig * (G * 4);
          const float* step_at = k_step + (sub * 16 + half * 8 + g) * G;
          if constexpr (G == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(at);
            w[half][0] = x.x, w[half][1] = x.y, w[half][2] = x.z, w[half][3] = x.w;
            const float4 y = *reinterpret_cast<const float4*>(step_at);
            st[half][0] = y.x, st[half][1] = y.y, st[half][2] = y.z, st[half][3] = y.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            w[half][0] = x.x, w[half][1] = x.y;
            const float2 y = *reinterpret_cast<const float2*>(step_at);
            st[half][0] = y.x, st[half][1] = y.y;
          }
        }
        {
          const uint8_t* at = ks + G * 2 + (tig % (G / 2)) * 4;
          const uint32_t low0 = *reinterpret_cast<const uint32_t*>(at + r0 * C::kStepRow), low1 = *reinterpret_cast<const uint32_t*>(at + r1 * C::kStepRow);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            mma1688<T>(c, low0, low1, qs[nb][0]);
            if (kPieces * G > 8) mma1688<T>(c, low0, low1, qs[nb][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[sub][nb][i] = c[i] * kLowMul;
          }
        }
#pragma unroll
        for (int j = 0; j < G; ++j) {
          uint32_t a0[4], a1[4];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            low_codes(w[half][j], a0[half], a0[half + 2]);
            high_codes(w[half][j], a1[half], a1[half + 2]);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float c[4];
            const uint4 q = queries[(nb * G + j) * 32 + lane];
            mma16816_first<__half>(c, a0, q.x, q.y);
            mma16816<__half>(c, a1, q.z, q.w);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[sub][nb][i] = fmaf(st[i >> 1][j], c[i], s[sub][nb][i]);
          }
        }
      }
      if (k0 + kC4Piece > min(hi_min, key1) || there < kC4Piece) {
        const int end = k0 + there;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (k0 + sub * 16 + (i >> 1) * 8 + c4_row(g) >= min(hi[nb][i & 1], end)) s[sub][nb][i] = -INFINITY;
      }
      if (kWindow && k0 < old_max && k0 + kC4Piece > p.sinks) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int v = k0 + sub * 16 + (i >> 1) * 8 + c4_row(g);
              if (v < hi[nb][i & 1] - p.window && v >= p.sinks) s[sub][nb][i] = -INFINITY;
            }
      }
      // ---- probabilities
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float mx[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          mx[c] = fmaxf(fmaxf(s[0][nb][c], s[0][nb][c + 2]), fmaxf(s[1][nb][c], s[1][nb][c + 2]));
          mx[c] = fmaxf(mx[c], __shfl_xor_sync(0xffffffffu, mx[c], 4));
          mx[c] = fmaxf(mx[c], __shfl_xor_sync(0xffffffffu, mx[c], 8));
          mx[c] = fmaxf(mx[c], __shfl_xor_sync(0xffffffffu, mx[c], 16)) * row_mul[nb][c];
        }
        // exact whatever the reference is, as long as all terms share it: raised only when it is kC4Above behind
        if (mx[0] > m[nb][0] + kC4Above || mx[1] > m[nb][1] + kC4Above) {
          float alpha[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float top = fmaxf(m[nb][c], mx[c]);
            alpha[c] = top > -INFINITY ? ex2(m[nb][c] - top) : 1.f;
            m[nb][c] = top;
            l[nb][c] *= alpha[c];
          }
          scale_sums(alpha[0], alpha[1], nb);
        }
        const float neg_ref[2] = {m[nb][0] > -INFINITY ? kC4ProbLog2 - m[nb][0] : 0.f, m[nb][1] > -INFINITY ? kC4ProbLog2 - m[nb][1] : 0.f};
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[sub][nb][i] = ex2(fmaf(s[sub][nb][i], row_mul[nb][i & 1], neg_ref[i & 1]));
            l[nb][i & 1] += s[sub][nb][i];
          }
      }
      // ---- values
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        uint32_t w[4][G / 2];                                // keys 2 tig, + 1, 2 tig + 8, + 9
        const int r0 = sub * 16 + c4_row(2 * tig), r1 = sub * 16 + c4_row(2 * tig + 1);
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
        float st[2][G];                                      // keys g, g + 8
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float* at = v_step + (sub * 16 + half * 8 + g) * G;
          if constexpr (G == 4) {
            const float4 y = *reinterpret_cast<const float4*>(at);
            st[half][0] = y.x, st[half][1] = y.y, st[half][2] = y.z, st[half][3] = y.w;
          } else {
            const float2 y = *reinterpret_cast<const float2*>(at);
            st[half][0] = y.x, st[half][1] = y.y;
          }
        }
        {
          // (rows from 8 on are nobody's: any group's middles do, and so they do for the rows behind the last group)
          const uint2 v = *reinterpret_cast<const uint2*>(v_mid + (g % G) * kC4Piece + (sub * 4 + tig) * 4);
          const uint32_t a[4] = {v.x, v.x, v.y, v.y};
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float* x = s[sub][nb];
            mma16816<__half>(om[nb], a, transpose8x8(pack_pair<__half>(x[0], x[1])), transpose8x8(pack_pair<__half>(x[2], x[3])));
          }
        }
#pragma unroll
        for (int j = 0; j < G; ++j) {
          // the four codes of group j in two neighbouring keys, side by side
          const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
          const uint32_t x = __byte_perm(w[0][j >> 1], w[1][j >> 1], sel), y = __byte_perm(w[2][j >> 1], w[3][j >> 1], sel);
          uint32_t a0[4], a1[4];
          low_codes(x, a0[0], a0[1]);
          low_codes(y, a0[2], a0[3]);
          high_codes(x, a1[0], a1[1]);
          high_codes(y, a1[2], a1[3]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float* q = s[sub][nb];
            const uint32_t b0 = transpose8x8(pack_pair<__half>(q[0] * st[0][j], q[1] * st[0][j]));
            const uint32_t b1 = transpose8x8(pack_pair<__half>(q[2] * st[1][j], q[3] * st[1][j]));
            mma16816<__half>(o[2 * j][nb], a0, b0, b1);
            mma16816<__half>(o[2 * j + 1][nb], a1, b0, b1);
            mma16816<__half>(o[2 * j][nb], eight, b0, b1);
            mma16816<__half>(o[2 * j + 1][nb], eight, b0, b1);
          }
        }
      }
    }
    __syncwarp();
    if (piece + C::kStages < n_pieces) load_piece(piece + C::kStages, slot);
    if (++slot == C::kStages) {
      slot = 0;
      phase ^= 1u;
    }
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 4; i < 32; i <<= 1) l[nb][c] += __shfl_xor_sync(0xffffffffu, l[nb][c], i);
  __syncthreads();                                           // every piece has been read: the rings become the join area
  const bool gave_up = ctl->abort_flag != 0;
  if (gave_up) {
    // a wait ran out: copies in flight land before the block ends; nothing is written (and nothing added to a cluster's rows)
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    if (!clustered) return;
  }
  rows_join<T, D, kC4Warps, kC4Threads, 8 * NB>(p, {qr, kvh, row0, n_rows, parts, clustered != 0}, (float*)smem, [&](float* part, float* stat) {
    // To the values' own scale.  Sums of numbers next to the type's largest would pass fp32 before they are divided: there the whole part is held times
    // 2^-20, its reference as much above.
    const int room = e_run > 96 ? 20 : 0;
    const float f = pow2i(e_run - kC4MidLog2 - room), f_l = pow2i(-kC4ProbLog2 - room);
    constexpr float kProb = 1.f / (1 << kC4ProbLog2);
    constexpr float kSteps = kProb * 0x1p24f * (1 << (kC4MidLog2 - kC4StepLog2));       // (codes are held times 2^-24)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = warp * 8 * NB + nb * 8 + 2 * tig + c;
        float* dst = part + r * D;
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const float low = __shfl_sync(0xffffffffu, om[nb][c], j * 4 + tig) * kProb * f;        // row j
#pragma unroll
          for (int i = 2 * j; i < 2 * j + 2; ++i) {
            dst[i * 16 + g] = fmaf(o[i][nb][c] * kSteps, f, low);
            dst[i * 16 + g + 8] = fmaf(o[i][nb][c + 2] * (kSteps * 0.0625f), f, low);
          }
        }
        if (g == 0) {
          float* st = stat + r * 4;
          st[0] = m[nb][c] + (float)room;
          st[1] = gave_up ? 0.f : l[nb][c] * f_l;
          st[2] = l[nb][c] * f_l;
        }
      }
  });
}

template <typename T, int D, int NB, bool kWindow>
int launch_cache4_kernel(const tra_packed_ctx& c, const tra_cache4_launch& a, int chunk, bool clustered) {
  constexpr auto kern = tra_cache4_rows_kernel<T, D, NB, kWindow>;
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
