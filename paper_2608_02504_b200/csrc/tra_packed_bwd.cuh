// Gradients of attention over packed sequences: two kernels that recompute the probabilities from lse and keep every sum
// inside one thread block (no atomics: the same bits every time).
//
// P = exp(S - lse), dP = dO V^T, dS = P (dP - delta), delta = rowsum(dO O) (a small kernel of its own).
//   tra_packed_dkv_kernel: one block per 128 keys of a (sequence, key/value head), walks the query tiles that see them:
//     S^T = K Q^T and dP^T = V dO^T (tcgen05, both operands in shared memory), the softmax threads (one key per
//     lane, 64 query rows per thread) write P^T and dS^T back to tensor memory in the 16-bit type, where they are the
//     A operands of dV += P^T dO and dK += dS^T Q.  A query tile holds all heads of the group, so the sum over the heads that
//     share a key/value head is the product's own.
//   tra_packed_dq_kernel: one block per 128-row query tile, walks its key blocks: S = Q K^T, dP = dO V^T, dQ += dS K.
// Seven products instead of the five that one pass over the pairs needs: the fifth sum, dQ, would have to leave the
// block through memory (fp32 atomics whose order changes the result, or 4 bytes per row, channel and key block).
//
// Order on the tensor pipe, so that it always has a product that waits for nobody:
//   dkv: dV(i), S(i+1), dK(i), dP(i+1): the threads turn dP(i) into dS(i) under the first two and S(i+1) into P(i+1)
//        under the last two;
//   dq : S(i+1) as soon as the threads hold S(i) in registers, dP(i+1) likewise, then dQ(i).
// Tensor memory: S [0, 128), dP [128, 256), two sums of D columns from 256 and 384 (dkv) or one and dS (dq).  P and dS of the
// warpgroup that owns columns 64 h .. 64 h + 63 overwrite the first 32 of those columns, which only its own threads
// read (dkv); dq keeps dS apart, because dP(i+1) is issued before dQ(i) has read it.
//
// Rows past a sequence's end (another sequence's, or anything) meet zero probabilities, but 0 * NaN is NaN where such a row is on the
// summed side of a product: an idle warp zeroes them in shared memory (dkv: rows of Q and dO; dq: rows of K and V).
#pragma once
#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kBwdThreads = 384;
constexpr int kBwdRegsSoftmax = 216;     // 2 * 216 + 72 = 3 * 168, the registers of the launch
constexpr int kBwdRegsControl = 72;
constexpr int kBwdStages = 2;

template <int D>
struct BwdCfg {
  static constexpr int kAtoms = D / 64;
  static constexpr int kAtomBytes = kTileM * 128;
  static constexpr int kTileBytes = kAtoms * kAtomBytes;
  static constexpr int kSmemData = (2 + 2 * kBwdStages) * kTileBytes;      // two resident tiles, stages of two tiles
  static constexpr int kSmemNeeded = kSmemData + 1024 + 512 + 2 * kBwdStages * kTileM * 4;
  // at least 120 KB so that one block owns an SM and its whole tensor memory
  static constexpr int kSmemBytes = kSmemNeeded > 120 * 1024 ? kSmemNeeded : 120 * 1024;
};

struct BwdCtl {
  uint64_t own_full;                     // the resident tiles
  uint64_t a_full[kBwdStages], b_full[kBwdStages];   // streamed tiles: Q / dO (dkv), K / V (dq)
  uint64_t stage_free[kBwdStages];
  uint64_t stat_full[kBwdStages], stat_free[kBwdStages];
  uint64_t s_full, dp_full;
  uint64_t s_read, dp_read;              // dq: the threads hold S / dP in registers
  uint64_t p_ready[2], ds_ready[2];      // per 64-column half
  uint64_t tail_full, tail_ready;
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
  tra_unit unit;
};
static_assert(sizeof(BwdCtl) <= 512, "control block");

// Set-up shared by the two kernels: barriers and the block's (sequence, unit).
__device__ __forceinline__ void bwd_init(BwdCtl* ctl) {
  mbar_init(smem_u32(&ctl->own_full), 1);
  for (int i = 0; i < kBwdStages; ++i) {
    mbar_init(smem_u32(&ctl->a_full[i]), 1);
    mbar_init(smem_u32(&ctl->b_full[i]), 1);
    mbar_init(smem_u32(&ctl->stage_free[i]), 1);
    mbar_init(smem_u32(&ctl->stat_full[i]), 1);
    mbar_init(smem_u32(&ctl->stat_free[i]), 8);
  }
  mbar_init(smem_u32(&ctl->s_full), 1);
  mbar_init(smem_u32(&ctl->dp_full), 1);
  mbar_init(smem_u32(&ctl->s_read), 8);
  mbar_init(smem_u32(&ctl->dp_read), 8);
  for (int h = 0; h < 2; ++h) {
    mbar_init(smem_u32(&ctl->p_ready[h]), 4);
    mbar_init(smem_u32(&ctl->ds_ready[h]), 4);
  }
  mbar_init(smem_u32(&ctl->tail_full), 1);
  mbar_init(smem_u32(&ctl->tail_ready), 1);
  mbar_init(smem_u32(&ctl->drain), 1);
  ctl->abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void bwd_teardown(BwdCtl* ctl, uint32_t tmem, int warp) {
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    if (ctl->abort_flag) {
      // let copies and MMAs that were in flight when the block gave up land before releasing
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_after();
    tmem_free_all(tmem);
  }
}

// 64 consecutive fp32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t* r) {
  tmem_ld32(taddr, r);
  tmem_ld32(taddr + 32, r + 32);
  tmem_wait_ld(r);
  reg_fence32(r + 32);
}

// Product of two K-major tiles in shared memory: D[tmem] = A B^T over the D channels.
template <int D>
__device__ __forceinline__ void mma_tiles(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  constexpr uint32_t kHi = desc_hi(1024);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    const uint32_t off = ((kk >> 2) * BwdCfg<D>::kAtomBytes + (kk & 3) * 32) >> 4;
    tc_mma_ss(d, a_lo + off, kHi, b_lo + off, kHi, idesc, kk > 0 ? 1u : 0u);
  }
}

// Stores 32 channels of one row, scaled and rounded.
template <typename T>
__device__ __forceinline__ void store32(T* dst, const uint32_t* bits, float mul) {
  uint4* out = reinterpret_cast<uint4*>(dst);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = pack_pair<T>(__uint_as_float(bits[q * 8 + 2 * j]) * mul, __uint_as_float(bits[q * 8 + 2 * j + 1]) * mul);
    out[q] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ------------------------------------------------------------------------------------ dK, dV
template <typename T, int D, bool kCausal>
__global__ void __launch_bounds__(kBwdThreads, 1) tra_packed_dkv_kernel(const __grid_constant__ tra_packed_launch p) {
  using C = BwdCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sK = smem;
  uint8_t* sV = smem + C::kTileBytes;
  uint8_t* sStage = smem + 2 * C::kTileBytes;               // [stage][Q, dO]
  BwdCtl* ctl = (BwdCtl*)(smem + C::kSmemData);
  float* s_lse2 = (float*)(smem + C::kSmemData + 512);       // [stage][128], then delta
  float* s_delta = s_lse2 + kBwdStages * kTileM;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kvh = blockIdx.y;

  const int tile_tokens = p.tile_tokens, box_rows = tile_tokens * p.group;

  // set-up in parallel, one barrier (see the forward kernel)
  if (warp == 0) {
    const tra_unit u = tra_find_unit(p, true, p.max_k <= kTileM, kTileM, (int)blockIdx.x);
    if (lane == 0) ctl->unit = u;
  } else if (warp == 9) {
    tmem_alloc_all(&ctl->tmem_base);
  } else if (tid == 32) {
    bwd_init(ctl);
  } else if (tid == 64) {
    prefetch_map(&p.map_q);
    prefetch_map(&p.map_do);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  if (box_rows < kTileM && warp >= 2 && warp < 8)        // rows that no box fills
    zero_tile_rows(sStage, box_rows, kTileM, 2 * kBwdStages * C::kAtoms, C::kAtomBytes, tid - 64, 192);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  const tra_seq_range qr = ctl->unit.q, kr = ctl->unit.k;
  const int key0 = ctl->unit.index * kTileM;
  if (ctl->unit.seq < 0 || key0 >= kr.len) {
    if (warp == 9) tmem_free_all(tmem);
    return;
  }
  const int ahead = kr.len - qr.len;
  const int n_tiles_all = (qr.len + tile_tokens - 1) / tile_tokens;
  // causal: key j is seen by the tokens from j - ahead on
  const int first_tile = kCausal ? max(key0 - ahead, 0) / tile_tokens : 0;
  const int n = max(n_tiles_all - first_tile, 0);
  const int tail_rows = (qr.len - (n_tiles_all - 1) * tile_tokens) * p.group;      // rows of the last tile
  const bool tail = n > 0 && tail_rows < box_rows;
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBwdRegsControl));
    if (warp == 8) {
      // ================================================================== TMA producer
      if (lane == 0) {
        const uint32_t own = smem_u32(&ctl->own_full);
        mbar_expect_tx(own, 2 * C::kTileBytes);
        for (int a = 0; a < C::kAtoms; ++a) {
          tma_load_3d(smem_u32(sK + a * C::kAtomBytes), &p.map_k, own, a * 64, kvh, kr.begin + key0);
          tma_load_3d(smem_u32(sV + a * C::kAtomBytes), &p.map_v, own, a * 64, kvh, kr.begin + key0);
        }
        for (int i = 0; i < n; ++i) {
          const int st = i % kBwdStages;
          if (i >= kBwdStages && !mbar_wait(smem_u32(&ctl->stage_free[st]), (uint32_t)(i / kBwdStages - 1) & 1u, abort_flag, p.status))
            break;
          const bool last_tail = tail && i == n - 1;
          const uint32_t qbar = smem_u32(last_tail ? &ctl->tail_full : &ctl->a_full[st]);
          const uint32_t obar = smem_u32(last_tail ? &ctl->tail_full : &ctl->b_full[st]);
          const uint32_t bytes = C::kAtoms * box_rows * 128;
          const int tok = qr.begin + (first_tile + i) * tile_tokens;
          uint8_t* dst = sStage + st * 2 * C::kTileBytes;
          if (last_tail) {
            mbar_expect_tx(qbar, 2 * bytes);
          } else {
            mbar_expect_tx(qbar, bytes);
            mbar_expect_tx(obar, bytes);
          }
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(dst + a * C::kAtomBytes), &p.map_q, qbar, a * 64, kvh * p.group, tok);
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(dst + C::kTileBytes + a * C::kAtomBytes), &p.map_do, obar, a * 64, kvh * p.group, tok);
        }
      }
    } else if (warp == 10) {
      // ================================================================== rows past the sequence's end
      if (tail && mbar_wait_warp(smem_u32(&ctl->tail_full), 0u, abort_flag, p.status)) {
        uint8_t* st = sStage + ((n - 1) % kBwdStages) * 2 * C::kTileBytes;
        zero_tile_rows(st, tail_rows, box_rows, 2 * C::kAtoms, C::kAtomBytes, lane, 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready));
      }
    } else if (warp == 11) {
      // ================================================================== lse and delta of the query rows
      for (int i = 0; i < n; ++i) {
        const int st = i % kBwdStages;
        if (i >= kBwdStages && !mbar_wait_warp(smem_u32(&ctl->stat_free[st]), (uint32_t)(i / kBwdStages - 1) & 1u, abort_flag, p.status))
          break;
        const int tok0 = (first_tile + i) * tile_tokens;
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int r = r4 * 32 + lane;
          const int tok = tok0 + r / p.group;
          float lse2 = INFINITY, delta = 0.f;           // a row that is not there, or sees no key: probability 0
          if (r < box_rows && tok < qr.len) {
            const long long row = (long long)(qr.begin + tok) * p.heads + kvh * p.group + r % p.group;
            const float v = p.lse[row] * kLog2e;
            lse2 = v == -INFINITY ? INFINITY : v;
            delta = p.delta[row];
          }
          s_lse2[st * kTileM + r] = lse2;
          s_delta[st * kTileM + r] = delta;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->stat_full[st]));
      }
    } else if (warp == 9) {
      // ================================================================== MMA issuer
      constexpr uint32_t kIdescS = make_idesc_t<T>(kTileM, false);
      constexpr uint32_t kIdescD = make_idesc_t<T>(D, true);
      constexpr uint32_t kHi = desc_hi(1024);
      const uint32_t k_lo = desc_lo(smem_u32(sK), 16), v_lo = desc_lo(smem_u32(sV), 16);
      const uint32_t stage_k = desc_lo(smem_u32(sStage), 16);                  // K-major views of Q; dO one tile behind
      const uint32_t stage_mn = desc_lo(smem_u32(sStage), C::kAtomBytes);      // MN-major views
      constexpr uint32_t kTile = C::kTileBytes >> 4;
      bool alive = mbar_wait(smem_u32(&ctl->own_full), 0u, abort_flag, p.status);
      auto wait_q = [&](int i) -> bool {
        if (tail && i == n - 1) return mbar_wait(smem_u32(&ctl->tail_ready), 0u, abort_flag, p.status);
        return mbar_wait(smem_u32(&ctl->a_full[i % kBwdStages]), (uint32_t)(i / kBwdStages) & 1u, abort_flag, p.status);
      };
      auto wait_do = [&](int i) -> bool {
        if (tail && i == n - 1) return true;                                   // came with Q
        return mbar_wait(smem_u32(&ctl->b_full[i % kBwdStages]), (uint32_t)(i / kBwdStages) & 1u, abort_flag, p.status);
      };
      auto issue_s = [&](int i) {
        tc_fence_after();
        mma_tiles<D>(tmem, k_lo, stage_k + (uint32_t)(i % kBwdStages) * 2 * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->s_full));
      };
      auto issue_dp = [&](int i) {
        tc_fence_after();
        mma_tiles<D>(tmem + 128, v_lo, stage_k + ((uint32_t)(i % kBwdStages) * 2 + 1) * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->dp_full));
      };
      // sum[tmem] += A[tmem, its 128 rows per half] * B[MN-major tile]
      auto issue_sum = [&](uint32_t d, uint32_t a, uint32_t b_lo, uint64_t* ready, int i) -> bool {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!mbar_wait(smem_u32(&ready[h]), (uint32_t)i & 1u, abort_flag, p.status)) return false;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma_ts(d, a + h * 64 + kk * 8, b_lo + (h * 4 + kk) * (2048 >> 4), kHi, kIdescD, h + kk > 0 ? 1u : (i > 0 ? 1u : 0u));
        }
        return true;
      };
      if (alive && n > 0) {
        alive = wait_q(0);
        if (alive) issue_s(0);
        if (alive) alive = wait_do(0);
        if (alive) issue_dp(0);
      }
      for (int i = 0; i < n && alive; ++i) {
        const uint32_t st = (uint32_t)(i % kBwdStages) * 2;
        if (!(alive = issue_sum(tmem + 256, tmem, stage_mn + (st + 1) * kTile, ctl->p_ready, i))) break;      // dV += P^T dO
        if (i + 1 < n) {
          if (!(alive = wait_q(i + 1))) break;
          issue_s(i + 1);
        }
        if (!(alive = issue_sum(tmem + 384, tmem + 128, stage_mn + st * kTile, ctl->ds_ready, i))) break;     // dK += dS^T Q
        tc_commit(smem_u32(&ctl->stage_free[i % kBwdStages]));
        if (i + 1 < n) {
          if (!(alive = wait_do(i + 1))) break;
          issue_dp(i + 1);
        }
      }
      tc_commit(smem_u32(&ctl->drain));
      mbar_wait(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kBwdRegsSoftmax));
    // ================================================================== probabilities and their gradients
    const int h = warp >> 2;                                 // columns 64 h .. 64 h + 63
    const int r = tid & (kTileM - 1);                        // key inside the tile
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lane_base + h * 64, t_dp = t_s + 128;
    const float scale_log2 = p.sm_scale * kLog2e;
    bool alive = true;
    for (int i = 0; i < n; ++i) {
      const int st = i % kBwdStages;
      const float4* lse4 = reinterpret_cast<const float4*>(s_lse2 + st * kTileM + h * 64);
      const float4* delta4 = reinterpret_cast<const float4*>(s_delta + st * kTileM + h * 64);
      if (!mbar_wait_warp(smem_u32(&ctl->stat_full[st]), (uint32_t)(i / kBwdStages) & 1u, abort_flag, p.status) ||
          !mbar_wait_warp(smem_u32(&ctl->s_full), (uint32_t)i & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      uint32_t s[64];
      float pr[64];
      tmem_ld64(t_s, s);
#pragma unroll
      for (int c4 = 0; c4 < 16; ++c4) {
        const float4 v = lse4[c4];
        pr[c4 * 4] = ex2(fmaf(__uint_as_float(s[c4 * 4]), scale_log2, -v.x));
        pr[c4 * 4 + 1] = ex2(fmaf(__uint_as_float(s[c4 * 4 + 1]), scale_log2, -v.y));
        pr[c4 * 4 + 2] = ex2(fmaf(__uint_as_float(s[c4 * 4 + 2]), scale_log2, -v.z));
        pr[c4 * 4 + 3] = ex2(fmaf(__uint_as_float(s[c4 * 4 + 3]), scale_log2, -v.w));
      }
      // causal: columns of tokens in front of key - ahead do not see this key
      const int blind = kCausal ? max(key0 + r - ahead - (first_tile + i) * tile_tokens, 0) * p.group - h * 64 : 0;
      if (kCausal && __any_sync(0xffffffffu, blind > 0)) {
#pragma unroll
        for (int c = 0; c < 64; ++c)
          if (c < blind) pr[c] = 0.f;
      }
      {
        uint32_t pk[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) pk[c] = pack_pair<T>(pr[2 * c], pr[2 * c + 1]);
        tmem_st32(t_s, pk);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->p_ready[h]));
      }
      if (!mbar_wait_warp(smem_u32(&ctl->dp_full), (uint32_t)i & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      tmem_ld64(t_dp, s);
      {
        uint32_t pk[32];
#pragma unroll
        for (int c4 = 0; c4 < 16; ++c4) {
          const float4 v = delta4[c4];
          pk[c4 * 2] = pack_pair<T>(pr[c4 * 4] * (__uint_as_float(s[c4 * 4]) - v.x), pr[c4 * 4 + 1] * (__uint_as_float(s[c4 * 4 + 1]) - v.y));
          pk[c4 * 2 + 1] = pack_pair<T>(pr[c4 * 4 + 2] * (__uint_as_float(s[c4 * 4 + 2]) - v.z), pr[c4 * 4 + 3] * (__uint_as_float(s[c4 * 4 + 3]) - v.w));
        }
        tmem_st32(t_dp, pk);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&ctl->ds_ready[h]));
          mbar_arrive(smem_u32(&ctl->stat_free[st]));
        }
      }
    }
    // ---- epilogue: warpgroup h stores channels h D / 2 .. of both gradients
    if (alive && n > 0) alive = mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    if (alive) {
      tc_fence_after();
      const bool row_valid = key0 + r < kr.len;
      const long long row = kr.begin + key0 + (row_valid ? r : 0);
      T* out[2] = {(T*)p.dv + row * p.dv_stride[0] + kvh * p.dv_stride[1], (T*)p.dk + row * p.dk_stride[0] + kvh * p.dk_stride[1]};
#pragma unroll
      for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const int col = h * (D / 2) + c * 32;
          uint32_t bits[32];
          if (n > 0) {
            tmem_ld32(tmem + lane_base + 256 + which * 128 + col, bits);
            tmem_wait_ld(bits);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) bits[j] = 0u;
          }
          if (row_valid) store32<T>(out[which] + col, bits, which ? p.sm_scale : 1.f);
        }
      }
    }
  }
  bwd_teardown(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------ dQ
template <typename T, int D, bool kCausal>
__global__ void __launch_bounds__(kBwdThreads, 1) tra_packed_dq_kernel(const __grid_constant__ tra_packed_launch p) {
  using C = BwdCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;
  uint8_t* sDO = smem + C::kTileBytes;
  uint8_t* sStage = smem + 2 * C::kTileBytes;               // [stage][K, V]
  BwdCtl* ctl = (BwdCtl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kvh = blockIdx.y;
  const int tile_tokens = p.tile_tokens, box_rows = tile_tokens * p.group;

  // set-up in parallel, one barrier (see the forward kernel)
  if (warp == 0) {
    // the last tiles of a causal sequence are the longest: launched first
    const tra_unit u = tra_find_unit(p, false, p.max_q <= tile_tokens, tile_tokens, (int)gridDim.x - 1 - (int)blockIdx.x);
    if (lane == 0) ctl->unit = u;
  } else if (warp == 9) {
    tmem_alloc_all(&ctl->tmem_base);
  } else if (tid == 32) {
    bwd_init(ctl);
  } else if (tid == 64) {
    prefetch_map(&p.map_q);
    prefetch_map(&p.map_do);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  if (box_rows < kTileM && warp >= 2 && warp < 8)        // rows that no box fills
    zero_tile_rows(sQ, box_rows, kTileM, 2 * C::kAtoms, C::kAtomBytes, tid - 64, 192);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  const tra_seq_range qr = ctl->unit.q, kr = ctl->unit.k;
  const int tok0 = ctl->unit.index * tile_tokens;
  if (ctl->unit.seq < 0 || tok0 >= qr.len) {
    if (warp == 9) tmem_free_all(tmem);
    return;
  }
  const int ahead = kr.len - qr.len;
  const int last_tok = min(tok0 + tile_tokens, qr.len) - 1;
  const int keys = kCausal ? min(max(last_tok + 1 + ahead, 0), kr.len) : kr.len;
  const int n = (keys + kTileM - 1) / kTileM;
  const bool tail = n > 0 && n * kTileM > kr.len;
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBwdRegsControl));
    if (warp == 8) {
      // ================================================================== TMA producer
      if (lane == 0) {
        const uint32_t own = smem_u32(&ctl->own_full);
        mbar_expect_tx(own, 2 * C::kAtoms * box_rows * 128);
        for (int a = 0; a < C::kAtoms; ++a) {
          tma_load_3d(smem_u32(sQ + a * C::kAtomBytes), &p.map_q, own, a * 64, kvh * p.group, qr.begin + tok0);
          tma_load_3d(smem_u32(sDO + a * C::kAtomBytes), &p.map_do, own, a * 64, kvh * p.group, qr.begin + tok0);
        }
        for (int i = 0; i < n; ++i) {
          const int st = i % kBwdStages;
          if (i >= kBwdStages && !mbar_wait(smem_u32(&ctl->stage_free[st]), (uint32_t)(i / kBwdStages - 1) & 1u, abort_flag, p.status))
            break;
          const bool last_tail = tail && i == n - 1;
          const uint32_t kbar = smem_u32(last_tail ? &ctl->tail_full : &ctl->a_full[st]);
          const uint32_t vbar = smem_u32(last_tail ? &ctl->tail_full : &ctl->b_full[st]);
          uint8_t* dst = sStage + st * 2 * C::kTileBytes;
          if (last_tail) {
            mbar_expect_tx(kbar, 2 * C::kTileBytes);
          } else {
            mbar_expect_tx(kbar, C::kTileBytes);
            mbar_expect_tx(vbar, C::kTileBytes);
          }
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(dst + a * C::kAtomBytes), &p.map_k, kbar, a * 64, kvh, kr.begin + i * kTileM);
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(dst + C::kTileBytes + a * C::kAtomBytes), &p.map_v, vbar, a * 64, kvh, kr.begin + i * kTileM);
        }
      }
    } else if (warp == 10) {
      // ================================================================== rows past the sequence's end
      if (tail && mbar_wait_warp(smem_u32(&ctl->tail_full), 0u, abort_flag, p.status)) {
        uint8_t* st = sStage + ((n - 1) % kBwdStages) * 2 * C::kTileBytes;
        zero_tile_rows(st, kr.len - (n - 1) * kTileM, kTileM, 2 * C::kAtoms, C::kAtomBytes, lane, 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready));
      }
    } else if (warp == 9) {
      // ================================================================== MMA issuer
      constexpr uint32_t kIdescS = make_idesc_t<T>(kTileM, false);
      constexpr uint32_t kIdescD = make_idesc_t<T>(D, true);
      constexpr uint32_t kHi = desc_hi(1024);
      const uint32_t q_lo = desc_lo(smem_u32(sQ), 16), do_lo = desc_lo(smem_u32(sDO), 16);
      const uint32_t stage_k = desc_lo(smem_u32(sStage), 16);
      const uint32_t stage_mn = desc_lo(smem_u32(sStage), C::kAtomBytes);
      constexpr uint32_t kTile = C::kTileBytes >> 4;
      bool alive = mbar_wait(smem_u32(&ctl->own_full), 0u, abort_flag, p.status);
      auto wait_k = [&](int i) -> bool {
        if (tail && i == n - 1) return mbar_wait(smem_u32(&ctl->tail_ready), 0u, abort_flag, p.status);
        return mbar_wait(smem_u32(&ctl->a_full[i % kBwdStages]), (uint32_t)(i / kBwdStages) & 1u, abort_flag, p.status);
      };
      auto wait_v = [&](int i) -> bool {
        if (tail && i == n - 1) return true;                                   // came with K
        return mbar_wait(smem_u32(&ctl->b_full[i % kBwdStages]), (uint32_t)(i / kBwdStages) & 1u, abort_flag, p.status);
      };
      auto issue_s = [&](int i) {
        tc_fence_after();
        mma_tiles<D>(tmem, q_lo, stage_k + (uint32_t)(i % kBwdStages) * 2 * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->s_full));
      };
      auto issue_dp = [&](int i) {
        tc_fence_after();
        mma_tiles<D>(tmem + 128, do_lo, stage_k + ((uint32_t)(i % kBwdStages) * 2 + 1) * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->dp_full));
      };
      if (alive && n > 0) {
        alive = wait_k(0);
        if (alive) issue_s(0);
        if (alive) alive = wait_v(0);
        if (alive) issue_dp(0);
      }
      for (int i = 0; i < n && alive; ++i) {
        if (i + 1 < n) {
          if (!(alive = mbar_wait(smem_u32(&ctl->s_read), (uint32_t)i & 1u, abort_flag, p.status) && wait_k(i + 1))) break;
          issue_s(i + 1);
          if (!(alive = mbar_wait(smem_u32(&ctl->dp_read), (uint32_t)i & 1u, abort_flag, p.status) && wait_v(i + 1))) break;
          issue_dp(i + 1);
        }
        const uint32_t b_lo = stage_mn + (uint32_t)(i % kBwdStages) * 2 * kTile;        // dQ += dS K
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!(alive = mbar_wait(smem_u32(&ctl->ds_ready[h]), (uint32_t)i & 1u, abort_flag, p.status))) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma_ts(tmem + 256, tmem + 384 + (h * 4 + kk) * 8, b_lo + (h * 4 + kk) * (2048 >> 4), kHi, kIdescD,
                      h + kk > 0 ? 1u : (i > 0 ? 1u : 0u));
        }
        if (!alive) break;
        tc_commit(smem_u32(&ctl->stage_free[i % kBwdStages]));
      }
      tc_commit(smem_u32(&ctl->drain));
      mbar_wait(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kBwdRegsSoftmax));
    const int h = warp >> 2;                                 // key columns 64 h .. 64 h + 63 of a block
    const int r = tid & (kTileM - 1);                        // query row
    const int r_tok = r / p.group, r_head = r - r_tok * p.group;
    const int tok = tok0 + r_tok;
    const bool row_valid = r < box_rows && tok < qr.len;
    const long long tok_g = qr.begin + (row_valid ? tok : 0);
    const int head = kvh * p.group + (row_valid ? r_head : 0);
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const float scale_log2 = p.sm_scale * kLog2e;
    float lse2 = INFINITY, delta = 0.f;                      // a row that is not there, or sees no key: probability 0
    if (row_valid) {
      const float v = p.lse[tok_g * p.heads + head] * kLog2e;
      lse2 = v == -INFINITY ? INFINITY : v;
      delta = p.delta[tok_g * p.heads + head];
    }
    const int seen = kCausal ? min(max(min(tok, last_tok) + 1 + ahead, 0), kr.len) : kr.len;
    bool alive = true;
    for (int i = 0; i < n; ++i) {
      if (!mbar_wait_warp(smem_u32(&ctl->s_full), (uint32_t)i & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      uint32_t s[64];
      float pr[64];
      tmem_ld64(tmem + lane_base + h * 64, s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->s_read));
#pragma unroll
      for (int c = 0; c < 64; ++c) pr[c] = ex2(fmaf(__uint_as_float(s[c]), scale_log2, -lse2));
      const int limit = seen - i * kTileM - h * 64;          // columns at and past it are not seen
      if (__any_sync(0xffffffffu, limit < 64)) {
#pragma unroll
        for (int c = 0; c < 64; ++c)
          if (c >= limit) pr[c] = 0.f;
      }
      if (!mbar_wait_warp(smem_u32(&ctl->dp_full), (uint32_t)i & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      tmem_ld64(tmem + lane_base + 128 + h * 64, s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->dp_read));
      uint32_t pk[32];
#pragma unroll
      for (int c = 0; c < 32; ++c)
        pk[c] = pack_pair<T>(pr[2 * c] * (__uint_as_float(s[2 * c]) - delta), pr[2 * c + 1] * (__uint_as_float(s[2 * c + 1]) - delta));
      // the product that read the last dS has retired (it also freed that stage)
      if (i > 0 && !mbar_wait_warp(smem_u32(&ctl->stage_free[(i - 1) % kBwdStages]), (uint32_t)((i - 1) / kBwdStages) & 1u,
                                   abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      tmem_st32(tmem + lane_base + 384 + h * 32, pk);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->ds_ready[h]));
    }
    if (alive && n > 0) alive = mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    if (alive) {
      tc_fence_after();
      T* out = (T*)p.dq + tok_g * p.dq_stride[0] + head * p.dq_stride[1];
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const int col = h * (D / 2) + c * 32;
        uint32_t bits[32];
        if (n > 0) {
          tmem_ld32(tmem + lane_base + 256 + col, bits);
          tmem_wait_ld(bits);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) bits[j] = 0u;
        }
        if (row_valid) store32<T>(out + col, bits, p.sm_scale);
      }
    }
  }
  bwd_teardown(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------ delta
// delta = sum over the channels of dO O, d / 8 threads per (token, head), 16 bytes each.
template <typename T, int D>
__global__ void __launch_bounds__(256) tra_packed_delta_kernel(const __grid_constant__ tra_packed_launch p) {
  constexpr int kLanes = D / 8;
  const long long row = (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const int lane = threadIdx.x % kLanes;
  const long long rows = (long long)p.total_q * p.heads;
  float s = 0.f;
  if (row < rows) {
    const long long tok = row / p.heads;
    const int head = (int)(row - tok * p.heads);
    const uint4 a = *reinterpret_cast<const uint4*>((const T*)p.o_in + tok * p.o_stride[0] + head * p.o_stride[1] + lane * 8);
    const uint4 b = *reinterpret_cast<const uint4*>((const T*)p.d_o + tok * p.do_stride[0] + head * p.do_stride[1] + lane * 8);
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x0, x1, y0, y1;
      unpack_pair<T>(x[i], x0, x1);
      unpack_pair<T>(y[i], y0, y1);
      s = fmaf(x0, y0, s);
      s = fmaf(x1, y1, s);
    }
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (row < rows && lane == 0) p.delta[row] = s;
}

template <typename T, int D, bool kCausal>
int launch_bwd(const tra_packed_ctx& c, const tra_packed_launch& a) {
  const long long rows = (long long)a.total_q * a.heads;
  if (rows > 0) {
    constexpr int kRows = 256 / (D / 8);
    tra_packed_delta_kernel<T, D><<<(unsigned)((rows + kRows - 1) / kRows), 256, 0, c.stream>>>(a);
    TRA_CUDA_CHECK(cudaGetLastError());
  }
  if (a.max_k > 0) {
    auto dkv = tra_packed_dkv_kernel<T, D, kCausal>;
    TRA_CUDA_CHECK(cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, BwdCfg<D>::kSmemBytes));
    const unsigned units = (unsigned)((a.max_k <= kTileM ? 0 : a.total_k / kTileM) + a.n_seq);
    dkv<<<dim3(units, (unsigned)a.kv_heads), kBwdThreads, BwdCfg<D>::kSmemBytes, c.stream>>>(a);
    TRA_CUDA_CHECK(cudaGetLastError());
  }
  if (a.max_q > 0) {
    auto dq = tra_packed_dq_kernel<T, D, kCausal>;
    TRA_CUDA_CHECK(cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, BwdCfg<D>::kSmemBytes));
    const unsigned units = (unsigned)((a.max_q <= a.tile_tokens ? 0 : a.total_q / a.tile_tokens) + a.n_seq);
    dq<<<dim3(units, (unsigned)a.kv_heads), kBwdThreads, BwdCfg<D>::kSmemBytes, c.stream>>>(a);
    TRA_CUDA_CHECK(cudaGetLastError());
  }
  return TRA_OK;
}

template <int D>
int launch_bwd_shape(const tra_packed_ctx& c, const tra_packed_launch& a) {
  if (c.h->cfg.dtype == TRA_BF16)
    return a.causal ? launch_bwd<__nv_bfloat16, D, true>(c, a) : launch_bwd<__nv_bfloat16, D, false>(c, a);
  return a.causal ? launch_bwd<__half, D, true>(c, a) : launch_bwd<__half, D, false>(c, a);
}

}  // namespace
