// Gradients of attention over packed sequences: one launch of two kinds of blocks that recompute the probabilities from lse
// and keep every sum inside one thread block (no atomic sums: the same bits every time).
//
// P = exp(S - lse), dP = dO V^T, dS = P (dP - delta), delta = rowsum(dO O) (a small kernel in front).
//   dkv_block: one block per 128 keys of a (sequence, key/value head), walks the query tiles that see them:
//     S^T = K Q^T and dP^T = V dO^T (tcgen05, both operands in shared memory), the softmax threads (one key per
//     lane, 64 query rows per thread) write P^T and dS^T back to tensor memory in the 16-bit type, where they are the
//     A operands of dV += P^T dO and dK += dS^T Q.  A query tile holds all heads of the group, so the sum over the heads that
//     share a key/value head is the product's own.
//   dq_block: one block per 128-row query tile, walks its key blocks: S = Q K^T, dP = dO V^T, dQ += dS K.
// Seven products instead of the five that one pass over the pairs needs: the fifth sum, dQ, would have to leave the
// block through memory (fp32 atomics whose order changes the result, or 4 bytes per row, channel and key block).
//
// 4,096 tokens, 16 heads, d 128: 0.36 ms (957 TFLOP/s of the five products that the gradients need, 1,340 of the seven); four causal
// sequences of them, 40 / 8 heads: 2.13 ms (807); four, 16 heads, d 64: 1.09 ms (630); nine of 1,560, 12 heads, d 64: 0.40 ms.
//
// Order on the tensor pipe, so that it always has a product that waits for nobody:
//   dkv: S(i+1) as soon as the threads hold dP(i) in registers, dV(i), then dK(i), dP(i+1): the threads turn dP(i) into dS(i)
//        under the first two and S(i+1) into P(i+1) under the last two;
//   dq : S(i+1) as soon as the threads hold S(i) in registers, dP(i+1) likewise, then dQ(i).
// Tensor memory: two places of a step's columns, then the sums.  dkv: S(i) in one place, dP(i) in the other; P and dS of the
// warpgroup that owns columns 64 h .. 64 h + 63 overwrite its scores (the first and the last 32 of those columns), which only its
// own threads read; so dP's place is free for S(i+1) before the products have read P(i) and dS(i), and theirs takes dP(i+1).
// dq: S, dP, dQ, and dS apart, because dP(i+1) is issued before dQ(i) has read it.
//
// Rows past a sequence's end (another sequence's, or anything) meet zero probabilities, but 0 * NaN is NaN where such a row is on the
// summed side of a product: an idle warp zeroes them in shared memory (dkv: rows of Q and dO; dq: rows of K and V).
#pragma once
#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kStatStages = 2;           // of the query rows' lse and delta (dkv)

// fp16 holds P and dS = P (dP - delta) for their products only where they are not small: below 2^-14 its steps stop shrinking, and
// a long row's P, or any row's dS under a small dO, lies there (4,096 keys seen about evenly, d 128: dq 4 % off at
// |dO| = 1e-4, 34 % at 1e-5).  So both are rounded in
// fp16 as multiples, by powers of two that the epilogue's fp32 factor takes out again (0.03 and 0.16 % then, the latter the steps
// of dO and dq themselves):
//   P 2^12: P <= 1 up to the error of its exponent, so 2^12 leaves four binades for that; full precision down to P = 2^-26;
//   dP - delta times tau, the power of two that brings its bound 2 max|dO row| max|V row| into [1, 2) (|delta| is a mean of the dP):
//   dS 2^12 tau < 2^13, full precision 27 binades down.  The maxima, over the rows of a key/value head's sequences, are formed beside
// delta (atomic maxima: the same bits in any order), which costs a clearing, a read of V and 8 us more beside delta (nine sequences
// of 1,560 tokens, 12 heads, d 64: training step 478 -> 490 us).  bf16 has the range of fp32 and needs none of it.
template <typename T>
constexpr bool kScaled = std::is_same<T, __half>::value;
constexpr float kProbLog2 = 12.f, kProbMul = 4096.f;

__device__ __forceinline__ float grad_tau(const tra_packed_launch& p, int kvh) {
  const float x = __uint_as_float(p.norms[kvh]) * __uint_as_float(p.norms[p.kv_heads + kvh]);      // 2^-96 .. 2^78, or 0
  if (!(x > 0.f)) return 1.f;
  const int e = (int)(__float_as_uint(x) >> 23) - 127;               // 2 sqrt(x) < 2^(1 + (e + 1) / 2)
  return __uint_as_float((uint32_t)(127 - ((e + 2) >> 1)) << 23);
}

// kHalves: groups of 64 columns that a step walks, with one warpgroup of softmax threads each.
//   2: streamed tiles of 128 rows, one block per SM.
//   1: streamed tiles of 64 rows, half of the tensor memory, two blocks per SM: where the products are short (D = 64) one block's
//      start and end are hidden by the other (nine sequences of 1,560 tokens, 12 heads: 0.46 -> 0.40 ms; of 4,096: level).
template <int D, int kHalves>
struct BwdCfg {
  static constexpr int kAtoms = D / 64;
  static constexpr int kAtomBytes = kTileM * 128;                          // resident tiles
  static constexpr int kTileBytes = kAtoms * kAtomBytes;
  static constexpr int kStream = 64 * kHalves;                             // rows of a streamed tile
  static constexpr int kStreamAtom = kStream * 128;
  static constexpr int kStreamBytes = kAtoms * kStreamAtom;
  // Rings of streamed tiles.  A = Q (dkv) or K (dq), which two products use, the second one a step later; B = dO or V, done
  // with earlier.  A ring of two A tiles left the tensor pipe waiting for its loads (440 cycles of 3,750 per step, dkv).
  static constexpr int kA = D == 128 ? 3 : 4;
  static constexpr int kB = D == 128 ? 2 : 4;
  static constexpr int kSmemData = 2 * kTileBytes + (kA + kB) * kStreamBytes;
  static constexpr int kSmemNeeded = kSmemData + 512 + 2 * kStatStages * kStream * 4;
  // At least 120 KB so that one block owns an SM and its whole tensor memory; with halves 113 KB, so that two fit and neither shares
  // the SM with a block that wants all of it.
  static constexpr int kSmemLeast = kHalves == 2 ? 120 * 1024 : 113 * 1024;
  static constexpr int kSmemBytes = kSmemNeeded > kSmemLeast ? kSmemNeeded : kSmemLeast;
  static_assert(kSmemBytes <= (kHalves == 2 ? 232448 : kSmemLeast), "shared memory of a block");
  static constexpr int kSoftWarps = 4 * kHalves;
  static constexpr int kThreads = 32 * kSoftWarps + 128;
  static constexpr int kBlocks = kHalves == 2 ? 1 : 2;                     // per SM
  static constexpr int kRegsSoftmax = kHalves == 2 ? 216 : 200;            // 2 * 216 + 72 = 3 * 168, the registers of the launch;
  static constexpr int kRegsControl = kHalves == 2 ? 72 : 56;              // 200 + 56 = 2 * 128
  // Tensor memory: two places of a step's width, for the scores and dP, and the sums; P and dS over the scores (dkv), dS apart (dq).
  static constexpr int kColumns = 256 * kHalves;
  static constexpr int kDp = kStream;
  static constexpr int kSum0 = 2 * kStream, kSum1 = 3 * kStream;           // dV and dK; dQ and dS
  static_assert(D <= kStream, "the sums' columns");
};

struct BwdCtl {
  uint64_t own_full;                     // the resident tiles
  uint64_t a_full[4], b_full[4], a_free[4], b_free[4];       // streamed tiles
  uint64_t stat_full[kStatStages], stat_free[kStatStages];
  uint64_t s_full, dp_full;
  uint64_t s_read, dp_read;              // the threads hold S / dP in registers (dkv: and have stored P, before dp_read)
  uint64_t ds_ready;
  uint64_t tail_full, tail_ready;
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
  float tau;                             // fp16: see kScaled (dkv)
  tra_unit unit;
};
static_assert(sizeof(BwdCtl) <= 512, "control block");

// Set-up shared by the two kernels: barriers and the block's (sequence, unit).
template <int kHalves>
__device__ __forceinline__ void bwd_init(BwdCtl* ctl) {
  mbar_init(smem_u32(&ctl->own_full), 1);
  for (int i = 0; i < 4; ++i) {
    mbar_init(smem_u32(&ctl->a_full[i]), 1);
    mbar_init(smem_u32(&ctl->b_full[i]), 1);
    mbar_init(smem_u32(&ctl->a_free[i]), 1);
    mbar_init(smem_u32(&ctl->b_free[i]), 1);
  }
  for (int i = 0; i < kStatStages; ++i) {
    mbar_init(smem_u32(&ctl->stat_full[i]), 1);
    mbar_init(smem_u32(&ctl->stat_free[i]), 4 * kHalves);
  }
  mbar_init(smem_u32(&ctl->s_full), 1);
  mbar_init(smem_u32(&ctl->dp_full), 1);
  mbar_init(smem_u32(&ctl->s_read), 4 * kHalves);
  mbar_init(smem_u32(&ctl->dp_read), 4 * kHalves);
  mbar_init(smem_u32(&ctl->ds_ready), 4 * kHalves);
  mbar_init(smem_u32(&ctl->tail_full), 1);
  mbar_init(smem_u32(&ctl->tail_ready), 1);
  mbar_init(smem_u32(&ctl->drain), 1);
  ctl->abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

template <class C>
__device__ __forceinline__ void bwd_teardown(BwdCtl* ctl, uint32_t tmem, int warp) {
  tc_fence_before();
  __syncthreads();
  if (warp == C::kSoftWarps + 1) {
    if (ctl->abort_flag) {
      // let copies and MMAs that were in flight when the block gave up land before releasing
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_after();
    tmem_free<C::kColumns>(tmem);
  }
}

// Position in a ring: tile i lies in slot i % N and is the (i / N)-th of its slot.
template <int N>
struct RingPos {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++slot == N) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// The producer's loop of either kernel: tile i of each ring as soon as its slot is free.  The
// last pair goes to tail_full when rows past the sequence's end have to be zeroed in it.
template <class C, typename LoadA, typename LoadB>
__device__ __forceinline__ void bwd_produce(BwdCtl* ctl, int n, bool tail, uint32_t bytes, volatile int* abort_flag, int* status,
                                            LoadA load_a, LoadB load_b) {
  RingPos<C::kA> a;
  RingPos<C::kB> b;
  for (int i = 0; i < n; ++i) {
    const bool last = tail && i == n - 1;
    const uint32_t abar = smem_u32(last ? &ctl->tail_full : &ctl->a_full[a.slot]);
    const uint32_t bbar = smem_u32(last ? &ctl->tail_full : &ctl->b_full[b.slot]);
    if (last) mbar_expect_tx(abar, 2 * bytes);
    auto do_a = [&]() -> bool {
      if (i >= C::kA && !mbar_wait(smem_u32(&ctl->a_free[a.slot]), a.phase ^ 1u, abort_flag, status)) return false;
      if (!last) mbar_expect_tx(abar, bytes);
      load_a(i, a.slot, abar);
      return true;
    };
    auto do_b = [&]() -> bool {
      if (i >= C::kB && !mbar_wait(smem_u32(&ctl->b_free[b.slot]), b.phase ^ 1u, abort_flag, status)) return false;
      if (!last) mbar_expect_tx(bbar, bytes);
      load_b(i, b.slot, bbar);
      return true;
    };
    if (!(do_a() && do_b())) break;
    a.next();
    b.next();
  }
}

// 64 consecutive fp32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t* r) {
  tmem_ld32(taddr, r);
  tmem_ld32(taddr + 32, r + 32);
  tmem_wait_ld(r);
  reg_fence32(r + 32);
}

// Product of two K-major tiles in shared memory: D[tmem] = A B^T over the D channels (atoms of 128 rows where there are two).
template <int D>
__device__ __forceinline__ void mma_tiles(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  constexpr uint32_t kHi = desc_hi(1024);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    const uint32_t off = ((kk >> 2) * kTileM * 128 + (kk & 3) * 32) >> 4;
    tc_mma_ss(d, a_lo + off, kHi, b_lo + off, kHi, idesc, kk > 0 ? 1u : 0u);
  }
}

// The warpgroup's share (kChannels from h kChannels on) of a sum in tensor memory, scaled and rounded, to the rows' memory.
template <typename T, int kChannels>
__device__ __forceinline__ void store_share(const RowAddresses& rows, uint32_t taddr, int h, bool any, float mul) {
#pragma unroll 1
  for (int c = 0; c < kChannels / 32; ++c) {
    uint32_t v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = 0u;
    if (any) {
      tmem_ld32(taddr + h * kChannels + c * 32, v);
      tmem_wait_ld(v);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = pack_pair<T>(__uint_as_float(v[2 * j]) * mul, __uint_as_float(v[2 * j + 1]) * mul);
    rows.store64(v, h * kChannels * 2 + c * 64);
  }
}

// ------------------------------------------------------------------------------------ dK, dV
template <typename T, int D, int kHalves, bool kCausal>
__device__ __forceinline__ void dkv_block(const tra_packed_launch& p, uint8_t* smem, const int unit, const int kvh) {
  using C = BwdCfg<D, kHalves>;
  uint8_t* sK = smem;
  uint8_t* sV = smem + C::kTileBytes;
  uint8_t* sA = smem + 2 * C::kTileBytes;                   // Q tiles
  uint8_t* sB = sA + C::kA * C::kStreamBytes;                 // dO tiles
  BwdCtl* ctl = (BwdCtl*)(smem + C::kSmemData);
  float* s_lse2 = (float*)(smem + C::kSmemData + 512);       // [stage][streamed row], then delta
  float* s_delta = s_lse2 + kStatStages * C::kStream;
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;

  const int tile_tokens = p.stream_tokens, box_rows = tile_tokens * p.group;

  // set-up in parallel, one barrier (see the forward kernel)
  if (warp == 0) {
    const tra_unit u = tra_find_unit(p, true, p.max_k <= kTileM, kTileM, unit);
    if (lane == 0) ctl->unit = u;
  } else if (warp == C::kSoftWarps + 1) {
    tmem_alloc<C::kColumns>(&ctl->tmem_base);
  } else if (tid == 32) {
    bwd_init<kHalves>(ctl);
  } else if (tid == 64) {
    prefetch_map(&p.map_q_stream);
    prefetch_map(&p.map_do_stream);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  if (box_rows < C::kStream && warp >= 2 && warp < C::kSoftWarps)        // rows that no box fills
    zero_tile_rows(sA, box_rows, C::kStream, (C::kA + C::kB) * C::kAtoms, C::kStreamAtom, tid - 64, 32 * (C::kSoftWarps - 2));
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  const tra_seq_range qr = ctl->unit.q, kr = ctl->unit.k;
  const int key0 = ctl->unit.index * kTileM;
  if (ctl->unit.seq < 0) {
    if (warp == C::kSoftWarps + 1) tmem_free<C::kColumns>(tmem);
    wait_last_launch();          // no block ends before the launch in front of it
    return;
  }
  const int ahead = kr.len - qr.len;
  const int n_tiles_all = (qr.len + tile_tokens - 1) / tile_tokens;
  // causal: key j is seen by the tokens from j - ahead on
  const int first_tile = kCausal ? max(key0 - ahead, 0) / tile_tokens : 0;
  const int n_all = max(n_tiles_all - first_tile, 0), n = n_all;
  const int tail_rows = (qr.len - (n_tiles_all - 1) * tile_tokens) * p.group;      // rows of the last tile
  const bool tail_all = n > 0 && tail_rows < box_rows, tail = tail_all;
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp >= C::kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsControl));
    if (warp == C::kSoftWarps) {
      // ================================================================== TMA producer
      if (lane == 0) {
        const uint32_t own = smem_u32(&ctl->own_full);
        mbar_expect_tx(own, 2 * C::kTileBytes);
        for (int a = 0; a < C::kAtoms; ++a)
          for (int b = 0; b < kTileM; b += C::kStream) {
            tma_load_3d(smem_u32(sK + a * C::kAtomBytes + b * 128), &p.map_k, own, a * 64, kvh, kr.begin + key0 + b);
            tma_load_3d(smem_u32(sV + a * C::kAtomBytes + b * 128), &p.map_v, own, a * 64, kvh, kr.begin + key0 + b);
          }
        const int tok0 = qr.begin + first_tile * tile_tokens;
        bwd_produce<C>(
            ctl, n, tail, C::kAtoms * box_rows * 128, abort_flag, p.status,
            [&](int i, int slot, uint32_t bar) {
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sA + slot * C::kStreamBytes + a * C::kStreamAtom), &p.map_q_stream, bar, a * 64, kvh * p.group, tok0 + i * tile_tokens);
            },
            [&](int i, int slot, uint32_t bar) {
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sB + slot * C::kStreamBytes + a * C::kStreamAtom), &p.map_do_stream, bar, a * 64, kvh * p.group, tok0 + i * tile_tokens);
            });
      }
    } else if (warp == C::kSoftWarps + 2) {
      // ================================================================== rows past the sequence's end
      if (tail && mbar_wait_warp(smem_u32(&ctl->tail_full), 0u, abort_flag, p.status)) {
        zero_tile_rows(sA + ((n - 1) % C::kA) * C::kStreamBytes, tail_rows, box_rows, C::kAtoms, C::kStreamAtom, lane, 32);
        zero_tile_rows(sB + ((n - 1) % C::kB) * C::kStreamBytes, tail_rows, box_rows, C::kAtoms, C::kStreamAtom, lane, 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready));
      }
    } else if (warp == C::kSoftWarps + 3) {
      // ================================================================== lse and delta of the query rows
      wait_last_launch();                                 // delta
      float tau = 1.f;
      if (kScaled<T> && n > 0) {
        tau = grad_tau(p, kvh);
        if (lane == 0) ctl->tau = tau;                    // read behind the first stat_full
      }
      // read before the wait for the slot, so that the loads' latency is not added to it
      constexpr int kPer = C::kStream / 32;
      int r_tok[kPer], r_row[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int r = k * 32 + lane;
        r_tok[k] = r < box_rows ? r / p.group : 1 << 30;             // past every sequence: a row no box fills
        r_row[k] = r % p.group;
      }
      for (int i = 0; i < n; ++i) {
        const int st = i % kStatStages;
        const int tok0 = (first_tile + i) * tile_tokens;
        float lse2[kPer], delta[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          lse2[k] = INFINITY;                             // a row that is not there, or sees no key: probability 0
          delta[k] = 0.f;
          if (r_tok[k] < qr.len - tok0) {
            const long long row = (long long)(qr.begin + tok0 + r_tok[k]) * p.heads + kvh * p.group + r_row[k];
            lse2[k] = p.lse[row];
            delta[k] = p.delta[row];
          }
        }
        if (i >= kStatStages && !mbar_wait_warp(smem_u32(&ctl->stat_free[st]), (uint32_t)(i / kStatStages - 1) & 1u, abort_flag, p.status))
          break;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {                     // negated for the packed multiply-add
          s_lse2[st * C::kStream + k * 32 + lane] =
              lse2[k] == -INFINITY ? -INFINITY : kScaled<T> ? fmaf(-lse2[k], kLog2e, kProbLog2) : -lse2[k] * kLog2e;
          s_delta[st * C::kStream + k * 32 + lane] = -delta[k] * tau;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->stat_full[st]));
      }
    } else if (warp == C::kSoftWarps + 1) {
      // ================================================================== MMA issuer
      constexpr uint32_t kIdescS = make_idesc_t<T>(C::kStream, false);
      constexpr uint32_t kIdescD = make_idesc_t<T>(D, true);
      constexpr uint32_t kHi = desc_hi(1024);
      const uint32_t k_lo = desc_lo(smem_u32(sK), 16), v_lo = desc_lo(smem_u32(sV), 16);
      const uint32_t a_k = desc_lo(smem_u32(sA), 16), a_mn = desc_lo(smem_u32(sA), C::kStreamAtom);     // K-major and MN-major views
      const uint32_t b_k = desc_lo(smem_u32(sB), 16), b_mn = desc_lo(smem_u32(sB), C::kStreamAtom);
      constexpr uint32_t kTile = C::kStreamBytes >> 4;
      RingPos<C::kA> qs, qd;                 // Q of the next S, of the next dK
      RingPos<C::kB> os, od;                 // dO of the next dP, of the next dV
      const uint32_t tmem = uniform(ctl->tmem_base);
      const int n = uniform(n_all);
      const bool tail = uniform(tail_all);
      bool alive = mbar_wait_warp(smem_u32(&ctl->own_full), 0u, abort_flag, p.status);
      // Q and dO of the next scores and dP are in shared memory
      auto tiles_here = [&](int i) -> bool {
        if (tail && i == n - 1) return mbar_wait_warp(smem_u32(&ctl->tail_ready), 0u, abort_flag, p.status);
        return mbar_wait_warp(smem_u32(&ctl->a_full[qs.slot]), qs.phase, abort_flag, p.status) &&
               mbar_wait_warp(smem_u32(&ctl->b_full[os.slot]), os.phase, abort_flag, p.status);
      };
      auto issue_s = [&](int i) {
        mma_tiles<D>(tmem + (i & 1 ? C::kDp : 0), k_lo, a_k + (uint32_t)qs.slot * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->s_full));
        qs.next();
      };
      auto issue_dp = [&](int i) {
        mma_tiles<D>(tmem + (i & 1 ? 0 : C::kDp), v_lo, b_k + (uint32_t)os.slot * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->dp_full));
        os.next();
      };
      // sum[tmem] += A[tmem] * B[MN-major tile]
      auto issue_sum = [&](uint32_t d, uint32_t a, uint32_t b_lo, int i) {
#pragma unroll
        for (int kk = 0; kk < 4 * kHalves; ++kk)
          tc_mma_ts(d, a + (kk >> 2) * 64 + (kk & 3) * 8, b_lo + kk * (2048 >> 4), kHi, kIdescD, kk > 0 ? 1u : (i > 0 ? 1u : 0u));
      };
      alive = alive && n > 0 && tiles_here(0);
      if (alive) {
        tc_fence_after();
        issue_s(0);
        issue_dp(0);
      }
      // Every wait costs this warp about 120 cycles, met or not, and the threads wait for the scores: so the tiles are waited for
      // while the threads compute P, P needs no barrier of its own (dp_read comes behind its stores), and the scores go first.
      // Waits end in a vote and values from shared memory in a reduction, so that descriptors stay in uniform registers (2.24 ->
      // 2.15 ms, four causal sequences of 4,096 tokens, 40 / 8 heads, d 128; 1.15 -> 1.09 ms, 16 heads, d 64, not causal).
      for (int i = 0; i < n && alive; ++i) {
        const bool next = i + 1 < n;
        const uint32_t t_p = tmem + (i & 1 ? C::kDp : 0);
        if (next && !(alive = tiles_here(i + 1))) break;
        if (!(alive = mbar_wait_warp(smem_u32(&ctl->dp_read), (uint32_t)i & 1u, abort_flag, p.status))) break;
        tc_fence_after();
        if (next) issue_s(i + 1);                                                   // in dP's place
        issue_sum(tmem + C::kSum0, t_p, b_mn + (uint32_t)od.slot * kTile, i);       // dV += P^T dO
        tc_commit(smem_u32(&ctl->b_free[od.slot]));
        od.next();
        if (!(alive = mbar_wait_warp(smem_u32(&ctl->ds_ready), (uint32_t)i & 1u, abort_flag, p.status))) break;
        tc_fence_after();
        issue_sum(tmem + C::kSum1, t_p + 32, a_mn + (uint32_t)qd.slot * kTile, i);  // dK += dS^T Q
        tc_commit(smem_u32(&ctl->a_free[qd.slot]));
        qd.next();
        if (next) issue_dp(i + 1);                                                  // in the place of P and dS
      }
      tc_commit(smem_u32(&ctl->drain));
      mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
    // ================================================================== probabilities and their gradients
    const int h = warp >> 2;                                 // columns 64 h .. 64 h + 63
    int r = tid & (kTileM - 1);                              // key inside the tile
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const float scale_log2 = p.sm_scale * kLog2e;
    const uint64_t scale2 = pack2(scale_log2, scale_log2);
    int blind_tok = key0 + r - ahead - first_tile * tile_tokens;         // tokens of the first tile in front of the first seer
    bool alive = true;
    for (int i = 0; i < n; ++i) {
      const int st = i % kStatStages;
      const uint32_t t_s = tmem + lane_base + h * 64 + (i & 1 ? C::kDp : 0), t_dp = tmem + lane_base + h * 64 + (i & 1 ? 0 : C::kDp);
      const ulonglong2* lse4 = reinterpret_cast<const ulonglong2*>(s_lse2 + st * C::kStream + h * 64);        // negated
      const ulonglong2* delta4 = reinterpret_cast<const ulonglong2*>(s_delta + st * C::kStream + h * 64);
      if (!mbar_wait_warp(smem_u32(&ctl->s_full), (uint32_t)i & 1u, abort_flag, p.status) ||
          !mbar_wait_warp(smem_u32(&ctl->stat_full[st]), (uint32_t)(i / kStatStages) & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      uint32_t s[64];
      float pr[64];
      tmem_ld64(t_s, s);
#pragma unroll
      for (int c4 = 0; c4 < 16; ++c4) {
        const ulonglong2 v = lse4[c4];
        float t[4];
        unpack2(ffma2(pack2(__uint_as_float(s[c4 * 4]), __uint_as_float(s[c4 * 4 + 1])), scale2, v.x), t[0], t[1]);
        unpack2(ffma2(pack2(__uint_as_float(s[c4 * 4 + 2]), __uint_as_float(s[c4 * 4 + 3])), scale2, v.y), t[2], t[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) pr[c4 * 4 + j] = ex2(t[j]);
      }
      // causal: columns of tokens in front of key - ahead do not see this key
      const int blind = kCausal ? max(blind_tok, 0) * p.group - h * 64 : 0;
      blind_tok -= tile_tokens;
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
      }
      if (!mbar_wait_warp(smem_u32(&ctl->dp_full), (uint32_t)i & 1u, abort_flag, p.status)) {
        alive = false;
        break;
      }
      tc_fence_after();
      tmem_ld64(t_dp, s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->dp_read));
      {
        const float tau = kScaled<T> ? *(volatile float*)&ctl->tau : 1.f;
        const uint64_t tau2 = pack2(tau, tau);
        auto minus_delta = [&](uint64_t dp, uint64_t neg_delta) { return kScaled<T> ? ffma2(dp, tau2, neg_delta) : fadd2(dp, neg_delta); };
        uint32_t pk[32];
#pragma unroll
        for (int c4 = 0; c4 < 16; ++c4) {
          const ulonglong2 v = delta4[c4];
          float t[4];
          unpack2(fmul2(pack2(pr[c4 * 4], pr[c4 * 4 + 1]), minus_delta(pack2(__uint_as_float(s[c4 * 4]), __uint_as_float(s[c4 * 4 + 1])), v.x)), t[0], t[1]);
          unpack2(fmul2(pack2(pr[c4 * 4 + 2], pr[c4 * 4 + 3]), minus_delta(pack2(__uint_as_float(s[c4 * 4 + 2]), __uint_as_float(s[c4 * 4 + 3])), v.y)), t[2], t[3]);
          pk[c4 * 2] = pack_pair<T>(t[0], t[1]);
          pk[c4 * 2 + 1] = pack_pair<T>(t[2], t[3]);
        }
        tmem_st32(t_s + 32, pk);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&ctl->ds_ready));
          mbar_arrive(smem_u32(&ctl->stat_free[st]));
        }
      }
    }
    // ---- epilogue: warpgroup h stores channels h D / 2 .. of both gradients
    if (alive && n > 0) alive = mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    if (alive) {
      tc_fence_after();
      // read again from shared memory and the thread index: the loop above needs the registers
      asm volatile("" : "+r"(r));
      const int key = *(volatile int*)&ctl->unit.index * kTileM + r;
      const bool row_valid = key < *(volatile int*)&ctl->unit.k.len;
      const long long row = *(volatile int*)&ctl->unit.k.begin + (row_valid ? key : 0);
      const float mul = kScaled<T> && n > 0 ? 1.f / kProbMul : 1.f;
      const float mul_k = kScaled<T> && n > 0 ? p.sm_scale / (kProbMul * *(volatile float*)&ctl->tau) : p.sm_scale;
      T* out[2] = {(T*)p.dv + row * p.dv_stride[0] + kvh * p.dv_stride[1], (T*)p.dk + row * p.dk_stride[0] + kvh * p.dk_stride[1]};
#pragma unroll 1
      for (int which = 0; which < 2; ++which)
        store_share<T, D / kHalves>(RowAddresses(row_valid ? out[which] : nullptr), tmem + lane_base + (which ? C::kSum1 : C::kSum0), h, n > 0,
                         which ? mul_k : mul);
    }
  }
  bwd_teardown<C>(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------ dQ
template <typename T, int D, int kHalves, bool kCausal>
__device__ __forceinline__ void dq_block(const tra_packed_launch& p, uint8_t* smem, const int unit, const int kvh) {
  using C = BwdCfg<D, kHalves>;
  uint8_t* sQ = smem;
  uint8_t* sDO = smem + C::kTileBytes;
  uint8_t* sA = smem + 2 * C::kTileBytes;                   // K tiles
  uint8_t* sB = sA + C::kA * C::kStreamBytes;                 // V tiles
  BwdCtl* ctl = (BwdCtl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const int tile_tokens = p.tile_tokens, box_rows = tile_tokens * p.group;

  // set-up in parallel, one barrier (see the forward kernel)
  if (warp == 0) {
    const tra_unit u = tra_find_unit(p, false, p.max_q <= tile_tokens, tile_tokens, unit);
    if (lane == 0) ctl->unit = u;
  } else if (warp == C::kSoftWarps + 1) {
    tmem_alloc<C::kColumns>(&ctl->tmem_base);
  } else if (tid == 32) {
    bwd_init<kHalves>(ctl);
  } else if (tid == 64) {
    prefetch_map(&p.map_q);
    prefetch_map(&p.map_do);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  if (box_rows < kTileM && warp >= 2 && warp < C::kSoftWarps)        // rows that no box fills
    zero_tile_rows(sQ, box_rows, kTileM, 2 * C::kAtoms, C::kAtomBytes, tid - 64, 32 * (C::kSoftWarps - 2));
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  const tra_seq_range qr = ctl->unit.q, kr = ctl->unit.k;
  // the last tiles, the longest of a causal sequence, come first
  const int tok0 = (ctl->unit.count - 1 - ctl->unit.index) * tile_tokens;
  if (ctl->unit.seq < 0) {
    if (warp == C::kSoftWarps + 1) tmem_free<C::kColumns>(tmem);
    wait_last_launch();          // no block ends before the launch in front of it
    return;
  }
  const int ahead = kr.len - qr.len;
  const int last_tok = min(tok0 + tile_tokens, qr.len) - 1;
  const int keys = kCausal ? min(max(last_tok + 1 + ahead, 0), kr.len) : kr.len;
  const int n_all = (keys + C::kStream - 1) / C::kStream, n = n_all;
  const bool tail_all = n > 0 && n * C::kStream > kr.len, tail = tail_all;
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp >= C::kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsControl));
    if (warp == C::kSoftWarps) {
      // ================================================================== TMA producer
      if (lane == 0) {
        const uint32_t own = smem_u32(&ctl->own_full);
        mbar_expect_tx(own, 2 * C::kAtoms * box_rows * 128);
        for (int a = 0; a < C::kAtoms; ++a) {
          tma_load_3d(smem_u32(sQ + a * C::kAtomBytes), &p.map_q, own, a * 64, kvh * p.group, qr.begin + tok0);
          tma_load_3d(smem_u32(sDO + a * C::kAtomBytes), &p.map_do, own, a * 64, kvh * p.group, qr.begin + tok0);
        }
        bwd_produce<C>(
            ctl, n, tail, C::kStreamBytes, abort_flag, p.status,
            [&](int i, int slot, uint32_t bar) {
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sA + slot * C::kStreamBytes + a * C::kStreamAtom), &p.map_k, bar, a * 64, kvh, kr.begin + i * C::kStream);
            },
            [&](int i, int slot, uint32_t bar) {
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sB + slot * C::kStreamBytes + a * C::kStreamAtom), &p.map_v, bar, a * 64, kvh, kr.begin + i * C::kStream);
            });
      }
    } else if (warp == C::kSoftWarps + 2) {
      // ================================================================== rows past the sequence's end
      if (tail && mbar_wait_warp(smem_u32(&ctl->tail_full), 0u, abort_flag, p.status)) {
        const int row0 = kr.len - (n - 1) * C::kStream;
        zero_tile_rows(sA + ((n - 1) % C::kA) * C::kStreamBytes, row0, C::kStream, C::kAtoms, C::kStreamAtom, lane, 32);
        zero_tile_rows(sB + ((n - 1) % C::kB) * C::kStreamBytes, row0, C::kStream, C::kAtoms, C::kStreamAtom, lane, 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready));
      }
    } else if (warp == C::kSoftWarps + 1) {
      // ================================================================== MMA issuer
      constexpr uint32_t kIdescS = make_idesc_t<T>(C::kStream, false);
      constexpr uint32_t kIdescD = make_idesc_t<T>(D, true);
      constexpr uint32_t kHi = desc_hi(1024);
      const uint32_t q_lo = desc_lo(smem_u32(sQ), 16), do_lo = desc_lo(smem_u32(sDO), 16);
      const uint32_t a_k = desc_lo(smem_u32(sA), 16), a_mn = desc_lo(smem_u32(sA), C::kStreamAtom), b_k = desc_lo(smem_u32(sB), 16);
      constexpr uint32_t kTile = C::kStreamBytes >> 4;
      RingPos<C::kA> ks, kd;                 // K of the next S, of the next dQ
      RingPos<C::kB> vs;
      const uint32_t tmem = uniform(ctl->tmem_base);
      const int n = uniform(n_all);
      const bool tail = uniform(tail_all);
      bool alive = mbar_wait_warp(smem_u32(&ctl->own_full), 0u, abort_flag, p.status);
      // K and V of the next scores and dP are in shared memory
      auto tiles_here = [&](int i) -> bool {
        if (tail && i == n - 1) return mbar_wait_warp(smem_u32(&ctl->tail_ready), 0u, abort_flag, p.status);
        return mbar_wait_warp(smem_u32(&ctl->a_full[ks.slot]), ks.phase, abort_flag, p.status) &&
               mbar_wait_warp(smem_u32(&ctl->b_full[vs.slot]), vs.phase, abort_flag, p.status);
      };
      auto issue_s = [&]() {
        mma_tiles<D>(tmem, q_lo, a_k + (uint32_t)ks.slot * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->s_full));
        ks.next();
      };
      auto issue_dp = [&]() {
        mma_tiles<D>(tmem + C::kDp, do_lo, b_k + (uint32_t)vs.slot * kTile, kIdescS);
        tc_commit(smem_u32(&ctl->dp_full));
        tc_commit(smem_u32(&ctl->b_free[vs.slot]));
        vs.next();
      };
      alive = alive && n > 0 && tiles_here(0);
      if (alive) {
        tc_fence_after();
        issue_s();
        issue_dp();
      }
      for (int i = 0; i < n && alive; ++i) {
        if (i + 1 < n) {
          if (!(alive = tiles_here(i + 1) && mbar_wait_warp(smem_u32(&ctl->s_read), (uint32_t)i & 1u, abort_flag, p.status))) break;
          tc_fence_after();
          issue_s();
          if (!(alive = mbar_wait_warp(smem_u32(&ctl->dp_read), (uint32_t)i & 1u, abort_flag, p.status))) break;
          tc_fence_after();
          issue_dp();
        }
        if (!(alive = mbar_wait_warp(smem_u32(&ctl->ds_ready), (uint32_t)i & 1u, abort_flag, p.status))) break;
        tc_fence_after();
        const uint32_t k_mn = a_mn + (uint32_t)kd.slot * kTile;           // dQ += dS K
#pragma unroll
        for (int kk = 0; kk < 4 * kHalves; ++kk)
          tc_mma_ts(tmem + C::kSum0, tmem + C::kSum1 + kk * 8, k_mn + kk * (2048 >> 4), kHi, kIdescD, kk > 0 ? 1u : (i > 0 ? 1u : 0u));
        tc_commit(smem_u32(&ctl->a_free[kd.slot]));
        kd.next();
      }
      tc_commit(smem_u32(&ctl->drain));
      mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
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
    wait_last_launch();                                      // delta
    if (row_valid) {
      const float v = p.lse[tok_g * p.heads + head] * kLog2e;
      lse2 = v == -INFINITY ? INFINITY : v;
      delta = p.delta[tok_g * p.heads + head];
    }
    const float tau = kScaled<T> && n > 0 ? grad_tau(p, kvh) * kProbMul : 1.f;      // dS times it, as in dkv_block
    delta *= tau;
    const uint64_t scale2 = pack2(scale_log2, scale_log2), neg_lse2 = pack2(-lse2, -lse2), neg_delta2 = pack2(-delta, -delta);
    const uint64_t tau2 = pack2(tau, tau);
    const int seen = kCausal ? min(max(min(tok, last_tok) + 1 + ahead, 0), kr.len) : kr.len;
    RingPos<C::kA> kd;                                       // K of the step before
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
      for (int c = 0; c < 64; c += 2) {
        float t0, t1;
        unpack2(ffma2(pack2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), scale2, neg_lse2), t0, t1);
        pr[c] = ex2(t0), pr[c + 1] = ex2(t1);
      }
      const int limit = seen - i * C::kStream - h * 64;          // columns at and past it are not seen
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
      tmem_ld64(tmem + lane_base + C::kDp + h * 64, s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->dp_read));
      uint32_t pk[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        float t0, t1;
        const uint64_t dp = pack2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1]));
        unpack2(fmul2(pack2(pr[2 * c], pr[2 * c + 1]), kScaled<T> ? ffma2(dp, tau2, neg_delta2) : fadd2(dp, neg_delta2)), t0, t1);
        pk[c] = pack_pair<T>(t0, t1);
      }
      // the product that read the last dS has retired (it also freed that stage)
      if (i > 0) {
        if (!mbar_wait_warp(smem_u32(&ctl->a_free[kd.slot]), kd.phase, abort_flag, p.status)) {
          alive = false;
          break;
        }
        kd.next();
      }
      tc_fence_after();
      tmem_st32(tmem + lane_base + C::kSum1 + h * 32, pk);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->ds_ready));
    }
    if (alive && n > 0) alive = mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    if (alive) {
      tc_fence_after();
      T* out = (T*)p.dq + tok_g * p.dq_stride[0] + head * p.dq_stride[1];
      store_share<T, D / kHalves>(RowAddresses(row_valid ? out : nullptr), tmem + lane_base + C::kSum0, h, n > 0, kScaled<T> ? p.sm_scale / tau : p.sm_scale);
    }
  }
  bwd_teardown<C>(ctl, tmem, warp);
}

// ------------------------------------------------------------------------------------ both
// Blocks of either kind in one launch, so that the shorter dQ blocks fill the SMs that the last dK/dV blocks leave: first
// dkv_units per key/value head, then dq_units.  Of a causal sequence the first keys and the last queries have most to
// do, and come first.
template <typename T, int D, int kHalves, bool kCausal>
__global__ void __launch_bounds__(BwdCfg<D, kHalves>::kThreads, BwdCfg<D, kHalves>::kBlocks)
    tra_packed_bwd_kernel(const __grid_constant__ tra_packed_launch p, int dkv_units, int dq_units) {
  extern __shared__ __align__(1024) uint8_t smem[];         // the swizzled tiles start on 1024-byte boundaries
  const int n_dkv = dkv_units * p.kv_heads, b = blockIdx.x;
  if (b < n_dkv)
    dkv_block<T, D, kHalves, kCausal>(p, smem, b % dkv_units, b / dkv_units);
  else
    dq_block<T, D, kHalves, kCausal>(p, smem, (b - n_dkv) % dq_units, (b - n_dkv) / dq_units);
}

// ------------------------------------------------------------------------------------ delta
// delta = sum over the channels of dO O, d / 8 threads per (token, head), 16 bytes each.  O with what its rounding took, when the
// forward call kept it: P (dP - delta) cancels where a row sees few keys or one dominates, and there the rounding of O is
// the larger part of what is left (two tokens, bf16: 9.4e-3 of a gradient, 3.3e-3 with the remainder).
// One thread's share of a row: eight channels of dO (o and its remainder).
template <typename T, int D>
__device__ __forceinline__ float delta_share(const tra_packed_launch& p, long long tok, int head, int lane, const uint4& d_o) {
  const uint4 a = *reinterpret_cast<const uint4*>((const T*)p.o_in + tok * p.o_stride[0] + head * p.o_stride[1] + lane * 8);
  const uint4 c = p.o_rest ? *reinterpret_cast<const uint4*>((const T*)p.o_rest + (tok * p.heads + head) * D + lane * 8) : make_uint4(0u, 0u, 0u, 0u);
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {d_o.x, d_o.y, d_o.z, d_o.w}, z[4] = {c.x, c.y, c.z, c.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x0, x1, y0, y1, z0, z1;
    unpack_pair<T>(x[i], x0, x1);
    unpack_pair<T>(y[i], y0, y1);
    unpack_pair<T>(z[i], z0, z1);
    x0 += z0;
    x1 += z1;
    s = fmaf(x0, y0, s);
    s = fmaf(x1, y1, s);
  }
  return s;
}
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float s) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
template <typename T>
__device__ __forceinline__ const uint4& row_piece(const void* base, const long long* stride, long long tok, int head, int lane) {
  return *reinterpret_cast<const uint4*>((const T*)base + tok * stride[0] + head * stride[1] + lane * 8);
}

template <typename T, int D>
__global__ void __launch_bounds__(256) tra_packed_delta_kernel(const __grid_constant__ tra_packed_launch p) {
  constexpr int kLanes = D / 8;
  allow_next_launch();
  const long long row = (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const int lane = threadIdx.x % kLanes;
  const long long rows = (long long)p.total_q * p.heads;
  float s = 0.f;
  if (row < rows) {
    const long long tok = row / p.heads;
    const int head = (int)(row - tok * p.heads);
    s = delta_share<T, D>(p, tok, head, lane, row_piece<T>(p.d_o, p.do_stride, tok, head, lane));
  }
  s = sum_lanes<kLanes>(s);
  if (row < rows && lane == 0) p.delta[row] = s;
}

// fp16: delta, and the largest squared norms behind grad_tau, of the rows of dO and of V that belong to a sequence and are finite.  A block
// takes `steps` times 256 / (d / 8) tokens of one head, first the heads of dO, then those of V, and leaves one atomic maximum behind (rows
// of mixed heads, as above, would leave one each: 12 -> 25 us at 14,040 tokens, 12 heads, d 64).
template <int D>
__global__ void __launch_bounds__(256) tra_packed_delta_norms_kernel(const __grid_constant__ tra_packed_launch p, int q_blocks, int steps) {
  using T = __half;
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;
  __shared__ uint32_t s_largest[8];
  allow_next_launch();
  const int lane = threadIdx.x % kLanes;
  const bool of_v = (int)blockIdx.x >= q_blocks;
  const int heads = of_v ? p.kv_heads : p.heads, total = of_v ? p.total_k : p.total_q;
  const int b = (int)blockIdx.x - (of_v ? q_blocks : 0), head = b % heads;
  const int from = of_v ? p.k_begin[0] : p.cu_q[0], to = of_v ? p.k_end[p.n_seq - 1] : p.cu_q[p.n_seq];
  long long tok = (long long)(b / heads) * steps * kRows + threadIdx.x / kLanes;
  float largest = 0.f;
  for (int i = 0; i < steps; ++i, tok += kRows) {
    const bool there = tok < total, counts = there && tok >= from && tok < to;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    float dot = 0.f, squares = 0.f;
    if (of_v) {
      if (counts) x = row_piece<T>(p.v, p.v_stride, tok, head, lane);
    } else if (there) {
      x = row_piece<T>(p.d_o, p.do_stride, tok, head, lane);
      dot = delta_share<T, D>(p, tok, head, lane, x);
    }
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float lo, hi;
      unpack_pair<T>(w[k], lo, hi);
      squares = fmaf(lo, lo, fmaf(hi, hi, squares));
    }
    squares = sum_lanes<kLanes>(squares);
    if (!of_v) {
      dot = sum_lanes<kLanes>(dot);
      if (there && lane == 0) p.delta[tok * p.heads + head] = dot;
    }
    if (counts && squares < INFINITY) largest = fmaxf(largest, squares);
  }
  const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(largest));
  if ((threadIdx.x & 31) == 0) s_largest[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x < 32) {
    const uint32_t all = __reduce_max_sync(0xffffffffu, threadIdx.x < 8 ? s_largest[threadIdx.x] : 0u);
    if (threadIdx.x == 0 && all) atomicMax(p.norms + (of_v ? p.kv_heads + head : head / p.group), all);
  }
}

template <int D>
int launch_delta_norms(const tra_packed_ctx& c, const tra_packed_launch& a) {
  constexpr int kRows = 256 / (D / 8);
  const long long q = ((long long)a.total_q + kRows - 1) / kRows, v = ((long long)a.total_k + kRows - 1) / kRows;
  const long long most = 32ll * c.h->sm_count;           // four times what runs at once
  const long long steps = (q * a.heads + v * a.kv_heads + most - 1) / most;
  const long long q_blocks = (q + steps - 1) / steps * a.heads, v_blocks = (v + steps - 1) / steps * a.kv_heads;
  if (cudaMemsetAsync(a.norms, 0, 2 * sizeof(uint32_t) * a.kv_heads, c.stream) != cudaSuccess) return TRA_ERR_CUDA;
  return tra_launch(tra_packed_delta_norms_kernel<D>, dim3((unsigned)(q_blocks + v_blocks)), 256, 0, c.stream, false, 1, a, (int)q_blocks, (int)steps);
}

template <typename T, int D, int kHalves, bool kCausal>
int launch_bwd(const tra_packed_ctx& c, const tra_packed_launch& a) {
  const long long rows = (long long)a.total_q * a.heads;
  int rc = TRA_OK;
  if (rows > 0) {
    constexpr int kRows = 256 / (D / 8);
    if constexpr (kScaled<T>)
      rc = launch_delta_norms<D>(c, a);
    else
      rc = tra_launch(tra_packed_delta_kernel<T, D>, dim3((unsigned)((rows + kRows - 1) / kRows)), 256, 0, c.stream, false, 1, a);
    if (rc != TRA_OK) return rc;
  }
  const int dkv_units = a.max_k > 0 ? (a.max_k <= kTileM ? 0 : a.total_k / kTileM) + a.n_seq : 0;
  const int dq_units = a.max_q > 0 ? (a.max_q <= a.tile_tokens ? 0 : a.total_q / a.tile_tokens) + a.n_seq : 0;
  const long long blocks = ((long long)dkv_units + dq_units) * a.kv_heads;
  if (blocks == 0) return TRA_OK;
  if (blocks > 0x7fffffffll) return TRA_ERR_UNSUPPORTED;
  using C = BwdCfg<D, kHalves>;
  constexpr auto kern = tra_packed_bwd_kernel<T, D, kHalves, kCausal>;
  if ((rc = tra_allow_smem<kern>(C::kSmemBytes)) != TRA_OK) return rc;
  return tra_launch(kern, dim3((unsigned)blocks), C::kThreads, C::kSmemBytes, c.stream, rows > 0, 1, a, dkv_units, dq_units);
}

template <int D, int kHalves>
int launch_bwd_shape(const tra_packed_ctx& c, const tra_packed_launch& a) {
  if (c.h->cfg.dtype == TRA_BF16)
    return a.causal ? launch_bwd<__nv_bfloat16, D, kHalves, true>(c, a) : launch_bwd<__nv_bfloat16, D, kHalves, false>(c, a);
  return a.causal ? launch_bwd<__half, D, kHalves, true>(c, a) : launch_bwd<__half, D, kHalves, false>(c, a);
}

}  // namespace
