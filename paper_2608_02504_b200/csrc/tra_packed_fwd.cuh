// Attention over packed sequences, forward: causal or not, grouped heads, whole prompts, chunks behind a cache, and
// (split over the keys) few rows over many keys.  The kernel template and its launcher.
//
// A row is one (token, query head); the rows of a sequence that share a key/value head are token-major, so 128
// consecutive ones are tile_tokens = 128 / group tokens times the group's heads: one 3-D TMA box.  Grouped heads
// cost nothing then: a key/value tile is fetched once for all the heads that share it, and a causal tile's diagonal
// is as narrow as its few tokens.  One thread block owns two neighbouring 128-row tiles of one (sequence,
// key/value head) and walks the key blocks of 128 that the later tile sees; warps, tensor-memory columns and the order
// of the tensor pipe per key block (PV_0, S_0 of the next, PV_1, S_1 of the next) are those of the dense launch in
// tra_attn_kernel.cuh.  The earlier tile stops at its own last block.  Blocks whose 128 keys are all seen by all rows of a
// warp skip the mask.
//
// Keys past a sequence's end belong to another sequence or to nobody, and may hold anything.  Their scores are
// replaced before they are looked at; their V rows would still meet the zero probabilities in the product (0 * NaN), so an
// idle warp zeroes them in shared memory before the tensor pipe reads that last tile.
//
// Split launches (gridDim.z > 1) give every block a range of the key blocks; the parts O / l and log2 l go to a
// workspace and tra_packed_join_kernel adds them.
//
// Bound: tensor cores, at the power cap (see tra_attn_kernel.cuh), for long sequences.
#pragma once
#include <cuda_fp16.h>

#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kFwdThreads = 384;
constexpr int kFwdRegsSoftmax = 216;     // 2 * 216 + 72 = 3 * 168, the registers of the launch
constexpr int kFwdRegsControl = 72;
constexpr int kKeyTile = 128;

template <int D>
struct FwdCfg {
  static constexpr int kTileBytes = kTileM * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 6;
  static constexpr int kAtoms = D / 64;
  static constexpr int kAtomBytes = kTileM * 128;
  static constexpr int kSmemData = (2 + kSlots) * kTileBytes;
  static constexpr int kSmemNeeded = kSmemData + 1024 /*alignment slack*/ + 512 /*barriers*/;
  // at least 120 KB so that one block owns an SM and its whole tensor memory
  static constexpr int kSmemBytes = kSmemNeeded > 120 * 1024 ? kSmemNeeded : 120 * 1024;
};

struct FwdCtl {
  uint64_t q_full;
  uint64_t kv_full[6];
  uint64_t kv_release[8];
  uint64_t s_full[2];
  uint64_t p_ready[2][2];     // [tile][64-key half]
  uint64_t tail_full, tail_ready;   // the V tile that reaches past the sequence's end: loaded; its foreign rows zeroed
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
  tra_unit unit;
};
static_assert(sizeof(FwdCtl) <= 512, "control block");

template <typename T, int D, bool kCausal, bool kExact>
__global__ void __launch_bounds__(kFwdThreads, 1) tra_packed_fwd_kernel(const __grid_constant__ tra_packed_launch p) {
  using C = FwdCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;
  uint8_t* sKV = smem + 2 * C::kTileBytes;
  FwdCtl* ctl = (FwdCtl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kvh = blockIdx.y;
  // the last tiles of a causal sequence are the longest: launched first
  const int unit = p.n_units - 1 - (int)blockIdx.x;

  const int box_rows = p.tile_tokens * p.group;
  // set-up in parallel, one barrier: the block's unit, the mbarriers, tensor memory, and zeros in the rows of the query tiles
  // that no box fills (group does not divide 128), so that they stay harmless
  if (warp == 0) {
    const tra_unit u = tra_find_unit(p, false, p.max_q <= 2 * p.tile_tokens, 2 * p.tile_tokens, unit);
    if (lane == 0) ctl->unit = u;
  } else if (warp == 9) {
    tmem_alloc_all(&ctl->tmem_base);
  } else if (tid == 32) {
    mbar_init(smem_u32(&ctl->q_full), 1);
    for (int i = 0; i < C::kSlots; ++i) mbar_init(smem_u32(&ctl->kv_full[i]), 1);
    for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&ctl->kv_release[i]), 1);
    for (int k = 0; k < 2; ++k) {
      mbar_init(smem_u32(&ctl->s_full[k]), 1);
      mbar_init(smem_u32(&ctl->p_ready[k][0]), 4);
      mbar_init(smem_u32(&ctl->p_ready[k][1]), 4);
    }
    mbar_init(smem_u32(&ctl->tail_full), 1);
    mbar_init(smem_u32(&ctl->tail_ready), 1);
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (tid == 64) {
    prefetch_map(&p.map_q);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  if (box_rows < kTileM && warp >= 2 && warp < 8) zero_tile_rows(sQ, box_rows, kTileM, 2 * C::kAtoms, C::kAtomBytes, tid - 64, 192);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (gridDim.z > 1) allow_next_launch();                 // the join of the parts
  const uint32_t tmem = ctl->tmem_base;
  const tra_seq_range qr = ctl->unit.q, kr = ctl->unit.k;
  const int tok0 = ctl->unit.index * 2 * p.tile_tokens;   // first token of tile 0, inside the sequence
  if (ctl->unit.seq < 0 || tok0 >= qr.len) {              // past the last unit, or a sequence without queries
    if (warp == 9) tmem_free_all(tmem);
    return;
  }
  const int ahead = kr.len - qr.len;                      // causal: token i sees keys 0 .. i + ahead
  // keys the last token of a tile sees, and the tile's key blocks
  auto tile_keys = [&](int k) -> int {
    const int first = tok0 + k * p.tile_tokens;
    if (first >= qr.len) return 0;
    const int last = min(first + p.tile_tokens, qr.len) - 1;
    return kCausal ? min(max(last + 1 + ahead, 0), kr.len) : kr.len;
  };
  const int nb0 = (tile_keys(0) + kKeyTile - 1) / kKeyTile, nb1 = (tile_keys(1) + kKeyTile - 1) / kKeyTile;
  const int nb = max(nb0, nb1);                           // nb0 <= nb1 when there is a second tile
  const int per_split = (nb + (int)gridDim.z - 1) / (int)gridDim.z;
  const int v_begin = min((int)blockIdx.z * per_split, nb), v_end = min(v_begin + per_split, nb);
  const int n_entries = v_end - v_begin;
  const int n_own[2] = {max(min(nb0, v_end) - v_begin, 0), max(min(nb1, v_end) - v_begin, 0)};
  const bool tail = n_entries > 0 && v_end * kKeyTile > kr.len;      // the last V tile reaches past the sequence
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFwdRegsControl));
    if (warp == 8) {
      // ================================================================== TMA producer
      if (lane == 0) {
        const uint32_t qbar = smem_u32(&ctl->q_full);
        mbar_expect_tx(qbar, 2 * C::kAtoms * box_rows * 128);
        for (int k = 0; k < 2; ++k)                // a missing tile loads rows nobody uses (past the tensor: zeros)
          for (int a = 0; a < C::kAtoms; ++a)
            tma_load_3d(smem_u32(sQ + k * C::kTileBytes + a * C::kAtomBytes), &p.map_q, qbar, a * 64, kvh * p.group,
                        qr.begin + tok0 + k * p.tile_tokens);
        // loads K0, V0, K1, V1, ... into consecutive slots; load j is freed by release event (j + 1) / 2
        int slot = 0, n_load = 0;
        bool alive = true;
        for (int e = 0; e < n_entries && alive; ++e) {
          for (int kv = 0; kv < 2; ++kv) {
            if (n_load >= C::kSlots) {
              const int r = (n_load - C::kSlots + 1) >> 1;
              if (!mbar_wait(smem_u32(&ctl->kv_release[r & 7]), (uint32_t)(r >> 3) & 1u, abort_flag, p.status)) {
                alive = false;
                break;
              }
            }
            ++n_load;
            const uint32_t bar = smem_u32(kv == 1 && tail && e == n_entries - 1 ? &ctl->tail_full : &ctl->kv_full[slot]);
            mbar_expect_tx(bar, C::kTileBytes);
            for (int a = 0; a < C::kAtoms; ++a)
              tma_load_3d(smem_u32(sKV + slot * C::kTileBytes + a * C::kAtomBytes), kv == 0 ? &p.map_k : &p.map_v, bar,
                          a * 64, kvh, kr.begin + (v_begin + e) * kKeyTile);
            if (++slot == C::kSlots) slot = 0;
          }
        }
      }
    } else if (warp == 10) {
      // ================================================================== rows past the sequence's end
      if (tail) {
        if (mbar_wait_warp(smem_u32(&ctl->tail_full), 0u, abort_flag, p.status)) {
          const int slot = (2 * n_entries - 1) % C::kSlots;
          zero_tile_rows(sKV + slot * C::kTileBytes, kr.len - (v_end - 1) * kKeyTile, kKeyTile, C::kAtoms, C::kAtomBytes,
                         lane, 32);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready));
        }
      }
    } else if (warp == 9) {
      // ================================================================== MMA issuer
      constexpr uint32_t kIdescQK = make_idesc_t<T>(kKeyTile, false);
      constexpr uint32_t kIdescPV = make_idesc_t<T>(D, true);
      bool alive = mbar_wait(smem_u32(&ctl->q_full), 0u, abort_flag, p.status);
      tc_fence_after();
      constexpr uint32_t kHi = desc_hi(1024);
      const uint32_t q_lo0 = desc_lo(smem_u32(sQ), 16), q_lo1 = desc_lo(smem_u32(sQ + C::kTileBytes), 16);
      const uint32_t k_lo0 = desc_lo(smem_u32(sKV), 16), v_lo0 = desc_lo(smem_u32(sKV), C::kAtomBytes);
      auto issue_s = [&](int k, int kslot) {
        const uint32_t qa = k ? q_lo1 : q_lo0, ka = k_lo0 + (uint32_t)kslot * (C::kTileBytes >> 4);
        const uint32_t d = tmem + k * 128;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * C::kAtomBytes + (kk & 3) * 32) >> 4;
          tc_mma_ss(d, qa + off, kHi, ka + off, kHi, kIdescQK, kk > 0 ? 1u : 0u);
        }
        tc_commit(smem_u32(&ctl->s_full[k]));
      };
      auto issue_pv = [&](int k, int vslot, uint32_t parity, uint32_t started) -> bool {
        const uint32_t va = v_lo0 + (uint32_t)vslot * (C::kTileBytes >> 4);
        const uint32_t d = tmem + 256 + k * 128, pa = tmem + k * 128;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!mbar_wait(smem_u32(&ctl->p_ready[k][half]), parity, abort_flag, p.status)) return false;
          tc_fence_after();
#pragma unroll
          for (int kk = half * 4; kk < half * 4 + 4; ++kk)
            tc_mma_ts(d, pa + kk * 8, va + kk * (2048 >> 4), kHi, kIdescPV, kk > 0 ? 1u : started);
        }
        return true;
      };
      int slot = 0;
      uint32_t phase = 0;
      auto advance = [&]() {
        if (++slot == C::kSlots) {
          slot = 0;
          phase ^= 1u;
        }
      };
      if (alive && n_entries > 0) {
        alive = mbar_wait(smem_u32(&ctl->kv_full[slot]), phase, abort_flag, p.status);       // first K tile
        if (alive) {
          tc_fence_after();
          for (int k = 0; k < 2; ++k)
            if (n_own[k] > 0) issue_s(k, slot);
          tc_commit(smem_u32(&ctl->kv_release[0]));            // release event 0: K0
          advance();
        }
      }
      uint32_t n_release = 1;
      for (int e = 0; e < n_entries && alive; ++e) {
        const int vslot = slot;
        const uint32_t vphase = phase;
        advance();
        const int kslot = slot;
        const uint32_t kphase = phase;
        const bool have_next = e + 1 < n_entries;
        const bool v_tail = tail && !have_next;
        alive = v_tail ? mbar_wait(smem_u32(&ctl->tail_ready), 0u, abort_flag, p.status)
                       : mbar_wait(smem_u32(&ctl->kv_full[vslot]), vphase, abort_flag, p.status);
        bool k_ready = false;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (!alive || e >= n_own[k]) continue;
          alive = issue_pv(k, vslot, (uint32_t)e & 1u, e > 0 ? 1u : 0u);
          if (!alive) break;
          if (e + 1 < n_own[k]) {
            if (!k_ready) {
              alive = mbar_wait(smem_u32(&ctl->kv_full[kslot]), kphase, abort_flag, p.status);
              k_ready = true;
              if (!alive) break;
              tc_fence_after();
            }
            issue_s(k, kslot);
          }
        }
        if (!alive) break;
        tc_commit(smem_u32(&ctl->kv_release[n_release & 7u]));     // V of this block and K of the next
        ++n_release;
        if (have_next) advance();
      }
      tc_commit(smem_u32(&ctl->drain));
      mbar_wait(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFwdRegsSoftmax));
    // ================================================================== softmax + epilogue
    const int k = warp >> 2;
    int r = tid & (kTileM - 1);
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_o = tmem + lane_base + 256 + k * 128, t_s = tmem + lane_base + k * 128;
    const int n = n_own[k];
    float m = -INFINITY, l = 0.f, l_exact = 0.f;
    bool alive = true;
    if ((warp & 3) * 32 >= box_rows || tok0 + k * p.tile_tokens + (warp & 3) * 32 / p.group >= qr.len) {
      // a warp without a row keeps up with the barriers; what its lanes multiply stays in its own, unstored rows
      for (int e = 0; e < n && alive; ++e) {
        alive = mbar_wait_warp(smem_u32(&ctl->s_full[k]), (uint32_t)e & 1u, abort_flag, p.status);
        if (alive && lane == 0) {
          mbar_arrive(smem_u32(&ctl->p_ready[k][0]));
          mbar_arrive(smem_u32(&ctl->p_ready[k][1]));
        }
        __syncwarp();
      }
    } else {
      const float scale_log2 = p.sm_scale * kLog2e;
      // columns of the first block that the row sees; rows that hold no query follow the tile's last one, so that they force
      // no mask on their warp
      const int mask_tok = min(tok0 + k * p.tile_tokens + r / p.group, min(tok0 + (k + 1) * p.tile_tokens, qr.len) - 1);
      int col_limit = (kCausal ? min(max(mask_tok + 1 + ahead, 0), kr.len) : kr.len) - v_begin * kKeyTile;
      for (int e = 0; e < n; ++e, col_limit -= kKeyTile) {
        if (!mbar_wait_warp(smem_u32(&ctl->s_full[k]), (uint32_t)e & 1u, abort_flag, p.status)) {
          alive = false;
          break;
        }
        tc_fence_after();
        uint32_t sb[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &sb[c * 32]);
        tmem_wait_ld(&sb[0]);
#pragma unroll
        for (int c = 1; c < 4; ++c) reg_fence32(&sb[c * 32]);
        if (__any_sync(0xffffffffu, col_limit < kKeyTile)) {
#pragma unroll
          for (int j = 0; j < 128; ++j)
            if (j >= col_limit) sb[j] = 0xff800000u;                  // -inf
        }
        float mx0 = __uint_as_float(sb[0]), mx1 = __uint_as_float(sb[1]);
#pragma unroll
        for (int j = 2; j + 3 < 128; j += 4) {
          mx0 = fmax3(mx0, __uint_as_float(sb[j]), __uint_as_float(sb[j + 1]));
          mx1 = fmax3(mx1, __uint_as_float(sb[j + 2]), __uint_as_float(sb[j + 3]));
        }
        mx0 = fmax3(mx0, __uint_as_float(sb[126]), __uint_as_float(sb[127]));
        const float m_blk = fmaxf(mx0, mx1) * scale_log2;
        float alpha = 1.f;
        if (m_blk > m + kRescaleThreshold) {          // also the first block that holds a key (m = -inf)
          alpha = ex2(m - m_blk);
          l *= alpha;
          l_exact *= alpha;
          m = m_blk;
        }
        if (__any_sync(0xffffffffu, alpha != 1.f) && e > 0) {
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(t_o + c * 32, o);
            tmem_wait_ld(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
            tmem_st32(t_o + c * 32, o);
          }
        }
        const float neg_m = m > -INFINITY ? -m : 0.f;       // no key seen so far: every score is -inf
        const uint64_t scale2 = pack2(scale_log2, scale_log2), neg_m2 = pack2(neg_m, neg_m);
        float l_lo = 0.f, l_hi = 0.f;
        uint64_t e2 = 0ull;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const uint64_t t2 =
                ffma2(pack2(__uint_as_float(sb[c * 32 + j]), __uint_as_float(sb[c * 32 + j + 1])), scale2, neg_m2);
            float t0, t1;
            unpack2(t2, t0, t1);
            const float x0 = ex2(t0), x1 = ex2(t1);
            // the sum that normalises O is taken over the rounded probabilities the product uses (numerator and
            // denominator agree); lse keeps the unrounded one
            const uint32_t packed = pack_pair<T>(x0, x1);
            add_pair<T>(l_lo, l_hi, packed);
            if (kExact) e2 = fadd2(e2, pack2(x0, x1));
            pk[j >> 1] = packed;
          }
          tmem_st16(t_s + c * 16, pk);
          if (c & 1) {
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->p_ready[k][c >> 1]));
          }
        }
        l += l_lo + l_hi;
        if (kExact) {
          float a, b;
          unpack2(e2, a, b);
          l_exact += a + b;
        }
      }
    }

    // ---- epilogue --------------------------------------------------------------------------
    if (alive && n > 0) alive = mbar_wait_warp(smem_u32(&ctl->drain), 0u, abort_flag, p.status);
    // Read again from shared memory and the thread index: the loop above needs every register for the score row.
    asm volatile("" : "+r"(r));
    tra_unit own;
    own.index = *(volatile int*)&ctl->unit.index;
    own.q.begin = *(volatile int*)&ctl->unit.q.begin;
    own.q.len = *(volatile int*)&ctl->unit.q.len;
    const int tok = own.index * 2 * p.tile_tokens + k * p.tile_tokens + r / p.group;     // inside the sequence
    const int r_head = r % p.group;
    const bool row_valid = r < p.tile_tokens * p.group && tok < own.q.len;
    if (alive) {
      tc_fence_after();
      const float inv_l = l > 0.f ? 1.f / l : 0.f;
      const long long tok_g = own.q.begin + (row_valid ? tok : 0);
      const int head = kvh * p.group + (row_valid ? r_head : 0);
      const long long row_g = tok_g * p.heads + head;
      T* orow = (T*)p.o + tok_g * p.o_stride[0] + head * p.o_stride[1];
      const bool parts = gridDim.z > 1;
      const long long part_row = (long long)blockIdx.z * p.total_q * p.heads + row_g;
      float4* prow = (float4*)(p.part_o + part_row * D);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o_bits[32];
        float o[32];
        if (n > 0) {
          tmem_ld32(t_o + c * 32, o_bits);
          tmem_wait_ld(o_bits);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = l != 0.f ? __uint_as_float(o_bits[j]) * inv_l : 0.f;
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = 0.f;
        }
        if (row_valid) {
          if (parts) {
#pragma unroll
            for (int q4 = 0; q4 < 8; ++q4)
              prow[c * 8 + q4] = make_float4(o[q4 * 4], o[q4 * 4 + 1], o[q4 * 4 + 2], o[q4 * 4 + 3]);
          } else {
            uint4* dst = (uint4*)(orow + c * 32);
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
              dst[q4] = make_uint4(pack_pair<T>(o[q4 * 8], o[q4 * 8 + 1]), pack_pair<T>(o[q4 * 8 + 2], o[q4 * 8 + 3]),
                                   pack_pair<T>(o[q4 * 8 + 4], o[q4 * 8 + 5]), pack_pair<T>(o[q4 * 8 + 6], o[q4 * 8 + 7]));
          }
        }
      }
      if (row_valid) {
        if (parts) {
          p.part_lse2[part_row] = l > 0.f ? m + log2f(l) : (l != l ? l : -INFINITY);
          if (kExact) p.part_exact[part_row] = l_exact > 0.f ? m + log2f(l_exact) : (l != l ? l : -INFINITY);
        } else if (kExact) {
          p.lse[row_g] = l_exact > 0.f ? (m + log2f(l_exact)) * kLn2 : (l != l ? l : -INFINITY);
        }
      }
    }
  }

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

template <typename T, int D, bool kCausal, bool kExact>
int launch_fwd(const tra_packed_ctx& c, const tra_packed_launch& a) {
  constexpr auto kern = tra_packed_fwd_kernel<T, D, kCausal, kExact>;
  const int rc = tra_allow_smem<kern>(FwdCfg<D>::kSmemBytes, c.h->device);
  if (rc != TRA_OK) return rc;
  return tra_launch(kern, dim3((unsigned)a.n_units, (unsigned)a.kv_heads, (unsigned)a.splits), kFwdThreads, FwdCfg<D>::kSmemBytes,
                    c.stream, false, 1, a);
}

template <int D>
int launch_fwd_shape(const tra_packed_ctx& c, const tra_packed_launch& a) {
  const bool exact = a.lse != nullptr;
  if (c.h->cfg.dtype == TRA_BF16) {
    if (a.causal) return exact ? launch_fwd<__nv_bfloat16, D, true, true>(c, a) : launch_fwd<__nv_bfloat16, D, true, false>(c, a);
    return exact ? launch_fwd<__nv_bfloat16, D, false, true>(c, a) : launch_fwd<__nv_bfloat16, D, false, false>(c, a);
  }
  if (a.causal) return exact ? launch_fwd<__half, D, true, true>(c, a) : launch_fwd<__half, D, true, false>(c, a);
  return exact ? launch_fwd<__half, D, false, true>(c, a) : launch_fwd<__half, D, false, false>(c, a);
}

}  // namespace
