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
// P is rounded to the 16-bit type, the only operand type of the product with V that keeps its rate; the sum that divides O is
// taken over the rounded values, so that what is left of the rounding is u sum p |v - o|.
//
// Split launches give every unit a range of the key blocks; the parts O / l and log2 l go to a
// workspace and tra_packed_join_kernel adds them.
//
// Bound: tensor cores, at the power cap (see tra_attn_kernel.cuh), for long sequences: two of 32,760 tokens and one of 10,921, 12 heads, d
// 128, 11.1 ms (1,250 TFLOP/s); eight causal prompts of 1 to 8,192 tokens, 40 / 8 heads, 775 us (1,180 TFLOP/s), 0.9 ms back to back.
#pragma once
#include <cuda_fp16.h>

#include "tra_packed.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kFwdThreads = 384;
constexpr int kFwdRegsSoftmax = 216;     // 2 * 216 + 72 = 3 * 168, the registers of the launch
constexpr int kFwdRegsControl = 72;
constexpr int kKeyTile = 128;
constexpr int kAskAhead = 1;             // key blocks a unit's producer has left to load when the next unit is asked for

template <int D>
struct FwdCfg {
  static constexpr int kTileBytes = kTileM * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 6;
  static constexpr int kAtoms = D / 64;
  static constexpr int kAtomBytes = kTileM * 128;
  static constexpr int kSmemData = (2 + kSlots) * kTileBytes;
  static constexpr int kSmemNeeded = kSmemData + 512 /*barriers*/;
  // at least 120 KB so that one block owns an SM and its whole tensor memory
  static constexpr int kSmemBytes = kSmemNeeded > 120 * 1024 ? kSmemNeeded : 120 * 1024;
};

// One unit of work: a pair of query tiles of a (sequence, key/value head), over one part of its key blocks.
struct FwdWork {
  tra_unit unit;             // unit.seq = -1: no more work
  int kvh, split;
};

struct FwdCtl {
  uint4 launch;               // answer to the scheduler's request for another block's work
  uint64_t launch_full;
  uint64_t want;              // the producer nears the end of its unit
  uint64_t work_full[2], work_free[2];
  uint64_t q_full, q_free;
  uint64_t kv_full[6];
  uint64_t kv_release[8];
  uint64_t s_full[2];
  uint64_t p_ready[2][2];     // [tile][64-key half]
  uint64_t o_full[2], o_free[2];    // [tile]: the last product of a unit has retired / its sum has been read
  uint64_t tail_full[2], tail_ready[2];   // V tiles that reach past the sequence's end: loaded; their foreign rows zeroed
  uint64_t drain;
  int freed_by[6];            // release event that frees a slot's tile (producer only)
  int tail_slot[2];
  uint32_t tmem_base;
  int abort_flag;
  FwdWork work[2];
};
static_assert(sizeof(FwdCtl) <= 512, "control block");

// What a unit asks of every role.
template <bool kCausal>
struct FwdPlan {
  int tok0;                   // first token of tile 0, inside the sequence
  int v_begin, n_entries;     // key blocks v_begin .. v_begin + n_entries - 1
  int n_own[2];               // entries of each tile (n_own[0] <= n_own[1] where there is a second tile)
  bool tail;                  // the last V tile reaches past the sequence
  __device__ __forceinline__ FwdPlan(const FwdWork& w, const tra_packed_launch& p) {
    const int q_len = w.unit.q.len, k_len = w.unit.k.len;
    tok0 = w.unit.index * 2 * p.tile_tokens;
    const int ahead = k_len - q_len;                      // causal: token i sees keys 0 .. i + ahead
    int blocks[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int first = tok0 + k * p.tile_tokens;
      const int last = min(first + p.tile_tokens, q_len) - 1;
      const int keys = first >= q_len ? 0 : kCausal ? min(max(last + 1 + ahead, 0), k_len) : k_len;
      blocks[k] = (keys + kKeyTile - 1) / kKeyTile;
    }
    const int nb = max(blocks[0], blocks[1]);
    const int per_split = (nb + p.splits - 1) / p.splits;
    v_begin = min(w.split * per_split, nb);
    const int v_end = min(v_begin + per_split, nb);
    n_entries = v_end - v_begin;
#pragma unroll
    for (int k = 0; k < 2; ++k) n_own[k] = max(min(blocks[k], v_end) - v_begin, 0);
    tail = n_entries > 0 && v_end * kKeyTile > k_len;
  }
};

// Stores a tile's rows of a finished unit, or their part of a split launch, and hands the sum's tensor memory back.
template <typename T, int D, bool kExact>
__device__ __forceinline__ void store_unit(const tra_packed_launch& p, FwdCtl* ctl, int slot, int k, uint32_t t_o, bool any, float m, float l,
                                        float l_exact) {
  const FwdWork& w = ctl->work[slot];
  const int r = threadIdx.x & (kTileM - 1);
  const int tok = w.unit.index * 2 * p.tile_tokens + k * p.tile_tokens + r / p.group;     // inside the sequence
  const bool row_valid = r < p.tile_tokens * p.group && tok < w.unit.q.len;
  const long long tok_g = w.unit.q.begin + (row_valid ? tok : 0);
  const int head = w.kvh * p.group + r % p.group;
  const long long row_g = tok_g * p.heads + head;
  const float inv_l = l > 0.f ? 1.f / l : 0.f;
  const bool seen = any && l != 0.f;
  const bool parts = p.splits > 1;
  const long long part_row = (long long)w.split * p.total_q * p.heads + row_g;
  const RowAddresses rows(!row_valid ? nullptr
                          : parts ? (void*)(p.part_o + part_row * D)
                                  : (void*)((T*)p.o + tok_g * p.o_stride[0] + head * p.o_stride[1]));
  const RowAddresses rests(kExact && p.o_rest && row_valid && !parts ? (void*)((T*)p.o_rest + row_g * D) : nullptr);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t o[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) o[j] = 0u;
    if (any) {
      tmem_ld32(t_o + c * 32, o);
      tmem_wait_ld(o);
      if (c == D / 32 - 1) {                                  // the next unit's products may overwrite the sum
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&ctl->o_free[k]));
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) o[j] = seen ? __float_as_uint(__uint_as_float(o[j]) * inv_l) : 0u;
    if (parts) {
      rows.store64(o, c * 128);
      rows.store64(o + 16, c * 128 + 64);
    } else {
      uint32_t y[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float a = __uint_as_float(o[2 * j]), b = __uint_as_float(o[2 * j + 1]);
        y[j] = pack_pair<T>(a, b);
        if (kExact) o[j] = rest_pair<T>(a, b, y[j]);
      }
      rows.store64(y, c * 64);
      if (kExact && p.o_rest) rests.store64(o, c * 64);
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
  __syncwarp();
}

// Blocks that stay, one per SM: while the softmax warps finish a unit, the loads and the first scores of the next one are under
// way already (a block per unit spent about 10 us on set-up, first loads and epilogue: as much as five key blocks).
template <typename T, int D, bool kCausal, bool kExact>
__global__ void __launch_bounds__(kFwdThreads, 1) tra_packed_fwd_kernel(const __grid_constant__ tra_packed_launch p) {
  using C = FwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];         // the swizzled tiles start on 1024-byte boundaries
  uint8_t* sQ = smem;
  uint8_t* sKV = smem + 2 * C::kTileBytes;
  FwdCtl* ctl = (FwdCtl*)(smem + C::kSmemData);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const int box_rows = p.tile_tokens * p.group;
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp == 9) {
    tmem_alloc<512>(&ctl->tmem_base);
  } else if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctl->work_full[i]), 1);
      mbar_init(smem_u32(&ctl->work_free[i]), 11);       // producer, MMA, tail and eight softmax warps
      mbar_init(smem_u32(&ctl->s_full[i]), 1);
      mbar_init(smem_u32(&ctl->p_ready[i][0]), 4);
      mbar_init(smem_u32(&ctl->p_ready[i][1]), 4);
      mbar_init(smem_u32(&ctl->o_full[i]), 1);
      mbar_init(smem_u32(&ctl->o_free[i]), 4);
      mbar_init(smem_u32(&ctl->tail_full[i]), 1);
      mbar_init(smem_u32(&ctl->tail_ready[i]), 1);
    }
    mbar_init(smem_u32(&ctl->launch_full), 1);
    mbar_init(smem_u32(&ctl->want), 1);
    mbar_init(smem_u32(&ctl->q_full), 1);
    mbar_init(smem_u32(&ctl->q_free), 1);
    for (int i = 0; i < 6; ++i) mbar_init(smem_u32(&ctl->kv_full[i]), 1);
    for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&ctl->kv_release[i]), 1);
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (tid == 32) {
    prefetch_map(&p.map_q);
    prefetch_map(&p.map_k);
    prefetch_map(&p.map_v);
  }
  // rows of the query tiles that no box fills (group does not divide 128): zeros, so that they stay harmless
  if (box_rows < kTileM && warp >= 2 && warp < 8) zero_tile_rows(sQ, box_rows, kTileM, 2 * C::kAtoms, C::kAtomBytes, tid - 64, 192);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (p.splits > 1) allow_next_launch();                  // the join of the parts
  const uint32_t tmem = ctl->tmem_base;

  // the n-th unit of this block, for one warp; false: none left (or a wait ran out)
  auto next_work = [&](int n) -> bool {
    if (!mbar_wait_warp(smem_u32(&ctl->work_full[n & 1]), (uint32_t)(n >> 1) & 1u, abort_flag, p.status)) return false;
    return *(volatile int*)&ctl->work[n & 1].unit.seq >= 0;
  };
  auto done_with_work = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ctl->work_free[n & 1]));
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFwdRegsControl));
    if (warp == 11) {
      // ================================================================== scheduler
      // The grid has a block per unit, in launch order: a sequence's last tiles come first, which are the longest of a causal
      // one.  A running block takes over blocks that have not been started yet, one at a time (cluster launch control), and so balances units of different lengths without a counter in memory.
      // The request is made when the producer is about to run out of loads: units taken over early are units that an idle block
      // cannot have.
      int n = 0, unit = blockIdx.x;
      uint32_t asked = 0;
      bool alive = true, more = true;
      while (alive && more) {
        const int j = unit / p.splits;
        FwdWork w;
        w.split = unit - j * p.splits;
        w.kvh = j / p.n_units;
        w.unit = tra_find_unit(p, false, p.max_q <= 2 * p.tile_tokens, 2 * p.tile_tokens, j - w.kvh * p.n_units);
        w.unit.index = w.unit.count - 1 - w.unit.index;
        if (w.unit.seq >= 0) {                                // there is something to do
          if (n >= 2) alive = mbar_wait_warp(smem_u32(&ctl->work_free[n & 1]), (uint32_t)((n >> 1) - 1) & 1u, abort_flag, p.status);
          if (!alive) break;
          if (lane == 0) {
            ctl->work[n & 1] = w;
            mbar_arrive(smem_u32(&ctl->work_full[n & 1]));
          }
          __syncwarp();
          if (!(alive = mbar_wait_warp(smem_u32(&ctl->want), (uint32_t)n & 1u, abort_flag, p.status))) break;
          ++n;
        }
        if (lane == 0) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the last answer has been read
          mbar_expect_tx(smem_u32(&ctl->launch_full), 16);
          ask_for_launch(smem_u32(&ctl->launch), smem_u32(&ctl->launch_full));
        }
        __syncwarp();
        alive = mbar_wait_warp(smem_u32(&ctl->launch_full), asked & 1u, abort_flag, p.status);
        ++asked;
        more = alive && launch_answer(smem_u32(&ctl->launch), unit);
        __syncwarp();
      }
      if (alive && n >= 2) alive = mbar_wait_warp(smem_u32(&ctl->work_free[n & 1]), (uint32_t)((n >> 1) - 1) & 1u, abort_flag, p.status);
      if (alive && lane == 0) {
        ctl->work[n & 1].unit.seq = -1;
        mbar_arrive(smem_u32(&ctl->work_full[n & 1]));
      }
      __syncwarp();
    } else if (warp == 8) {
      // ================================================================== TMA producer
      int slot = 0, n_load = 0, event0 = 0, units = 0, tails = 0;
      bool alive = true;
      for (int n = 0; alive && next_work(n); ++n) {
        const FwdWork w = ctl->work[n & 1];
        done_with_work(n);
        const FwdPlan<kCausal> u(w, p);
        if (u.n_entries <= kAskAhead && lane == 0) mbar_arrive(smem_u32(&ctl->want));
        if (u.n_entries == 0) continue;
        if (lane == 0) {
          if (units > 0) alive = mbar_wait(smem_u32(&ctl->q_free), (uint32_t)(units - 1) & 1u, abort_flag, p.status);
          if (alive) {
            const uint32_t qbar = smem_u32(&ctl->q_full);
            mbar_expect_tx(qbar, 2 * C::kAtoms * box_rows * 128);
            for (int k = 0; k < 2; ++k)              // a missing tile loads rows nobody uses (past the tensor: zeros)
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sQ + k * C::kTileBytes + a * C::kAtomBytes), &p.map_q, qbar, a * 64, w.kvh * p.group,
                            w.unit.q.begin + u.tok0 + k * p.tile_tokens);
          }
          // Loads K0, V0, K1, V1, ... into consecutive slots.  The MMA warp hands slots back in release events, n_entries + 1
          // per unit: the first frees K0, event e + 1 frees V_e and K_(e+1).  Event r arrives on kv_release[r % 8].
          for (int e = 0; e < u.n_entries && alive; ++e) {
            if (e + kAskAhead + 1 == u.n_entries) mbar_arrive(smem_u32(&ctl->want));
            for (int kv = 0; kv < 2; ++kv) {
              if (n_load >= C::kSlots) {
                const int r = ctl->freed_by[slot];
                if (!(alive = mbar_wait(smem_u32(&ctl->kv_release[r & 7]), (uint32_t)(r >> 3) & 1u, abort_flag, p.status))) break;
              } else {
                ++n_load;
              }
              ctl->freed_by[slot] = event0 + e + kv;
              uint32_t bar = smem_u32(&ctl->kv_full[slot]);
              if (kv == 1 && u.tail && e == u.n_entries - 1) {
                // rows of it are zeroed first: it is announced by tail_ready, and the slot's barrier only keeps its count
                mbar_arrive(bar);
                ctl->tail_slot[tails & 1] = slot;
                bar = smem_u32(&ctl->tail_full[tails & 1]);
              }
              mbar_expect_tx(bar, C::kTileBytes);
              for (int a = 0; a < C::kAtoms; ++a)
                tma_load_3d(smem_u32(sKV + slot * C::kTileBytes + a * C::kAtomBytes), kv == 0 ? &p.map_k : &p.map_v, bar,
                            a * 64, w.kvh, w.unit.k.begin + (u.v_begin + e) * kKeyTile);
              if (++slot == C::kSlots) slot = 0;
            }
          }
        }
        event0 += u.n_entries + 1;
        ++units;
        tails += u.tail;
        alive = __all_sync(0xffffffffu, alive);
      }
    } else if (warp == 10) {
      // ================================================================== rows past the sequence's end
      int tails = 0;
      for (int n = 0; next_work(n); ++n) {
        const FwdWork w = ctl->work[n & 1];
        done_with_work(n);
        const FwdPlan<kCausal> u(w, p);
        if (!u.tail) continue;
        if (!mbar_wait_warp(smem_u32(&ctl->tail_full[tails & 1]), (uint32_t)(tails >> 1) & 1u, abort_flag, p.status)) break;
        const int slot = *(volatile int*)&ctl->tail_slot[tails & 1];
        zero_tile_rows(sKV + slot * C::kTileBytes, w.unit.k.len - (u.v_begin + u.n_entries - 1) * kKeyTile, kKeyTile, C::kAtoms,
                       C::kAtomBytes, lane, 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tail_ready[tails & 1]));
        ++tails;
      }
    } else if (warp == 9) {
      // ================================================================== MMA issuer
      // Waits end in a vote and values from shared memory in a reduction, so that descriptors stay in uniform registers (four
      // sequences of 4,096 tokens: causal, 40 / 8 heads, d 128 0.750 -> 0.675 ms; 16 heads, d 64 0.389 -> 0.373, causal 0.273 -> 0.250).
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_flag, p.status); };
      const uint32_t tmem = uniform(ctl->tmem_base);
      constexpr uint32_t kIdescQK = make_idesc_t<T>(kKeyTile, false);
      constexpr uint32_t kIdescPV = make_idesc_t<T>(D, true);
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
          if (!wait(smem_u32(&ctl->p_ready[k][half]), parity)) return false;
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
      uint32_t event = 0, units = 0, tails = 0;
      uint32_t entries[2] = {0u, 0u};        // key blocks of a tile so far
      uint32_t sums[2] = {0u, 0u};           // units in which the tile had any
      bool alive = true;
      for (int n = 0; alive && uniform(next_work(n)); ++n) {
        const FwdWork w = ctl->work[n & 1];
        done_with_work(n);
        FwdPlan<kCausal> u(w, p);
        u.n_entries = uniform(u.n_entries);
        u.n_own[0] = uniform(u.n_own[0]);
        u.n_own[1] = uniform(u.n_own[1]);
        u.tail = uniform(u.tail);
        if (u.n_entries == 0) continue;
        alive = wait(smem_u32(&ctl->q_full), units & 1u) &&
                wait(smem_u32(&ctl->kv_full[slot]), phase);       // first K tile
        if (!alive) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (u.n_own[k] > 0) issue_s(k, slot);
        tc_commit(smem_u32(&ctl->kv_release[event++ & 7u]));
        if (u.n_entries == 1) tc_commit(smem_u32(&ctl->q_free));
        advance();
        for (int e = 0; e < u.n_entries; ++e) {
          const int vslot = slot;
          const bool have_next = e + 1 < u.n_entries;
          alive = wait(smem_u32(&ctl->kv_full[vslot]), phase);
          if (alive && u.tail && !have_next) {
            alive = wait(smem_u32(&ctl->tail_ready[tails & 1]), (tails >> 1) & 1u);
            ++tails;
          }
          advance();
          bool k_ready = false;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (!alive || e >= u.n_own[k]) continue;
            if (e == 0) {
              // the sum of the tile's last unit has been read
              if (sums[k] > 0 && !(alive = wait(smem_u32(&ctl->o_free[k]), (sums[k] - 1) & 1u))) continue;
              ++sums[k];
            }
            if (!(alive = issue_pv(k, vslot, entries[k] & 1u, e > 0 ? 1u : 0u))) continue;
            ++entries[k];
            if (e + 1 == u.n_own[k]) {
              tc_commit(smem_u32(&ctl->o_full[k]));
            } else {
              if (!k_ready) {
                alive = wait(smem_u32(&ctl->kv_full[slot]), phase);
                k_ready = true;
                if (!alive) continue;
                tc_fence_after();
              }
              issue_s(k, slot);
            }
          }
          if (!alive) break;
          tc_commit(smem_u32(&ctl->kv_release[event++ & 7u]));       // V of this block and K of the next
          if (e + 2 == u.n_entries) tc_commit(smem_u32(&ctl->q_free));
          if (have_next) advance();
        }
        ++units;
      }
      // every MMA has retired before tensor memory is released
      tc_commit(smem_u32(&ctl->drain));
      wait(smem_u32(&ctl->drain), 0u);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFwdRegsSoftmax));
    // ================================================================== softmax + epilogue
    const int k = warp >> 2;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_o = tmem + lane_base + 256 + k * 128, t_s = tmem + lane_base + k * 128;
    uint32_t entries = 0, sums = 0;          // key blocks, and units that had any, of this tile so far
    bool alive = true;
    for (int it = 0; alive && next_work(it); ++it) {
      float m = -INFINITY, l = 0.f, l_exact = 0.f;
      int n, col_limit;
      bool rows_here;
      {
        const FwdWork w = ctl->work[it & 1];
        const FwdPlan<kCausal> u(w, p);
        n = u.n_own[k];
        const int tile_tok = u.tok0 + k * p.tile_tokens;
        // (opaque to the compiler: what follows from the thread index alone would be kept in registers through all units)
        int r = tid & (kTileM - 1);
        asm volatile("" : "+r"(r));
        const int first_row = r & ~31;
        rows_here = first_row < p.tile_tokens * p.group && tile_tok + first_row / p.group < w.unit.q.len;
        // columns of the first block that the row sees; rows that hold no query follow the tile's last one, so that they
        // force no mask on their warp
        const int mask_tok = min(tile_tok + r / p.group, min(tile_tok + p.tile_tokens, w.unit.q.len) - 1);
        col_limit = (kCausal ? min(max(mask_tok + 1 + w.unit.k.len - w.unit.q.len, 0), w.unit.k.len) : w.unit.k.len) - u.v_begin * kKeyTile;
      }
      if (!rows_here) {
        // a warp without a row keeps up with the barriers; what its lanes multiply stays in its own, unstored rows
        for (int e = 0; e < n && alive; ++e) {
          alive = mbar_wait_warp(smem_u32(&ctl->s_full[k]), entries & 1u, abort_flag, p.status);
          ++entries;
          if (alive && lane == 0) {
            mbar_arrive(smem_u32(&ctl->p_ready[k][0]));
            mbar_arrive(smem_u32(&ctl->p_ready[k][1]));
          }
          __syncwarp();
        }
      } else {
        const float scale_log2 = p.sm_scale * kLog2e;
        for (int e = 0; e < n; ++e, col_limit -= kKeyTile) {
          if (!mbar_wait_warp(smem_u32(&ctl->s_full[k]), entries & 1u, abort_flag, p.status)) {
            alive = false;
            break;
          }
          ++entries;
          tc_fence_after();
          uint32_t sb[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &sb[c * 32]);
          tmem_wait_ld(&sb[0]);
#pragma unroll
          for (int c = 1; c < 4; ++c) reg_fence32(&sb[c * 32]);
          if (__any_sync(0xffffffffu, col_limit < kKeyTile)) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (!__any_sync(0xffffffffu, col_limit < (c + 1) * 32)) continue;      // all rows of the warp see these 32 keys
#pragma unroll
              for (int j = c * 32; j < c * 32 + 32; ++j)
                if (j >= col_limit) sb[j] = 0xff800000u;                  // -inf
            }
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

      // ---- epilogue ------------------------------------------------------------------------
      if (alive && n > 0) {
        alive = mbar_wait_warp(smem_u32(&ctl->o_full[k]), sums & 1u, abort_flag, p.status);
        ++sums;
        tc_fence_after();
      }
      if (!alive) break;
      store_unit<T, D, kExact>(p, ctl, it & 1, k, t_o, n > 0, m, l, l_exact);
      done_with_work(it);
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
    tmem_free<512>(tmem);
  }
}

template <typename T, int D, bool kCausal, bool kExact>
int launch_fwd(const tra_packed_ctx& c, const tra_packed_launch& a) {
  constexpr auto kern = tra_packed_fwd_kernel<T, D, kCausal, kExact>;
  const int rc = tra_allow_smem<kern>(FwdCfg<D>::kSmemBytes);
  if (rc != TRA_OK) return rc;
  const long long units = (long long)a.n_units * a.kv_heads * a.splits;
  if (units > 0x3fffffffll) return TRA_ERR_UNSUPPORTED;
  return tra_launch(kern, dim3((unsigned)units), kFwdThreads, FwdCfg<D>::kSmemBytes, c.stream, false,
                    1, a);
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
