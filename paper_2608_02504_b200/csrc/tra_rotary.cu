// What a layer does to Q, K and V between its projections and its attention, in one pass: a norm over the
// channels of every head (RMS or layer norm, optional), rotary positions with several axes, and the token
// order the attention calls want; and the gradients of all of it.
//
// One row = one (token, head), d channels.  n = x, x r or (x - mean) r with r = (mean square + eps)^-1/2;
// z = weight n + bias; the channel pair (z1, z2) of pair p turns by the angle pos[axis_p] * f_p:
//   y = (z1 cos - z2 sin, z1 sin + z2 cos).
// Gradients: u = the pair of dy turned back, dweight = sum u n, dbias = sum u, g = weight u,
//   dx = r (g - n mean(g n))            RMS norm
//   dx = r (g - mean g - n mean(g n))   layer norm.
//
// Angles.  F_p = f_p / 2 pi modulo one turn, as a 64-bit binary fraction (rounded once, on the host, from an integer
// product with 192 bits of 1 / 2 pi).  pos * F_p modulo 2^64 is then the angle in turns with its whole turns already gone, whatever the
// position: an integer product in place of a range reduction, off by pos * 2^-65 turns.  Its high word (2^-32 turns
// at most are cut), as a signed number of half turns rounded to fp32 (2^-25 half turns), goes to sincospif.
//
// Bound: HBM.  Every element is read once and written once (the norm's backward pass reads x too); a row stays
// in the registers of d / 16 neighbouring threads, 16 channels each (a 16-byte piece of either half of the row
// for 16-bit types, so that both ways of pairing channels find their partner in the same thread and a row is
// read in whole 128-byte lines), and its sums are shuffles among those threads.  The cosines and sines of a block's
// tokens are computed once, into shared memory, and used for all heads.  The weights' gradients stay in
// registers over a thread's rows, are added up per thread block in a fixed order, and a second small kernel
// adds the blocks: no atomics, the same bits every time.  75,600 tokens, 40 + 40 + 40 heads of 128, RMS norm, bf16: 750 us (6.2 TB/s, 95 %
// of the copy rate); its backward pass over 32,837 tokens, 12 + 12 + 12 heads: 148 us (5.5 TB/s).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include <new>

#include "tra_common.cuh"
#include "tra_tcgen05.cuh"

struct tra_rotary {
  int head_dim, n_axes, halves, norm;
  float eps;
  uint64_t turn[TRA_ROTARY_MAX_HEAD_DIM / 2];     // F_p
  uint8_t axis[TRA_ROTARY_MAX_HEAD_DIM / 2];
};

namespace {

constexpr int kThreads = 256;
constexpr int kMaxD = TRA_ROTARY_MAX_HEAD_DIM;
constexpr int kReduceRows = 32;       // block partials summed side by side in the second kernel
constexpr int kReduceCols = 8;

struct RotTensor {
  const void* src;       // forward: x; backward: dy
  void* dst;             // forward: y; backward: dx
  const void* x;         // backward with a norm: the forward's input
  const void* weight;
  const void* bias;
  float* partial;        // backward: [2][blocks][d] of this tensor, or NULL
  long long src_stride[3], dst_stride[3], x_stride[3];      // batch, token, head (elements)
  int heads, rotate, tile_major;
};

struct RotArgs {
  RotTensor t[3];
  uint64_t turn[kMaxD / 2];
  uint8_t axis[kMaxD / 2];
  const int32_t* raster_of_pos;   // plan, or NULL
  const int32_t* pos;             // explicit positions [tokens][n_axes], or NULL
  int n_axes, H, W, n_video;      // grid positions: token n -> (n / (H W), n / W % H, n % W)
  int d, lanes;                   // lanes: threads per row, d / 16 rounded up to a power of two
  int n_tensors, one_tensor;      // one_tensor: a block works on the tensor blockIdx.y, else on all of them
  int by_source;                  // !one_tensor: the rotated tensors are tile-major
  int head_slots, head_slots_log2, lanes_log2;   // heads of a token side by side in a block; both powers of two
  float eps, inv_d;
  int rows, tokens;               // rows = batch * tokens
};

// A thread's sixteen channels as loaded: eight of the lower half of the row, eight of the upper half.
template <typename T>
struct Raw {
  static constexpr int kVec = sizeof(T) / 2;         // 16-byte loads per eight channels
  uint4 v[2 * kVec];
  __device__ __forceinline__ void load(const T* lo, const T* hi) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      v[i] = reinterpret_cast<const uint4*>(lo)[i];
      v[kVec + i] = reinterpret_cast<const uint4*>(hi)[i];
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 2 * kVec; ++i) v[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void store(T* lo, T* hi) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      reinterpret_cast<uint4*>(lo)[i] = v[i];
      reinterpret_cast<uint4*>(hi)[i] = v[kVec + i];
    }
  }
};

// Rows on their way.  One row ahead waits in registers, except in the norm's backward pass of the 16-bit types, whose registers
// are taken: there every thread copies its own pieces into shared memory, [stage][piece][thread] 16 bytes each, kStages - 1
// rows ahead, and reads nothing but them, so that waiting for its own copies is all the synchronisation there is.  (Measured on the
// 32.7K-token shape: RMS backward 208 us with registers, 180 with the ring; fp32 308 and 397; forward 110 and 114.)
__device__ __forceinline__ void copy16(uint4* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

template <typename T, int kNorm, bool kBackward>
struct RotShape {
  static constexpr bool kSums = kBackward && kNorm != TRA_NORM_NONE;
  static constexpr bool kRing = kSums && sizeof(T) == 2;
  static constexpr int kPieces = 4 * Raw<T>::kVec;              // of dy, and of x
  static constexpr int kStages = kRing ? 4 : 2;                 // 2: one row ahead, in registers
  // As many as need no (or few) spills.  16-bit forward, 75,600 tokens with 40 + 40 + 40 heads of 128: 4 blocks 750 us, 3 827,
  // 5 811.  fp32, 32,837 tokens with 12 + 12 + 12 heads of 128, 3 blocks against 4: forward 221 against 244 us, with
  // layer norm 213 against 226, backward without a norm 212 against 264.
  static constexpr int kBlocksPerSm = kSums ? 2 : sizeof(T) == 4 ? 3 : 4;
  static constexpr int kRingBytes = kRing ? kStages * kPieces * kThreads * 16 : 0;
};

// two neighbouring channels of a 16-bit type
template <typename T>
__device__ __forceinline__ void split(uint32_t w, float& a, float& b);
template <>
__device__ __forceinline__ void split<__nv_bfloat16>(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
template <>
__device__ __forceinline__ void split<__half>(uint32_t w, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  a = f.x;
  b = f.y;
}
template <typename T>
__device__ __forceinline__ uint32_t join(float a, float b);
template <>
__device__ __forceinline__ uint32_t join<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t join<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The sixteen channels as eight fp32 pairs for the packed arithmetic: z[0 .. 3] the first channels of the rotation's pairs
// 0 .. 7 of the thread, z[4 .. 7] their second channels.
template <typename T, bool kHalves>
__device__ __forceinline__ void unpack(const Raw<T>& r, uint64_t* z) {
  if constexpr (sizeof(T) == 4) {
    const float* f = reinterpret_cast<const float*>(r.v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = 2 * (i & 3), second = i >> 2;
      z[i] = kHalves ? pack2(f[8 * second + j], f[8 * second + j + 1]) : pack2(f[2 * j + second], f[2 * j + 2 + second]);
    }
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(r.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b, c, d;
      split<T>(w[2 * i], a, b);
      split<T>(w[2 * i + 1], c, d);
      if (kHalves) {                                   // words 0 .. 3 first channels, 4 .. 7 second ones
        z[2 * i] = pack2(a, b);
        z[2 * i + 1] = pack2(c, d);
      } else {                                         // every word holds a pair
        z[i] = pack2(a, c);
        z[4 + i] = pack2(b, d);
      }
    }
  }
}
template <typename T, bool kHalves>
__device__ __forceinline__ void pack(const uint64_t* z, Raw<T>& r) {
  if constexpr (sizeof(T) == 4) {
    float* f = reinterpret_cast<float*>(r.v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = 2 * (i & 3), second = i >> 2;
      unpack2(z[i], f[kHalves ? 8 * second + j : 2 * j + second], f[kHalves ? 8 * second + j + 1 : 2 * j + 2 + second]);
    }
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(r.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b, c, d;
      unpack2(z[kHalves ? 2 * i : i], a, b);
      unpack2(z[kHalves ? 2 * i + 1 : 4 + i], c, d);
      w[2 * i] = kHalves ? join<T>(a, b) : join<T>(a, c);
      w[2 * i + 1] = kHalves ? join<T>(c, d) : join<T>(b, d);
    }
  }
}

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t both(float x) { return pack2(x, x); }
__device__ __forceinline__ float sum2(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}

// Sum over the threads of a row (a power of two of neighbouring lanes).
__device__ __forceinline__ float row_sum(float s, int lanes) {
  if (lanes == 8) {                                  // 128 channels
    s += __shfl_xor_sync(0xffffffffu, s, 4);
    s += __shfl_xor_sync(0xffffffffu, s, 2);
    return s + __shfl_xor_sync(0xffffffffu, s, 1);
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ float sum_of(const uint64_t* z) {
  return sum2(fadd2(fadd2(fadd2(z[0], z[1]), fadd2(z[2], z[3])), fadd2(fadd2(z[4], z[5]), fadd2(z[6], z[7]))));
}
__device__ __forceinline__ float dot_of(const uint64_t* a, const uint64_t* b) {
  uint64_t s = fmul2(a[0], b[0]), t = fmul2(a[1], b[1]);
#pragma unroll
  for (int i = 2; i < 8; i += 2) {
    s = ffma2(a[i], b[i], s);
    t = ffma2(a[i + 1], b[i + 1], t);
  }
  return sum2(fadd2(s, t));
}

// Four floats per lane and step q, the lanes' side by side: conflict-free 16-byte reads.
__device__ __forceinline__ void load_pairs(const float* table, int q, int lanes, int lane, uint64_t& a, uint64_t& b) {
  const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(table + (q * lanes + lane) * 4);
  a = v.x;
  b = v.y;
}
// turns the pairs by their angle, or back
template <bool kBack>
__device__ __forceinline__ void turn_pairs(uint64_t* z, const float* cs, const float* sn, int lanes, int lane) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint64_t c[2], s[2];
    load_pairs(cs, q, lanes, lane, c[0], c[1]);
    load_pairs(sn, q, lanes, lane, s[0], s[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint64_t& a = z[2 * q + i];
      uint64_t& b = z[4 + 2 * q + i];
      const uint64_t minus = s[i] ^ 0x8000000080000000ull;
      const uint64_t ta = ffma2(a, c[i], fmul2(b, kBack ? s[i] : minus));
      const uint64_t tb = ffma2(b, c[i], fmul2(a, kBack ? minus : s[i]));
      a = ta;
      b = tb;
    }
  }
}

__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

// Channel of entry i (0 .. 15) of a lane's z, and pair of entry j (0 .. 7).
template <bool kHalves>
__device__ __forceinline__ int channel_of(int d, int lane, int i) {
  if (kHalves) return (i < 8 ? 0 : d / 2 - 8) + lane * 8 + i;
  const int j = i & 7;
  return (j < 4 ? 0 : d / 2 - 8) + lane * 8 + 2 * j + (i >> 3);
}
template <bool kHalves>
__device__ __forceinline__ int pair_of(int d, int lane, int j) {
  return kHalves ? lane * 8 + j : (j < 4 ? 0 : d / 4 - 4) + lane * 4 + j;
}

// The token a thread works on: its index in the batch entry on the attention side (ordered) and on the projection side.
struct Token {
  int batch, ordered, source;
  bool there;
};

// A block takes groups of tokens_per_block tokens: the same number of threads for every token, each walking every
// head_slots-th head of the block's tensors (all of them one after the other, or the one blockIdx.y names).  Loads run ahead
// of the arithmetic, across heads, tensors and groups; the angles of the next group go to the other half of s_turn
// behind the current group's rows, so that a group costs one barrier and no exposed load.
template <typename T, int kNorm, bool kHalves, bool kBackward>
__global__ void __launch_bounds__(kThreads, RotShape<T, kNorm, kBackward>::kBlocksPerSm)
tra_rotary_kernel(const __grid_constant__ RotArgs p) {
  using Shape = RotShape<T, kNorm, kBackward>;
  constexpr bool kSums = Shape::kSums;
  constexpr int kStages = Shape::kStages, kVec = Raw<T>::kVec;
  extern __shared__ __align__(16) uint8_t smem[];
  uint4* const ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;       // [stage][piece] kThreads apart
  // per lane four floats and step, see load_pairs: [buffer][cosines, then sines][token of the group], 8 per lane
  float* const s_turn = reinterpret_cast<float*>(smem + Shape::kRingBytes);
  __shared__ __align__(16) float s_weight[kNorm != TRA_NORM_NONE ? 3 * kMaxD : 4], s_bias[kNorm == TRA_NORM_LAYER ? 3 * kMaxD : 4];
  __shared__ uint64_t s_freq[kMaxD / 2];
  __shared__ uint8_t s_axis[kMaxD / 2];
  const int tid = threadIdx.x, lanes = p.lanes;
  const int lane = tid & (lanes - 1), slot = tid >> p.lanes_log2;
  const bool on = lane * 16 < p.d;                     // d / 16 need not be a power of two
  const int c_lo = lane * 8, c_hi = p.d / 2 + lane * 8;
  const int head0 = slot & (p.head_slots - 1), token_slot = slot >> p.head_slots_log2;
  const int tokens_per_block = kThreads >> (p.lanes_log2 + p.head_slots_log2);
  const int sines = tokens_per_block * lanes * 8;
  const int t_first = p.one_tensor ? (int)blockIdx.y : 0, t_end = p.one_tensor ? t_first + 1 : p.n_tensors;
  const bool by_source = p.one_tensor ? p.t[t_first].tile_major != 0 : p.by_source != 0;
  const bool turns_any = !p.one_tensor || p.t[t_first].rotate;

  for (int i = tid; i < p.d / 2; i += kThreads) {
    s_freq[i] = p.turn[i];
    s_axis[i] = p.axis[i];
  }
  if (kNorm != TRA_NORM_NONE) {
    for (int i = tid; i < 16 * lanes; i += kThreads) {
      const int l = (i >> 2) & (lanes - 1), e = (i >> (2 + p.lanes_log2)) * 4 + (i & 3);
      const int c = channel_of<kHalves>(p.d, l, e);
      for (int k = t_first; k < t_end; ++k) {
        const RotTensor& t = p.t[k];
        const bool has = l * 16 < p.d;
        s_weight[k * kMaxD + i] = has && t.weight ? to_float(((const T*)t.weight)[c]) : 1.f;
        if (kNorm == TRA_NORM_LAYER) s_bias[k * kMaxD + i] = has && !kBackward && t.bias ? to_float(((const T*)t.bias)[c]) : 0.f;
      }
    }
  }
  uint64_t acc_w[kSums ? 8 : 1], acc_b[kSums && kNorm == TRA_NORM_LAYER ? 8 : 1];
  if (kSums) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      acc_w[i] = 0ull;
      if (kNorm == TRA_NORM_LAYER) acc_b[i] = 0ull;
    }
  }

  auto locate = [&](int base) -> Token {
    Token k = {0, 0, 0, base < p.rows && base + token_slot < p.rows};
    if (k.there) {
      k.ordered = base + token_slot;
      if (p.tokens != p.rows) {
        k.batch = k.ordered / p.tokens;
        k.ordered -= k.batch * p.tokens;
      }
      // tensors that are not tile-major ignore the source index
      k.source = p.raster_of_pos != nullptr && k.ordered < p.n_video ? __ldg(p.raster_of_pos + k.ordered) : k.ordered;
    }
    return k;
  };
  // cosines and sines of a token, shared out over its threads
  auto angles = [&](const Token& k, float* turn) {
    if (!turns_any) return;
    // positions belong to the projection side, which is the ordered index of a tensor that is not tile-major
    const int tok = by_source ? k.source : k.ordered;
    int frame = 0, y = 0, x = 0;
    if (p.pos == nullptr) {
      const int hw = p.H * p.W;
      frame = tok / hw;
      const int in_frame = tok - frame * hw;
      y = in_frame / p.W;
      x = in_frame - y * p.W;
    }
    // text keeps its channels; a token that does not exist turns its zeros by nothing
    const bool turned = k.there && (p.pos != nullptr || tok < p.n_video);
    float* const out = turn + token_slot * lanes * 8;
    for (int e = (head0 << p.lanes_log2) + lane; e < lanes * 8; e += lanes << p.head_slots_log2) {
      const int l = (e >> 2) & (lanes - 1), pair = pair_of<kHalves>(p.d, l, (e >> (2 + p.lanes_log2)) * 4 + (e & 3));
      float c = 1.f, sine = 0.f;
      if (turned && l * 16 < p.d) {
        const int axis = s_axis[pair];
        const int v = p.pos != nullptr ? __ldg(p.pos + (long long)tok * p.n_axes + axis) : axis == 0 ? frame : axis == 1 ? y : x;
        const uint64_t turns = (uint64_t)(int64_t)v * s_freq[pair];
        sincospif((float)(int32_t)(turns >> 32) * 4.656612873077393e-10f /* 2^-31 */, &sine, &c);
      }
      out[e] = c;
      out[sines + e] = sine;
    }
  };

  const int stride = (int)gridDim.x * tokens_per_block;
  int base = (int)blockIdx.x * tokens_per_block;
  Token cur = locate(base);

  // Ring: the row that is requested next, its token (and the one after it), tensor, head and addresses.
  Token ask = cur, ask_next = cur;
  int ask_base = base, ask_t = t_first, ask_h = head0, ask_stage = 0;
  // otherwise: the row ahead
  Raw<T> raw, xraw;
  bool in_on = false;
  const T *in = nullptr, *xin = nullptr;                 // both: its address, at the thread's lower channels
  auto aim = [&](const Token& k, int ti) {               // a token's first row of a tensor
    const RotTensor& t = p.t[ti];
    // forward reads at the source row and writes at the ordered one, backward the other way round
    const int source = t.tile_major ? k.source : k.ordered;
    in = (const T*)t.src + k.batch * t.src_stride[0] + (kBackward ? k.ordered : source) * t.src_stride[1] + head0 * t.src_stride[2] + c_lo;
    if (kSums && t.rotate) xin = (const T*)t.x + k.batch * t.x_stride[0] + source * t.x_stride[1] + head0 * t.x_stride[2] + c_lo;
  };
  auto request = [&]() {                                 // ring
    if (ask_base < p.rows) {
      const RotTensor& t = p.t[ask_t];
      uint4* dst = ring + ask_stage * Shape::kPieces * kThreads;
      const bool with_x = t.rotate != 0;
      if (ask.there && on && ask_h < t.heads) {
        copy16(dst, in);
        copy16(dst + kThreads, in + p.d / 2);
        if (with_x) {
          copy16(dst + 2 * kThreads, xin);
          copy16(dst + 3 * kThreads, xin + p.d / 2);
        }
      } else {                                           // a row that is not there is zeros
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i * kThreads] = make_uint4(0u, 0u, 0u, 0u);
      }
      ask_h += p.head_slots;
      if (ask_h - head0 < t.heads) {
        in += t.src_stride[2] << p.head_slots_log2;
        xin += t.x_stride[2] << p.head_slots_log2;
      } else {
        ask_h = head0;
        if (++ask_t == t_end) {
          ask_t = t_first;
          ask = ask_next;
          ask_base += stride;
          ask_next = locate(ask_base + stride);
        }
        aim(ask, ask_t);
      }
    }
    copy_commit();                                       // an empty group at the end keeps the count
    if (++ask_stage == kStages) ask_stage = 0;
  };
  auto load = [&](bool there, bool with_x) {             // no ring
    if (there) {
      raw.load(in, in + p.d / 2);
      if (kSums && with_x) xraw.load(xin, xin + p.d / 2);
    } else {
      raw.zero();
      if (kSums) xraw.zero();
    }
  };
  auto load_first = [&](const Token& k, int ti) {
    in_on = k.there && on;
    if (in_on) aim(k, ti);
    load(in_on && head0 < p.t[ti].heads, p.t[ti].rotate);
  };
  if constexpr (Shape::kRing) {
    ask_next = locate(base + stride);
    aim(ask, ask_t);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) request();
  } else {
    load_first(cur, t_first);
  }

  __syncthreads();
  angles(cur, s_turn);
  __syncthreads();
  int stage = 0;
  int buffer = 0;
  // All threads of a warp walk the same number of rows (row sums are warp-wide shuffles): a thread whose token or head
  // does not exist takes part with zeros.
  while (true) {
    const bool more = p.rows - base > stride;          // base + stride < rows
    const Token next = more ? locate(base + stride) : Token{0, 0, 0, false};
    const float* const cs = s_turn + buffer * 2 * sines + token_slot * lanes * 8;
    const float* const sn = cs + sines;
    for (int ti = t_first; ti < t_end; ++ti) {
      const RotTensor& t = p.t[ti];
      const int heads = t.heads, hs = p.head_slots;
      const bool rotate = t.rotate != 0;
      const long long out_step = t.dst_stride[2] << p.head_slots_log2;
      const bool out_on = cur.there && on;
      T* out = (T*)t.dst + cur.batch * t.dst_stride[0] +
               (kBackward && t.tile_major ? cur.source : cur.ordered) * t.dst_stride[1] + head0 * t.dst_stride[2];
      for (int h = head0; h - head0 < heads; h += hs, out += out_step) {
        const bool row_on = out_on && h < heads;
        Raw<T> row, xrow;
        if constexpr (Shape::kRing) {
          copy_wait<kStages - 2>();                    // this row's pieces are there
          const uint4* src = ring + stage * Shape::kPieces * kThreads;
#pragma unroll
          for (int i = 0; i < 2 * kVec; ++i) {
            row.v[i] = src[i * kThreads];
            xrow.v[i] = src[(2 * kVec + i) * kThreads];
          }
          if (++stage == kStages) stage = 0;
        } else {
          row = raw;
          if (kSums) xrow = xraw;
        }
        // the next row, while this one is worked on (ring: into the stage read one row ago)
        if constexpr (Shape::kRing) {
          request();
        } else if (h - head0 + hs < heads) {
          in += t.src_stride[2] << p.head_slots_log2;
          if (kSums) xin += t.x_stride[2] << p.head_slots_log2;
          load(in_on && h + hs < heads, rotate);
        } else if (ti + 1 < t_end) {
          load_first(cur, ti + 1);
        } else {
          load_first(next, t_first);
        }
        if (!rotate) {                                 // only moved
          if (row_on) row.store(out + c_lo, out + c_hi);
          continue;
        }
        uint64_t z[8];
        unpack<T, kHalves>(row, z);
        if (!kBackward) {
          if (kNorm != TRA_NORM_NONE) {
            if (kNorm == TRA_NORM_LAYER) {
              const float total = row_sum(sum_of(z), lanes);       // every lane shuffles
              const uint64_t mean = both(on ? -total * p.inv_d : 0.f);
#pragma unroll
              for (int i = 0; i < 8; ++i) z[i] = fadd2(z[i], mean);
            }
            const uint64_t r = both(rsqrtf(fmaf(row_sum(dot_of(z, z), lanes), p.inv_d, p.eps)));
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint64_t w[2], b[2] = {0ull, 0ull};
              load_pairs(s_weight + ti * kMaxD, q, lanes, lane, w[0], w[1]);
              if (kNorm == TRA_NORM_LAYER) load_pairs(s_bias + ti * kMaxD, q, lanes, lane, b[0], b[1]);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint64_t& v = z[2 * q + i];
                v = fmul2(v, r);
                v = kNorm == TRA_NORM_LAYER ? ffma2(v, w[i], b[i]) : fmul2(v, w[i]);
              }
            }
          }
          turn_pairs<false>(z, cs, sn, lanes, lane);
        } else {
          turn_pairs<true>(z, cs, sn, lanes, lane);    // z = u
          if constexpr (kSums) {
            uint64_t n[8];
            unpack<T, kHalves>(xrow, n);
            if (kNorm == TRA_NORM_LAYER) {
              const float total = row_sum(sum_of(n), lanes);
              const uint64_t mean = both(on ? -total * p.inv_d : 0.f);
#pragma unroll
              for (int i = 0; i < 8; ++i) n[i] = fadd2(n[i], mean);
            }
            // a row that does not exist is left out (eps = 0 would make 0 * inf of it)
            const float squares = row_sum(dot_of(n, n), lanes);
            const uint64_t r = both(row_on ? rsqrtf(fmaf(squares, p.inv_d, p.eps)) : 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              n[i] = fmul2(n[i], r);
              acc_w[i] = ffma2(z[i], n[i], acc_w[i]);
              if (kNorm == TRA_NORM_LAYER) acc_b[i] = fadd2(acc_b[i], z[i]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {              // z = g
              uint64_t w[2];
              load_pairs(s_weight + ti * kMaxD, q, lanes, lane, w[0], w[1]);
              z[2 * q] = fmul2(z[2 * q], w[0]);
              z[2 * q + 1] = fmul2(z[2 * q + 1], w[1]);
            }
            const uint64_t mgn = both(-row_sum(dot_of(z, n), lanes) * p.inv_d);
            const uint64_t mg = both(kNorm == TRA_NORM_LAYER ? -row_sum(sum_of(z), lanes) * p.inv_d : 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint64_t g = kNorm == TRA_NORM_LAYER ? fadd2(z[i], mg) : z[i];
              z[i] = fmul2(r, ffma2(n[i], mgn, g));
            }
          }
        }
        if (row_on) {
          Raw<T> y;
          pack<T, kHalves>(z, y);
          y.store(out + c_lo, out + c_hi);
        }
      }
    }
    if (!more) break;
    buffer ^= 1;
    angles(next, s_turn + buffer * 2 * sines);
    __syncthreads();
    base += stride;
    cur = next;
  }

  if constexpr (kSums) {
    const RotTensor& t = p.t[t_first];
    if (t.partial == nullptr) return;
    // threads of the same lane hold the same channels: add them over the warp, then over the block's warps in order
    float* s_red = reinterpret_cast<float*>(smem);     // [warp][d], d <= 256: the ring is empty now, or s_turn is done with
    const int warp = tid >> 5;
    __syncthreads();
#pragma unroll
    for (int which = 0; which < (kNorm == TRA_NORM_LAYER ? 2 : 1); ++which) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[2];
        unpack2(acc_w[i], v[0], v[1]);
        if constexpr (kNorm == TRA_NORM_LAYER)
          if (which == 1) unpack2(acc_b[i], v[0], v[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          for (int o = lanes; o < 32; o <<= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
          if ((tid & 31) < lanes && on) s_red[warp * p.d + channel_of<kHalves>(p.d, lane, 2 * i + k)] = v[k];
        }
      }
      __syncthreads();
      for (int c = tid; c < p.d; c += kThreads) {
        float v = 0.f;
        for (int k = 0; k < kThreads / 32; ++k) v += s_red[k * p.d + c];
        t.partial[((long long)which * gridDim.x + blockIdx.x) * p.d + c] = v;
      }
      __syncthreads();
    }
  }
}

struct ReduceArgs {
  const float* partial[6];
  float* out[6];
  int blocks, d;
};

// out[c] = sum over the blocks' partials, in a fixed order: 32 strided sums side by side, then those in order.
__global__ void __launch_bounds__(kReduceRows * kReduceCols) tra_rotary_reduce_kernel(const __grid_constant__ ReduceArgs p) {
  __shared__ float s[kReduceRows][kReduceCols];
  const int col = threadIdx.x % kReduceCols, r = threadIdx.x / kReduceCols;
  const int c = blockIdx.x * kReduceCols + col;
  float v = 0.f;
  if (c < p.d)
    for (int b = r; b < p.blocks; b += kReduceRows) v += p.partial[blockIdx.y][(long long)b * p.d + c];
  s[r][col] = v;
  __syncthreads();
  if (r == 0 && c < p.d) {
    for (int i = 1; i < kReduceRows; ++i) v += s[i][col];
    p.out[blockIdx.y][c] = v;
  }
}

int lanes_of(int d) {
  int l = 1;
  while (l * 16 < d) l *= 2;
  return l;
}

int log2_of(int n) {
  int l = 0;
  while ((1 << l) < n) ++l;
  return l;
}

constexpr int kBlocksMax = 4 * 148;

// f / 2 pi modulo one turn as a 64-bit binary fraction, |f| < 2^64.  f = m 2^e with a 53-bit m, so the fraction is m times
// floor(2^192 / 2 pi), shifted right by 128 - e >= 117 bits and rounded; the digits that the constant lacks weigh less than 2^-64 of its
// last bit.
uint64_t turn_of(double f) {
  constexpr uint64_t kInvTwoPi[3] = {0x36d8a5664f10e410ull, 0x7f09d5f47d4d3770ull, 0x28be60db9391054aull};
  int exponent = 0;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(f), &exponent), 53);
  const int shift = 128 + 53 - exponent;
  if (m == 0 || shift >= 245) return 0;                // the product is below 2^243: rounds to 0
  uint64_t w[5] = {0, 0, 0, 0, 0};
  unsigned __int128 carry = 0;
  for (int i = 0; i < 3; ++i) {
    carry += (unsigned __int128)m * kInvTwoPi[i];
    w[i] = (uint64_t)carry;
    carry >>= 64;
  }
  w[3] = (uint64_t)carry;
  const int half = shift - 1;                          // rounding: half of the last bit kept
  carry = 1ull << (half & 63);
  for (int i = half >> 6; i < 4; ++i) {
    carry += w[i];
    w[i] = (uint64_t)carry;
    carry >>= 64;
  }
  const int word = shift >> 6, bit = shift & 63;
  const uint64_t turns = bit ? w[word] >> bit | w[word + 1] << (64 - bit) : w[word];
  return f < 0 ? 0 - turns : turns;
}

int elem_bytes(int dtype) { return dtype == TRA_FP32 ? 4 : 2; }

bool aligned_strides(const int64_t* s, int dtype) {
  for (int i = 0; i < 3; ++i)
    if ((s[i] * elem_bytes(dtype)) & 15) return false;
  return true;
}

template <typename T, int kNorm, bool kHalves, bool kBackward>
int launch_kernel(dim3 grid, const RotArgs& a, cudaStream_t stream) {
  using Shape = RotShape<T, kNorm, kBackward>;
  int bytes = Shape::kRingBytes + 2 * 16 * kThreads / a.head_slots * (int)sizeof(float);
  if (bytes < kThreads / 32 * kMaxD * (int)sizeof(float)) bytes = kThreads / 32 * kMaxD * (int)sizeof(float);      // s_red
  const int rc = tra_allow_smem<tra_rotary_kernel<T, kNorm, kHalves, kBackward>>(Shape::kRingBytes + 2 * 16 * kThreads * (int)sizeof(float));
  if (rc != TRA_OK) return rc;
  tra_rotary_kernel<T, kNorm, kHalves, kBackward><<<grid, kThreads, bytes, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? TRA_OK : TRA_ERR_CUDA;
}
template <typename T, int kNorm, bool kBackward>
int launch_halves(bool halves, dim3 grid, const RotArgs& a, cudaStream_t stream) {
  return halves ? launch_kernel<T, kNorm, true, kBackward>(grid, a, stream) : launch_kernel<T, kNorm, false, kBackward>(grid, a, stream);
}
template <typename T, bool kBackward>
int launch_norm(int norm, bool halves, dim3 grid, const RotArgs& a, cudaStream_t stream) {
  return norm == TRA_NORM_RMS     ? launch_halves<T, TRA_NORM_RMS, kBackward>(halves, grid, a, stream)
         : norm == TRA_NORM_LAYER ? launch_halves<T, TRA_NORM_LAYER, kBackward>(halves, grid, a, stream)
                                  : launch_halves<T, TRA_NORM_NONE, kBackward>(halves, grid, a, stream);
}
// Blocks of a launch (per tensor, when a block works on one): what fits the SMs at once.
template <typename T>
int wave_of(int norm, bool backward) {
  if (!backward) return 148 * (norm == TRA_NORM_NONE ? RotShape<T, TRA_NORM_NONE, false>::kBlocksPerSm : RotShape<T, TRA_NORM_RMS, false>::kBlocksPerSm);
  return 148 * (norm == TRA_NORM_NONE ? RotShape<T, TRA_NORM_NONE, true>::kBlocksPerSm : RotShape<T, TRA_NORM_RMS, true>::kBlocksPerSm);
}

int run(const tra_rotary* rot, const tra_plan_t* plan, const int32_t* pos, const tra_rotary_tensor_t* tensors,
        int n_tensors, int B, int tokens, int dtype, bool backward, void* workspace, size_t workspace_bytes,
        cudaStream_t stream) {
  if (!rot || !tensors || n_tensors < 1 || n_tensors > 3 || B < 1 || tokens < 1) return TRA_ERR_INVALID_ARG;
  if (dtype != TRA_BF16 && dtype != TRA_FP16 && dtype != TRA_FP32) return TRA_ERR_INVALID_ARG;
  if (((uintptr_t)pos & 3)) return TRA_ERR_INVALID_ARG;
  int device = 0;
  if (plan) {
    if (cudaGetDevice(&device) != cudaSuccess) return TRA_ERR_CUDA;
    if (device != plan->device || tokens != plan->S) return TRA_ERR_INVALID_ARG;
    if (!pos && rot->n_axes != 3) return TRA_ERR_INVALID_ARG;
  }
  RotArgs a;
  memset(&a, 0, sizeof(a));
  bool any_rotate = false, mixed = false, grads = false;
  int common = 0, most_heads = 1;
  const int lanes = lanes_of(rot->head_dim);
  if ((long long)B * tokens > (1 << 30)) return TRA_ERR_UNSUPPORTED;
  const int rows = B * tokens;
  for (int i = 0; i < n_tensors; ++i) {
    const tra_rotary_tensor_t& s = tensors[i];
    RotTensor& t = a.t[i];
    if (!s.src || !s.dst || s.heads < 1 || (s.flags & ~(TRA_ROTARY_ROTATE | TRA_ROTARY_TILE_MAJOR))) return TRA_ERR_INVALID_ARG;
    t.rotate = (s.flags & TRA_ROTARY_ROTATE) != 0;
    t.tile_major = (s.flags & TRA_ROTARY_TILE_MAJOR) != 0;
    if (t.tile_major && !plan) return TRA_ERR_INVALID_ARG;
    const bool normed = t.rotate && rot->norm != TRA_NORM_NONE;
    if ((s.weight && !normed) || (s.bias && (!normed || rot->norm != TRA_NORM_LAYER))) return TRA_ERR_INVALID_ARG;
    if (backward ? (normed != (s.x != nullptr)) : (s.x != nullptr)) return TRA_ERR_INVALID_ARG;
    if ((s.weight_grad && (!backward || !normed)) || (s.bias_grad && (!backward || !normed || rot->norm != TRA_NORM_LAYER)))
      return TRA_ERR_INVALID_ARG;
    if (((uintptr_t)s.src | (uintptr_t)s.dst | (uintptr_t)s.x | (uintptr_t)s.weight | (uintptr_t)s.bias) & 15)
      return TRA_ERR_INVALID_ARG;
    if (!aligned_strides(s.src_stride, dtype) || !aligned_strides(s.dst_stride, dtype) ||
        (s.x && !aligned_strides(s.x_stride, dtype)))
      return TRA_ERR_INVALID_ARG;
    grads |= s.weight_grad != nullptr || s.bias_grad != nullptr;
    t.src = s.src, t.dst = s.dst, t.x = s.x, t.weight = s.weight, t.bias = s.bias;
    for (int k = 0; k < 3; ++k) {
      t.src_stride[k] = s.src_stride[k];
      t.dst_stride[k] = s.dst_stride[k];
      t.x_stride[k] = s.x_stride[k];
    }
    t.heads = s.heads;
    common |= s.heads;
    if (s.heads > most_heads) most_heads = s.heads;
    if (t.rotate) {
      mixed |= any_rotate && a.by_source != t.tile_major;
      a.by_source = t.tile_major;
      any_rotate = true;
    }
  }
  // Heads side by side in a block.  One: a token's set-up and angles serve all its rows, and 32 tokens share a barrier
  // (the norm's backward pass on the 32.7K-token shape: 146 us, 171 with four); the forward pass, whose groups are cheap, takes four
  // where that divides the heads of every tensor (75.6K-token layer: 752 us, 746 with one; 32.7K without a norm: 110 and
  // 116).  More while the launch does not fill the GPU, and then a block per tensor.
  const int slots = kThreads / lanes;
  const int wave = dtype == TRA_FP32 ? wave_of<float>(rot->norm, backward) : wave_of<__half>(rot->norm, backward);
  const bool sums = backward && rot->norm != TRA_NORM_NONE;
  auto groups = [&](int h) { return (rows + slots / h - 1) / (slots / h); };
  int hs = 1;
  while (!sums && hs < 4 && hs < slots && common % (2 * hs) == 0) hs *= 2;
  while (hs < slots && hs < most_heads && groups(hs) < wave) hs *= 2;
  a.head_slots = hs;
  a.head_slots_log2 = log2_of(hs);
  a.lanes_log2 = log2_of(lanes);
  // the weights' sums stay in registers: one tensor per block
  a.one_tensor = groups(hs) < wave || mixed || sums;
  if (any_rotate && !pos && !plan) return TRA_ERR_INVALID_ARG;
  memcpy(a.turn, rot->turn, sizeof(a.turn));
  memcpy(a.axis, rot->axis, sizeof(a.axis));
  a.raster_of_pos = plan ? plan->d_raster_of_pos : nullptr;
  a.pos = pos;
  a.n_axes = rot->n_axes;
  a.n_tensors = n_tensors;
  a.H = plan ? plan->cfg.H : 1;
  a.W = plan ? plan->cfg.W : 1;
  a.n_video = plan ? plan->N : 0;
  a.d = rot->head_dim;
  a.lanes = lanes;
  a.eps = rot->eps;
  a.inv_d = 1.0f / (float)rot->head_dim;
  a.rows = rows;
  a.tokens = tokens;

  int blocks = groups(hs);             // blocks that stay: one wave
  if (blocks > wave) blocks = wave;
  ReduceArgs red;
  memset(&red, 0, sizeof(red));
  int n_red = 0;
  if (grads) {
    if (!workspace || ((uintptr_t)workspace & 15)) return TRA_ERR_INVALID_ARG;
    if (workspace_bytes < tra_rotary_backward_workspace_bytes(rot)) return TRA_ERR_CAPACITY;
    const long long per = 2ll * blocks * rot->head_dim;
    for (int i = 0; i < n_tensors; ++i) {
      if (!tensors[i].weight_grad && !tensors[i].bias_grad) continue;
      a.t[i].partial = (float*)workspace + per * i;
      if (tensors[i].weight_grad) {
        red.partial[n_red] = a.t[i].partial;
        red.out[n_red++] = tensors[i].weight_grad;
      }
      if (tensors[i].bias_grad) {
        red.partial[n_red] = a.t[i].partial + blocks * rot->head_dim;
        red.out[n_red++] = tensors[i].bias_grad;
      }
    }
    red.blocks = blocks;
    red.d = rot->head_dim;
  }
  const dim3 grid((unsigned)blocks, a.one_tensor ? (unsigned)n_tensors : 1u);
  const bool halves = rot->halves != 0;
  const int rc = dtype == TRA_BF16   ? (backward ? launch_norm<__nv_bfloat16, true>(rot->norm, halves, grid, a, stream)
                                                 : launch_norm<__nv_bfloat16, false>(rot->norm, halves, grid, a, stream))
                 : dtype == TRA_FP16 ? (backward ? launch_norm<__half, true>(rot->norm, halves, grid, a, stream)
                                                 : launch_norm<__half, false>(rot->norm, halves, grid, a, stream))
                                     : (backward ? launch_norm<float, true>(rot->norm, halves, grid, a, stream)
                                                 : launch_norm<float, false>(rot->norm, halves, grid, a, stream));
  if (rc != TRA_OK) return rc;
  if (n_red) {
    tra_rotary_reduce_kernel<<<dim3((rot->head_dim + kReduceCols - 1) / kReduceCols, n_red), kReduceRows * kReduceCols, 0,
                               stream>>>(red);
    TRA_CUDA_CHECK(cudaGetLastError());
  }
  return TRA_OK;
}

}  // namespace

extern "C" int tra_rotary_create(tra_rotary_t** out, const tra_rotary_config_t* cfg) {
  if (!out || !cfg) return TRA_ERR_INVALID_ARG;
  *out = nullptr;
  if (!cfg->axis || !cfg->inv_freq || cfg->n_axes < 1 || cfg->n_axes > 4) return TRA_ERR_INVALID_ARG;
  if (cfg->norm != TRA_NORM_NONE && cfg->norm != TRA_NORM_RMS && cfg->norm != TRA_NORM_LAYER) return TRA_ERR_INVALID_ARG;
  if (!(cfg->eps >= 0.0 && cfg->eps < 1e30)) return TRA_ERR_INVALID_ARG;
  if (cfg->head_dim < 16 || cfg->head_dim > kMaxD || cfg->head_dim % 16) return TRA_ERR_UNSUPPORTED;
  for (int i = 0; i < cfg->head_dim / 2; ++i)
    if (cfg->axis[i] < 0 || cfg->axis[i] >= cfg->n_axes || !isfinite(cfg->inv_freq[i])) return TRA_ERR_INVALID_ARG;
  for (int i = 0; i < cfg->head_dim / 2; ++i)
    if (fabs(cfg->inv_freq[i]) >= 18446744073709551616.0) return TRA_ERR_UNSUPPORTED;
  tra_rotary* r = new (std::nothrow) tra_rotary;
  if (!r) return TRA_ERR_CAPACITY;
  memset(r, 0, sizeof(*r));
  r->head_dim = cfg->head_dim;
  r->n_axes = cfg->n_axes;
  r->halves = cfg->halves != 0;
  r->norm = cfg->norm;
  r->eps = (float)cfg->eps;
  for (int i = 0; i < cfg->head_dim / 2; ++i) {
    r->turn[i] = turn_of(cfg->inv_freq[i]);
    r->axis[i] = (uint8_t)cfg->axis[i];
  }
  *out = r;
  return TRA_OK;
}

extern "C" int tra_rotary_destroy(tra_rotary_t* rot) {
  if (!rot) return TRA_ERR_INVALID_ARG;
  delete rot;
  return TRA_OK;
}

extern "C" size_t tra_rotary_backward_workspace_bytes(const tra_rotary_t* rot) {
  return rot ? sizeof(float) * 3 * 2 * (size_t)kBlocksMax * rot->head_dim : 0;
}

extern "C" int tra_rotary_forward(const tra_rotary_t* rot, const tra_plan_t* plan, const int32_t* pos,
                                  const tra_rotary_tensor_t* tensors, int n_tensors, int B, int tokens, int dtype,
                                  void* stream) {
  return run(rot, plan, pos, tensors, n_tensors, B, tokens, dtype, false, nullptr, 0, (cudaStream_t)stream);
}

extern "C" int tra_rotary_backward(const tra_rotary_t* rot, const tra_plan_t* plan, const int32_t* pos,
                                   const tra_rotary_tensor_t* tensors, int n_tensors, int B, int tokens, int dtype,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  return run(rot, plan, pos, tensors, n_tensors, B, tokens, dtype, true, workspace, workspace_bytes, (cudaStream_t)stream);
}
