// The cache of 4 bits: keys and values are quantised as they are written, read back, and attended over.
#include <string.h>

#include "tra_cache4.h"
#include "tra_packed_ptx.cuh"

namespace {

struct Cache4Rows {
  const void *k, *v;                    // write: [n][kv_heads][d] behind strides; read: written
  long long k_stride[2], v_stride[2];
  uint8_t *k_codes, *v_codes;
  void *k_step, *v_step;
  const int32_t* slots;
  int n, tokens;
  bool wide;                            // rows of k and v start on 32 bytes
  int* status;
};

template <typename T>
struct Pair;
template <>
struct Pair<__half> {
  using type = __half2;
};
template <>
struct Pair<__nv_bfloat16> {
  using type = __nv_bfloat162;
};
template <typename T>
__device__ __forceinline__ typename Pair<T>::type as_pair(uint32_t x) {
  return *reinterpret_cast<typename Pair<T>::type*>(&x);
}
template <typename T>
__device__ __forceinline__ uint32_t as_bits(typename Pair<T>::type x) {
  return *reinterpret_cast<uint32_t*>(&x);
}

// 32 bytes, aligned to 16 (two accesses) or to 32 (one: whole sectors, where a warp's threads are 64 bytes apart)
__device__ __forceinline__ void load64(const void* p, bool wide, uint32_t* r) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(r[8 * i]), "=r"(r[8 * i + 1]), "=r"(r[8 * i + 2]), "=r"(r[8 * i + 3]), "=r"(r[8 * i + 4]), "=r"(r[8 * i + 5]), "=r"(r[8 * i + 6]),
                     "=r"(r[8 * i + 7])
                   : "l"((const uint8_t*)p + 32 * i)
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
    }
  }
}
__device__ __forceinline__ void store64(void* p, bool wide, const uint32_t* r) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[8 * i]), "r"(r[8 * i + 1]), "r"(r[8 * i + 2]), "r"(r[8 * i + 3]),
                   "r"(r[8 * i + 4]), "r"(r[8 * i + 5]), "r"(r[8 * i + 6]), "r"(r[8 * i + 7]), "l"((uint8_t*)p + 32 * i)
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
  }
}

// The codes of a row lie in pieces of 16 bytes, and a group's in all of them: the G lanes of a row, one group each, exchange words.  Lane j's
// words of group j (keys: word t; values: half words of g = 0 .. 7) <-> words 4 j .. 4 j + 3 of the row.
template <int G>
__device__ __forceinline__ void swap_key_words(uint32_t* w, int j) {          // its own inverse for G = 4
#pragma unroll
  for (int b = 1; b < G; b <<= 1) {
    const bool up = (j & b) != 0;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      if (u & b) continue;
      const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[u] : w[u | b], b);
      if (up)
        w[u] = got;
      else
        w[u | b] = got;
    }
  }
}
template <int G>
__device__ __forceinline__ void key_words_to_row(uint32_t* w, int j) {
  if constexpr (G == 4) {
    swap_key_words<4>(w, j);
  } else {                                     // word 2 t + j: t = 0, 1 and t = 2, 3
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, j ? w[u] : w[u + 2], 1);
      if (j)
        w[u] = got;                            // t = u + 2 of group 0
      else
        w[u + 2] = got;                        // t = u of group 1
    }
    const uint32_t x = w[1];                   // (t, j): 00 10 01 11 -> 00 01 10 11
    w[1] = w[2];
    w[2] = x;
  }
}
template <int G>
__device__ __forceinline__ void row_to_key_words(uint32_t* w, int j) {
  if constexpr (G == 4) {
    swap_key_words<4>(w, j);
  } else {
    const uint32_t x = w[1];
    w[1] = w[2];
    w[2] = x;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, j ? w[u] : w[u + 2], 1);
      if (j)
        w[u] = got;
      else
        w[u + 2] = got;
    }
  }
}
// h: eight halves of words in the low 16 bits; w: words 4 j .. 4 j + 3
template <int G>
__device__ __forceinline__ void value_halves_to_row(const uint32_t* h, uint32_t* w, int j) {
  // neighbours join halves: the even lane takes g = 0, 1, 4, 5 (d 64: 0 .. 3), the odd one the others
  const bool odd = j & 1;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int mine = G == 4 ? (u & 1) + (u & 2) * 2 : u, other = G == 4 ? mine + 2 : u + 4;
    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? h[mine] : h[other], 1);
    w[u] = odd ? __byte_perm(got, h[other], 0x5410) : __byte_perm(h[mine], got, 0x5410);
  }
  if constexpr (G == 4) {
    // words 2 g + x: lanes 0, 1 hold x = 0 of g = (0, 1, 4, 5), (2, 3, 6, 7), lanes 2, 3 hold x = 1 of them
    const bool up = j & 2;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[u] : w[u + 2], 2);
      if (up)
        w[u] = got;
      else
        w[u + 2] = got;
    }
    const uint32_t x = w[1];
    w[1] = w[2];
    w[2] = x;
  }
}
// the way back; p[i]: halves of g = 2 i and 2 i + 1, side by side
template <int G>
__device__ __forceinline__ void row_to_value_pairs(uint32_t* w, uint32_t* p, int j) {
  if constexpr (G == 4) {
    const uint32_t x = w[1];
    w[1] = w[2];
    w[2] = x;
    const bool up = j & 2;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[u] : w[u + 2], 2);
      if (up)
        w[u] = got;
      else
        w[u + 2] = got;
    }
  }
  const bool odd = j & 1;
  // own half of the own words, two to a register, and the neighbour's half of them for it
  const uint32_t own = odd ? 0x7632u : 0x5410u, his = odd ? 0x5410u : 0x7632u;
  uint32_t mine[2], got[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    mine[u] = __byte_perm(w[2 * u], w[2 * u + 1], own);
    got[u] = __shfl_xor_sync(0xffffffffu, __byte_perm(w[2 * u], w[2 * u + 1], his), 1);
  }
  if constexpr (G == 4) {                      // even: g = 01, 45 own, 23, 67 the neighbour's
    p[0] = odd ? got[0] : mine[0];
    p[1] = odd ? mine[0] : got[0];
    p[2] = odd ? got[1] : mine[1];
    p[3] = odd ? mine[1] : got[1];
  } else {                                     // even: g = 01, 23 own
    p[0] = odd ? got[0] : mine[0];
    p[1] = odd ? got[1] : mine[1];
    p[2] = odd ? mine[0] : got[0];
    p[3] = odd ? mine[1] : got[1];
  }
}

// ------------------------------------------------------------------------------------ write
// Of a group of 32 channels x: low = min x, step = the smallest number of the type with 15 step >= max x - low, code = floor((x - low) / step + 1/2)
// (so that |x - (low + code step)| <= step / 2, times 1 + 2^-16 for what follows).  A group that holds a NaN or an infinity gets a step and a lowest value of NaN.
//
// The quotient is a product with the reciprocal, taken 2^-22 too large so that halves go up, added to 1.5 2^23, where the last bit is 1 and the
// rounding to a whole number is the addition's.  (A quotient less than 2^-22 of itself below a half goes up as well.  Differences and
// steps of a 16-bit type lie that close to a half only where x is 2^-13 and less of the range: one element in 10^8 of normal ones.)  The sums'
// bits, shifted to their places, add up to the codes and a constant.
//
// Bound: HBM beside instruction issue (0.63 of a slot per cycle).  A thread takes one group, G = d / 32 neighbouring lanes a row.  16,381 tokens of
// eight heads, d 128, keys and values: 17 us, 5.1 TB/s (25 with 16-byte accesses 64 bytes apart, a quotient checked by its remainder, and codes packed
// one by one); read back 16 us (25).
template <typename T>
struct Group {
  uint32_t x[16];              // pairs of channels
  float mul, neg_low, inv;     // t = x mul - low mul, of steps of 1 / inv; inv 0: every code is 0
  uint32_t packed;             // step, lowest value

  __device__ __forceinline__ void measure() {
    typename Pair<T>::type lo = as_pair<T>(x[0]), hi = lo;
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      lo = __hmin2_nan(lo, as_pair<T>(x[i]));
      hi = __hmax2_nan(hi, as_pair<T>(x[i]));
    }
    float lo0, lo1, hi0, hi1;
    unpack_pair<T>(as_bits<T>(lo), lo0, lo1);
    unpack_pair<T>(as_bits<T>(hi), hi0, hi1);
    const bool finite = fabsf(lo0) < INFINITY && fabsf(lo1) < INFINITY && fabsf(hi0) < INFINITY && fabsf(hi1) < INFINITY;
    const float l = fminf(lo0, lo1), h = fmaxf(hi0, hi1);
    // in halves, so that a range past fp32 stays one
    const float half_range = fmaf(h, 0.5f, -0.5f * l);
    uint32_t bits = pack_pair<T>(half_range * (1.f / 7.5f), l);         // step (low half), lowest value
    float st, below, unused;
    unpack_pair<T>(bits, st, unused);
    unpack_pair<T>((bits & 0xffffu) - 1u, below, unused);
    // (the product is within two units of the quotient, far less than a step of the type: at most one up or down)
    if (7.5f * st < half_range)
      bits += 1u;
    else if (st > 0.f && 7.5f * below >= half_range)
      bits -= 1u;
    unpack_pair<T>(bits, st, unused);
    if (!finite) bits = std::is_same<T, __half>::value ? 0x7e007e00u : 0x7fc07fc0u;
    packed = bits;
    // steps of 2^-60 and less (bf16 only) are brought up first, so that their reciprocal is a number
    mul = !std::is_same<T, __half>::value && st < 0x1p-60f ? 0x1p60f : 0.5f;
    inv = finite && st > 0.f ? __frcp_rn(st * mul) * (1.f + 0x1p-22f) : 0.f;
    neg_low = inv == 0.f ? 0.f : -l * mul;
    if (inv == 0.f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0u;
    }
  }
  static constexpr float kMagic = 12582912.f;        // 1.5 2^23
  static constexpr uint32_t kMagicBits = 0x4b400000u;
  // kMagicBits plus the codes of a pair
  __device__ __forceinline__ void codes(uint32_t pair, uint32_t& a, uint32_t& b) const {
    float v0, v1;
    unpack_pair<T>(pair, v0, v1);
    unpack2(ffma2(ffma2(pack2(v0, v1), pack2(mul, mul), pack2(neg_low, neg_low)), pack2(inv, inv), pack2(kMagic, kMagic)), v0, v1);
    a = __float_as_uint(v0);
    b = __float_as_uint(v1);
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(256) tra_cache4_write_kernel(const __grid_constant__ Cache4Rows a) {
  constexpr int G = D / kCacheGroup, kRowsPerBlock = 256 / G;
  const int j = threadIdx.x % G, head = blockIdx.y;
  const long long i = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / G;
  const bool of_v = blockIdx.z != 0;
  int slot = i < a.n ? a.slots[i] : -1;
  if (slot >= a.tokens) {
    tra_set_status(a.status, TRA_ERR_INVALID_ARG);
    slot = -1;
  }
  Group<T> q;
  const long long* stride = of_v ? a.v_stride : a.k_stride;
  const T* src = (const T*)(of_v ? a.v : a.k) + (i * stride[0] + head * stride[1] + j * kCacheGroup);
#pragma unroll
  for (int c = 0; c < 16; ++c) q.x[c] = 0u;
  if (slot >= 0) load64(src, a.wide, q.x);
  q.measure();
  uint32_t out[4];             // words 4 j .. 4 j + 3 of the row
  constexpr uint32_t kFour = Group<T>::kMagicBits * 0x1111u;       // what four of them in a half word leave besides the codes
  if (!of_v) {
    // word t of the group: channels 8 (n % 4) + 2 t + n / 4
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t lo = 0u - kFour, hi = 0u - kFour;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t x0, x1;
        q.codes(q.x[4 * c + t], x0, x1);
        lo += x0 << (4 * c);
        hi += x1 << (4 * c);
      }
      out[t] = __byte_perm(lo, hi, 0x5410);
    }
    key_words_to_row<G>(out, j);
  } else {
    // half a word for every g: channels 8 n + g of the group; the other half is the neighbouring group's
    uint32_t h[8];
#pragma unroll
    for (int g = 0; g < 8; g += 2) {
      h[g] = h[g + 1] = 0u - kFour;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        uint32_t x0, x1;
        q.codes(q.x[4 * n + g / 2], x0, x1);
        h[g] += x0 << (4 * n);
        h[g + 1] += x1 << (4 * n);
      }
    }
    value_halves_to_row<G>(h, out, j);
  }
  if (slot < 0) return;
  const long long row = (long long)head * a.tokens + slot;
  *reinterpret_cast<uint4*>((of_v ? a.v_codes : a.k_codes) + row * (D / 2) + j * 16) = make_uint4(out[0], out[1], out[2], out[3]);
  uint16_t* st = (uint16_t*)(of_v ? a.v_step : a.k_step) + row * (2 * G);
  st[j] = (uint16_t)q.packed;
  st[G + j] = (uint16_t)(q.packed >> 16);
}

// ------------------------------------------------------------------------------------ read
// A group's values, rounded once: code * step + low is one fused multiply-add of the type.  Pairs of codes become pairs of numbers by an OR
// with a power of two that is taken off again (fp16: 1024 + n, bf16: 128 + n, both exact).  Of a range next to the type's own, low + 15 step passes the
// largest number by what the step was rounded up (-65504 and 65504 in fp16: 65536): it becomes that number.  A group that is not finite stays NaN.
template <typename T>
__device__ __forceinline__ uint32_t value_pair(uint32_t codes, uint32_t step2, uint32_t low2) {
  constexpr bool kHalf = std::is_same<T, __half>::value;
  const auto n = __hsub2(as_pair<T>(codes | (kHalf ? 0x64006400u : 0x43004300u)), as_pair<T>(kHalf ? 0x64006400u : 0x43004300u));
  return as_bits<T>(__hmin2_nan(__hfma2(n, as_pair<T>(step2), as_pair<T>(low2)), as_pair<T>(kHalf ? 0x7bff7bffu : 0x7f7f7f7fu)));
}

// A lane's share of a row: codes 16 j .. of the row, and group j's step and lowest value.
template <int D>
struct RowShare {
  uint32_t w[4], step, low;
  __device__ __forceinline__ RowShare() : w{0u, 0u, 0u, 0u}, step(0u), low(0u) {}
  __device__ __forceinline__ void load(const uint8_t* codes, const void* steps, long long row, int j) {
    constexpr int G = D / kCacheGroup;
    const uint4 v = *reinterpret_cast<const uint4*>(codes + row * (D / 2) + j * 16);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    const uint16_t* st = (const uint16_t*)steps + row * (2 * G);
    step = st[j], low = st[G + j];
  }
  // use(x, n, at): codes n (low half of x) and n + 4 (high half) are those of the pair of channels 2 at, 2 at + 1 of group j
  template <typename Use>
  __device__ __forceinline__ void each_pair(int j, bool of_v, Use use) {
    constexpr int G = D / kCacheGroup;
    uint32_t x[4];
    if (of_v) {
      row_to_value_pairs<G>(w, x, j);
    } else {
      row_to_key_words<G>(w, j);
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = w[t];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int n = 0; n < 4; ++n) use(x[t], n, 4 * n + t);
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(256) tra_cache4_read_kernel(const __grid_constant__ Cache4Rows a) {
  constexpr int G = D / kCacheGroup, kRowsPerBlock = 256 / G;
  const int j = threadIdx.x % G, head = blockIdx.y;
  const long long i = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / G;
  const bool of_v = blockIdx.z != 0;
  int slot = i < a.n ? a.slots[i] : -1;
  if (slot >= a.tokens) {
    tra_set_status(a.status, TRA_ERR_INVALID_ARG);
    slot = -1;
  }
  RowShare<D> s;
  if (slot >= 0) s.load(of_v ? a.v_codes : a.k_codes, of_v ? a.v_step : a.k_step, (long long)head * a.tokens + slot, j);
  uint32_t v[16];
  const uint32_t step2 = s.step * 0x10001u, low2 = s.low * 0x10001u;
  s.each_pair(j, of_v, [&](uint32_t x, int n, int at) { v[at] = value_pair<T>((x >> (4 * n)) & 0x000f000fu, step2, low2); });
  if (slot < 0) return;
  const long long* stride = of_v ? a.v_stride : a.k_stride;
  store64((T*)(of_v ? a.v : a.k) + i * stride[0] + head * stride[1] + j * kCacheGroup, a.wide, v);
}

// ------------------------------------------------------------------------------------ many rows: the keys read back first
// Sequence s of a pass gets the rows s * stride .. of two 16-bit tensors: the keys of its axis (tra_key_axis), as their ranges say, which the
// attention launch behind it reads as begin / end.  An element low + step n has up to 4 bits more than the type, and more where low and
// step are of different sizes; rounded to the type alone, keys and values would each add as much error as the rounding of the
// result (bf16, 97 queries over 65,500 keys: 3.8e-3 off, against 1.7e-3 for the result's rounding alone).  So
//   fp16: [rows][2][kv_heads][d], the rounded element and, as a second piece, what rounding took;
//   bf16: [rows][kv_heads][d] in fp16, of multiples that keep the largest of a sequence and head below 2^15 (kv_top), beside Q in fp16 by multiples of
//         its rows (q_mul): one product instead of two (four chunks, 40 / 8 heads, window 4,096: 385 us in pieces, 223 so).
struct Cache4Expand {
  tra_packed_launch a;
  const uint8_t *k_codes, *v_codes;
  const void *k_step, *v_step;
  void *k, *v;
  int32_t *begin, *end;
  int stride;
  uint32_t* top;               // bf16: [K, V][n_seq][kv_heads], cleared
  __half* q;                   //       [total_q][heads][d]
  float* q_mul;                //       [total_q][heads]
  int step_blocks;             //       blocks of a (sequence, head, side) that look at its steps
  bool wide;                   // k and v start on 32 bytes (a workspace need not); their rows then do
};

// A sequence's keys as the launches of a pass see them.
struct ExpandRange {
  tra_seq_range q, k;
  int gap, len;
  template <int kOrder>
  __device__ __forceinline__ static ExpandRange of(const Cache4Expand& e, int seq) {
    const tra_packed_launch& p = e.a;
    ExpandRange r;
    r.q = tra_clamp_range(p.cu_q[seq], p.cu_q[seq + 1], p.total_q, p.max_q, p.status);
    r.k = tra_clamp_range(p.k_begin[seq], p.k_end[seq], p.total_k, p.max_k, p.status);
    const tra_key_axis<kOrder> axis(p, r.k.len - r.q.len, r.k.len);
    r.gap = axis.gap;
    r.len = r.q.len > 0 ? min(axis.len, e.stride) : 0;
    return r;
  }
  __device__ __forceinline__ long long key(const tra_packed_launch& p, int v) const { return (long long)k.begin + (v >= p.sink_rows ? v + gap : v); }
};

// bf16: the largest size of what a sequence's keys and values of a head may stand for (blocks z < 2 n_seq), from steps and lowest values
// alone, and Q in fp16 (the other blocks: 256 / (d / 8) rows each, d / 8 threads a row).
template <int D, int kOrder>
__global__ void __launch_bounds__(256) tra_cache4_multiples_kernel(const __grid_constant__ Cache4Expand e) {
  using T = __nv_bfloat16;
  constexpr int G = D / kCacheGroup;
  const tra_packed_launch& p = e.a;
  allow_next_launch();
  const int n_top = e.step_blocks * p.kv_heads * 2 * p.n_seq;
  if ((int)blockIdx.x < n_top) {
    const int block = blockIdx.x % e.step_blocks, rest = blockIdx.x / e.step_blocks, head = rest % p.kv_heads, side = rest / p.kv_heads;
    const bool of_v = side & 1;
    const ExpandRange r = ExpandRange::of<kOrder>(e, side >> 1);
    float top = 0.f;
    for (int v = block * 256 + threadIdx.x; v < r.len; v += e.step_blocks * 256) {
      const uint32_t* w = (const uint32_t*)((const T*)(of_v ? e.v_step : e.k_step) + ((long long)head * p.total_k + r.key(p, v)) * (2 * G));
#pragma unroll
      for (int i = 0; i < G / 2; ++i) {
        float s0, s1, l0, l1;
        unpack_pair<T>(w[i], s0, s1);
        unpack_pair<T>(w[G / 2 + i], l0, l1);
        top = fmaxf(top, fmaxf(fmaf(15.f, s0, fabsf(l0)), fmaf(15.f, s1, fabsf(l1))));        // (NaN, of a group that is not finite, is left out)
      }
    }
    top = fminf(top, 3e38f);
    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
    if ((threadIdx.x & 31) == 0 && most) atomicMax(e.top + ((of_v ? p.n_seq : 0) + (side >> 1)) * p.kv_heads + head, most);
    return;
  }
  constexpr int kLanes = D / 8;
  const long long row = (long long)((int)blockIdx.x - n_top) * (256 / kLanes) + threadIdx.x / kLanes, rows = (long long)p.total_q * p.heads;
  const int lane = threadIdx.x % kLanes;
  uint4 x = make_uint4(0u, 0u, 0u, 0u);
  if (row < rows) x = *reinterpret_cast<const uint4*>((const T*)p.q + row / p.heads * p.q_stride[0] + row % p.heads * p.q_stride[1] + lane * 8);
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack_pair<T>(w[i], a, b);
    top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float mul = tra_fp16_mul(top);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack_pair<T>(w[i], a, b);
    w[i] = pack_pair<__half>(a * mul, b * mul);
  }
  if (row >= rows) return;
  reinterpret_cast<uint4*>(e.q + row * D)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
  if (lane == 0) e.q_mul[row] = tra_inverse_pow2(mul);
}

template <typename T, int D, int kOrder>
__global__ void __launch_bounds__(256) tra_cache4_expand_kernel(const __grid_constant__ Cache4Expand e) {
  constexpr int G = D / kCacheGroup, kRowsPerBlock = 256 / G;
  const tra_packed_launch& p = e.a;
  const int j = threadIdx.x % G, head = blockIdx.y, seq = blockIdx.z >> 1;
  const bool of_v = blockIdx.z & 1;
  const int v0 = blockIdx.x * kRowsPerBlock + threadIdx.x / G;
  const ExpandRange range = ExpandRange::of<kOrder>(e, seq);
  if (head == 0 && blockIdx.z == 2 * seq && blockIdx.x == 0 && threadIdx.x == 0) {
    e.begin[seq] = seq * e.stride;
    e.end[seq] = seq * e.stride + range.len;
  }
  RowShare<D> r;
  if (v0 < range.len) r.load(of_v ? e.v_codes : e.k_codes, of_v ? e.v_step : e.k_step, (long long)head * p.total_k + range.key(p, v0), j);
  uint32_t v[16], rest[16];
  float step, low, unused;
  unpack_pair<T>(r.step, step, unused);
  unpack_pair<T>(r.low, low, unused);
  constexpr bool kFp16 = std::is_same<T, __half>::value;
  if constexpr (!kFp16) {
    wait_last_launch();
    const float mul = tra_fp16_mul(__uint_as_float(e.top[((of_v ? p.n_seq : 0) + seq) * p.kv_heads + head]));
    step *= mul;
    low *= mul;
  }
  r.each_pair(j, of_v, [&](uint32_t x, int n, int at) {
    // 2^23 + code is a float; that power of two is taken off again, exactly
    const float a = __uint_as_float(0x4b000000u | ((x >> (4 * n)) & 15u)) - 8388608.f, b = __uint_as_float(0x4b000000u | ((x >> (4 * n + 16)) & 15u)) - 8388608.f;
    const float y = fmaf(a, step, low), z = fmaf(b, step, low);
    v[at] = pack_pair<__half>(y, z);
    if constexpr (kFp16) {                                   // (low + 15 step may pass the type's range by a step's rounding)
      float f, g;
      unpack_pair<T>(v[at], f, g);
      if (fabsf(f) == INFINITY || fabsf(g) == INFINITY) v[at] = pack_pair<T>(fminf(fmaxf(y, -65504.f), 65504.f), fminf(fmaxf(z, -65504.f), 65504.f));
      rest[at] = rest_pair<T>(y, z, v[at]);
    }
  });
  if (v0 >= range.len) return;
  T* dst = (T*)(of_v ? e.v : e.k) + (((long long)seq * e.stride + v0) * (kFp16 ? 2 : 1) * p.kv_heads + head) * D + j * kCacheGroup;
  store64(dst, e.wide, v);
  if constexpr (kFp16) store64(dst + (long long)p.kv_heads * D, e.wide, rest);
}

// ------------------------------------------------------------------------------------ host side
constexpr int kMaxSplits = 256, kClusterMax = 8;
// Rows per key/value head up to which the codes are read by the products' kernel; more are read back first.  40 / 8 heads, d 128, 60 and 80 rows, us, directly and
// read back: bf16, one sequence of 30,000 keys 71 and 146, 79 and 79; 16 of 16,000 528 and 645, 492 and 493; 64 of 1,000 165 and 209, 148 and 149; 8 of 4,000 75
// and 123, 82 and 82.  fp16: 70 and 137, 121 and 121; 516 and 632, 892 and 892; 162 and 207, 225 and 225: level at about 110 rows
// there (more rows only repeat the reading of the codes, 16 rows at a time).
constexpr int kRowsDirect = 64;
constexpr size_t kExpandBytes = 512u << 20;      // keys and values read back at a time (one sequence at least)

bool bad_cache(const tra_packed_t* h, const tra_cache4_t* c) {
  if (!h || !c || c->tokens < 0 || (c->tokens & 1)) return true;
  if (c->tokens == 0) return false;
  const uintptr_t all = (uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->k_step | (uintptr_t)c->v_step;
  return !c->k || !c->v || !c->k_step || !c->v_step || (all & 15);
}

// How a call runs: `direct` (few rows) in `splits` parts of `chunk` keys, or in passes of `seqs` sequences whose keys are read back.
struct Choice4 {
  bool direct, clustered;
  int splits, chunk, row_tiles;
  int seqs, stride;
};

Choice4 choose4(const tra_packed_t* h, int n_seq, int max_q, int max_k) {
  const int group = h->cfg.heads / h->cfg.kv_heads;
  Choice4 c = {};
  const long long rows = (long long)max_q * group;
  c.direct = rows <= kRowsDirect;
  c.splits = 1, c.chunk = 128, c.row_tiles = 1;
  if (max_q == 0) return c;
  if (c.direct) {
    c.row_tiles = (int)((rows + 15) / 16);
    int longest = tra_packed_longest_axis(h, max_k, max_q);
    if (longest < max_k) {                       // first tokens take whole pieces here
      const long long more = (long long)longest + 31;
      longest = more < max_k ? (int)more : max_k;
    }
    // Blocks that fit the GPU at once.  Few units: as many parts as fill it once, each of at least 256 keys, in a cluster where eight
    // are enough or the cache is short (see choose in tra_packed.cu).  Many units: parts of about 3,328 keys, so that blocks of different
    // lengths spread evenly, and no clusters, whose blocks start and end together (64 caches of up to 32K keys, eight heads: 510 us
    // whole, 555 in two clustered parts, 405 in two, 332 in parts of 3,328, 348 in parts of 2,048; 32 windows of 4,096 keys: 61 whole, 64
    // to 74 in two to six).  Parts of 2,048, 3,328, 5,120, 8,192 keys and whole, us: 64 caches of 32,768 632, 609, 607, 608, 738; 40 of up to 65,536
    // 428, 409, 408, 420, 759; 32 of 16,384 169, 166, 179, 197, 189; 128 of up to 8,192 188, 189, 190, 202, 202; 256 of 4,096 325, 300, 309, 309, 309; 200 of up to
    // 3,000 all 121; d 64, fp16, 12 heads, 64 of up to 32,768 335, 323, 326, 334, 429.
    const long long slots = (long long)(rows <= 8 ? 3 : 2) * h->sm_count;
    const long long units = (long long)n_seq * h->cfg.kv_heads * c.row_tiles;
    const bool many = 2 * units > slots;
    long long parts = many ? (longest + 1663) / 3328 : slots / units;
    const long long most = ((long long)longest + 255) / 256;
    if (parts > most) parts = most;
    if (!many && parts > kClusterMax && longest <= 1024 * kClusterMax) parts = kClusterMax;
    if (parts > kMaxSplits) parts = kMaxSplits;
    if (parts < 1) parts = 1;
    c.chunk = (int)(((longest + parts - 1) / parts + 127) / 128 * 128);
    if (c.chunk < 128) c.chunk = 128;
    c.splits = longest > 0 ? (int)(((long long)longest + c.chunk - 1) / c.chunk) : 1;
    c.clustered = !many && c.splits > 1 && c.splits <= kClusterMax;
  } else {
    c.stride = (tra_packed_longest_axis(h, max_k, max_q) + 7) / 8 * 8;
    const size_t one = (size_t)c.stride * h->cfg.kv_heads * h->cfg.head_dim * (h->cfg.dtype == TRA_BF16 ? 4 : 8);
    const size_t most = one ? kExpandBytes / one : n_seq;
    c.seqs = (int)(most < 1 ? 1 : most > (size_t)n_seq ? n_seq : most > 16384 ? 16384 : most);
    while ((long long)c.seqs * c.stride > (1 << 30)) --c.seqs;
  }
  return c;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace of a call that reads keys back.
struct Layout4 {
  size_t v, ranges, top, q_mul, q, attn, bytes;
};
Layout4 layout4(const tra_packed_t* h, const Choice4& c, int n_seq, int total_q, int max_q) {
  const bool bf16 = h->cfg.dtype == TRA_BF16;
  const size_t d = h->cfg.head_dim, kv = h->cfg.kv_heads, heads = h->cfg.heads;
  Layout4 l;
  l.v = round256((size_t)c.seqs * c.stride * kv * d * (bf16 ? 2 : 4));
  l.ranges = 2 * l.v;
  l.top = l.ranges + round256(sizeof(int32_t) * 2 * (size_t)c.seqs);
  l.q_mul = l.top + (bf16 ? round256(sizeof(uint32_t) * 2 * c.seqs * kv) : 0);
  l.q = l.q_mul + (bf16 ? round256(sizeof(float) * total_q * heads) : 0);
  l.attn = l.q + (bf16 ? round256((size_t)total_q * heads * d * 2) : 0);
  // (the last pass may hold fewer sequences, which take more parts)
  const int last = n_seq % c.seqs;
  const size_t pass = tra_packed_attn_workspace_bytes(h, c.seqs, total_q, max_q, c.stride);
  const size_t end = last ? tra_packed_attn_workspace_bytes(h, last, total_q, max_q, c.stride) : 0;
  l.bytes = l.attn + (pass > end ? pass : end);
  return l;
}

size_t workspace4(const tra_packed_t* h, const Choice4& c, int n_seq, int total_q, int max_q) {
  if (max_q == 0) return 0;
  if (c.direct) return c.splits > 1 && !c.clustered ? sizeof(float) * (size_t)c.splits * total_q * h->cfg.heads * (h->cfg.head_dim + 2) : 0;
  return layout4(h, c, n_seq, total_q, max_q).bytes;
}

template <typename T, int D>
int launch_rows_io(const Cache4Rows& a, int kv_heads, bool write, cudaStream_t stream) {
  constexpr int kRows = 256 / (D / kCacheGroup);
  const dim3 grid((unsigned)(((long long)a.n + kRows - 1) / kRows), (unsigned)kv_heads, 2);
  return write ? tra_launch(tra_cache4_write_kernel<T, D>, grid, 256, 0, stream, false, 1, a)
               : tra_launch(tra_cache4_read_kernel<T, D>, grid, 256, 0, stream, false, 1, a);
}

// The stride of a dimension of one entry is never used; the others are positive multiples of 16 bytes.
bool bad_rows(const void* ptr, const int64_t* stride, long long tokens, int heads) {
  if (!ptr || ((uintptr_t)ptr & 15)) return true;
  const long long n[2] = {tokens, heads};
  for (int i = 0; i < 2; ++i)
    if (n[i] > 1 && (stride[i] < 8 || (stride[i] & 7) || stride[i] >= (1ll << 38))) return true;
  return false;
}

int rows_io(const tra_packed_t* h, const tra_cache4_t* c, const void* k, const void* v, const int64_t* ks, const int64_t* vs, const int32_t* slots, int n,
            bool write, void* stream) {
  if (bad_cache(h, c) || n < 0) return TRA_ERR_INVALID_ARG;
  if (c->tokens > (1 << 30) || n > (1 << 30)) return TRA_ERR_UNSUPPORTED;
  if (n == 0) return TRA_OK;
  const int kv = h->cfg.kv_heads;
  if (!ks || !vs || !slots || ((uintptr_t)slots & 3) || bad_rows(k, ks, n, kv) || bad_rows(v, vs, n, kv)) return TRA_ERR_INVALID_ARG;
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return TRA_ERR_CUDA;
  if (device != h->device) return TRA_ERR_INVALID_ARG;
  const bool wide = !(((uintptr_t)k | (uintptr_t)v | (n > 1 ? (uintptr_t)(ks[0] | vs[0]) * 2 : 0) | (kv > 1 ? (uintptr_t)(ks[1] | vs[1]) * 2 : 0)) & 31);
  Cache4Rows a = {k, v, {ks[0], ks[1]}, {vs[0], vs[1]}, (uint8_t*)c->k, (uint8_t*)c->v, c->k_step, c->v_step, slots, n, c->tokens, wide, h->d_status};
  cudaStream_t s = (cudaStream_t)stream;
  if (h->cfg.head_dim == 128)
    return h->cfg.dtype == TRA_BF16 ? launch_rows_io<__nv_bfloat16, 128>(a, kv, write, s) : launch_rows_io<__half, 128>(a, kv, write, s);
  return h->cfg.dtype == TRA_BF16 ? launch_rows_io<__nv_bfloat16, 64>(a, kv, write, s) : launch_rows_io<__half, 64>(a, kv, write, s);
}

template <typename T, int D, int kOrder>
int launch_expand_order(const tra_packed_ctx& c, Cache4Expand e, bool first) {
  constexpr int kRows = 256 / (D / kCacheGroup);
  const int seqs = e.a.n_seq;
  const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
  if constexpr (bf16) {
    if (cudaMemsetAsync(e.top, 0, sizeof(uint32_t) * 2 * seqs * e.a.kv_heads, c.stream) != cudaSuccess) return TRA_ERR_CUDA;
    // about eight rounds of 256 keys per block, and enough blocks where there are few heads
    long long blocks = ((long long)e.stride + 2047) / 2048;
    const long long fill = 4ll * c.h->sm_count / (2ll * seqs * e.a.kv_heads) + 1, most = ((long long)e.stride + 255) / 256;
    if (blocks < fill) blocks = fill;
    e.step_blocks = (int)(blocks > most ? (most < 1 ? 1 : most) : blocks);
    const long long rows = first ? ((long long)e.a.total_q * e.a.heads + 256 / (D / 8) - 1) / (256 / (D / 8)) : 0;
    const long long grid = (long long)e.step_blocks * e.a.kv_heads * 2 * seqs + rows;
    if (grid > 0x7fffffffll) return TRA_ERR_UNSUPPORTED;
    const int rc = tra_launch(tra_cache4_multiples_kernel<D, kOrder>, dim3((unsigned)grid), 256, 0, c.stream, false, 1, e);
    if (rc != TRA_OK) return rc;
  }
  const int blocks = e.stride > 0 ? (e.stride + kRows - 1) / kRows : 1;
  return tra_launch(tra_cache4_expand_kernel<T, D, kOrder>, dim3((unsigned)blocks, (unsigned)e.a.kv_heads, (unsigned)(2 * seqs)), 256, 0, c.stream, bf16, 1, e);
}
template <typename T, int D>
int launch_expand(const tra_packed_ctx& c, const Cache4Expand& e, bool first) {
  return e.a.order == kOrderWindow ? launch_expand_order<T, D, kOrderWindow>(c, e, first) : launch_expand_order<T, D, kOrderCausal>(c, e, first);
}

}  // namespace

extern "C" int tra_cache4_write(const tra_packed_t* h, const tra_cache4_t* c, const void* k, const void* v, const int64_t* k_stride,
                                const int64_t* v_stride, const int32_t* slots, int n, void* stream) {
  return rows_io(h, c, k, v, k_stride, v_stride, slots, n, true, stream);
}

extern "C" int tra_cache4_read(const tra_packed_t* h, const tra_cache4_t* c, void* k, void* v, const int64_t* k_stride, const int64_t* v_stride,
                               const int32_t* slots, int n, void* stream) {
  return rows_io(h, c, k, v, k_stride, v_stride, slots, n, false, stream);
}

extern "C" size_t tra_packed_attn_cache4_workspace_bytes(const tra_packed_t* h, int n_seq, int total_q, int max_q, int max_k) {
  if (!h || n_seq < 1 || total_q < 0 || max_q < 0 || max_k < 0 || max_q > total_q) return 0;
  if (total_q > (1 << 30) || max_k > (1 << 30)) return 0;    // sizes that the call refuses
  return workspace4(h, choose4(h, n_seq, max_q, max_k), n_seq, total_q, max_q);
}

extern "C" int tra_packed_attn_cache4(const tra_packed_t* h, const tra_packed_args_t* args, const tra_cache4_t* cache, void* workspace,
                                      size_t workspace_bytes, void* stream_) {
  if (!args || bad_cache(h, cache)) return TRA_ERR_INVALID_ARG;
  tra_packed_args_t a = *args;
  if (a.o_rest) return TRA_ERR_INVALID_ARG;                  // there is no backward call that would read it
  a.total_k = cache->tokens;
  tra_cache4_launch q;
  memset(&q, 0, sizeof(q));
  int rc = tra_packed_begin(h, &a, false, &q.a);
  if (rc != TRA_OK) return rc;
  const tra_packed_ctx ctx = {h, (cudaStream_t)stream_};
  const Choice4 c = choose4(h, a.n_seq, a.max_q, a.max_k);
  const size_t need = workspace4(h, c, a.n_seq, a.total_q, a.max_q);
  if (need && (!workspace || ((uintptr_t)workspace & 15))) return TRA_ERR_INVALID_ARG;
  if (workspace_bytes < need) return TRA_ERR_CAPACITY;
  if (c.direct) {
    if (c.splits > 1 && !c.clustered && (long long)a.total_q * q.a.heads > 0x7fffffffll) return TRA_ERR_UNSUPPORTED;
    q.a.o = a.o;
    q.a.splits = c.splits;
    q.a.sink_rows = (int)(((long long)h->cfg.sinks + 31) / 32 * 32);
    q.k = (const uint8_t*)cache->k, q.v = (const uint8_t*)cache->v, q.k_step = cache->k_step, q.v_step = cache->v_step;
    q.row_tiles = c.row_tiles;
    if (need) {
      const long long rows = (long long)c.splits * a.total_q * q.a.heads;
      q.a.part_o = (float*)workspace;
      q.a.part_lse2 = q.a.part_o + rows * h->cfg.head_dim;
      q.a.part_exact = a.lse ? q.a.part_lse2 + rows : nullptr;
    }
    if ((long long)q.a.kv_heads * c.row_tiles > 65535) return TRA_ERR_UNSUPPORTED;
    rc = tra_cache4_rows(ctx, q, c.chunk, c.clustered);
    return rc != TRA_OK || !need ? rc : tra_packed_join(ctx, q.a);
  }
  // many rows: passes over sequences, keys read back into the workspace
  const bool bf16 = h->cfg.dtype == TRA_BF16;
  const int kv = h->cfg.kv_heads, d = h->cfg.head_dim;
  const Layout4 l = layout4(h, c, a.n_seq, a.total_q, a.max_q);
  uint8_t* ws = (uint8_t*)workspace;
  Cache4Expand e;
  memset(&e, 0, sizeof(e));
  e.a = q.a;
  if (e.a.order != kOrderWindow) e.a.sink_rows = 0;
  e.k_codes = (const uint8_t*)cache->k, e.v_codes = (const uint8_t*)cache->v, e.k_step = cache->k_step, e.v_step = cache->v_step;
  e.k = ws, e.v = ws + l.v;
  e.wide = !((uintptr_t)ws & 31);
  e.begin = (int32_t*)(ws + l.ranges), e.end = e.begin + c.seqs;
  e.top = (uint32_t*)(ws + l.top), e.q_mul = (float*)(ws + l.q_mul), e.q = (__half*)(ws + l.q);
  e.stride = c.stride;
  for (int s = 0; s < a.n_seq; s += c.seqs) {
    const int n = a.n_seq - s < c.seqs ? a.n_seq - s : c.seqs;
    e.a.cu_q = a.cu_q + s, e.a.k_begin = a.k_begin + s, e.a.k_end = a.k_end + s;
    e.a.n_seq = n;
    if (bf16)
      rc = d == 128 ? launch_expand<__nv_bfloat16, 128>(ctx, e, s == 0) : launch_expand<__nv_bfloat16, 64>(ctx, e, s == 0);
    else
      rc = d == 128 ? launch_expand<__half, 128>(ctx, e, s == 0) : launch_expand<__half, 64>(ctx, e, s == 0);
    if (rc != TRA_OK) return rc;
    tra_packed_args_t b = a;
    b.k = e.k, b.v = e.v;
    b.k_stride[0] = b.v_stride[0] = (int64_t)(bf16 ? 1 : 2) * kv * d, b.k_stride[1] = b.v_stride[1] = d;
    if (bf16) b.q = e.q, b.q_stride[0] = (int64_t)q.a.heads * d, b.q_stride[1] = d;
    b.cu_q = a.cu_q + s, b.k_begin = e.begin, b.k_end = e.end;
    b.n_seq = n, b.total_k = c.seqs * c.stride, b.max_k = c.stride;
    rc = tra_packed_attn_read_back(h, &b, e.q_mul, e.top, ws + l.attn, workspace_bytes - l.attn, stream_);
    if (rc != TRA_OK) return rc;
  }
  return TRA_OK;
}
