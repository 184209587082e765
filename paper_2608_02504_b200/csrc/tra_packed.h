// Kernel arguments of the packed-attention launches, where a thread block finds its sequence, and the per-shape
// launchers (one translation unit per kernel and head_dim, so that they compile in parallel).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tra_common.cuh"

struct tra_packed {
  tra_packed_config_t cfg;
  int device, sm_count;
  int* d_status;
};

// One launch, as the kernels see it.  Rows of a (sequence, key/value head) are its tokens times the `group` query
// heads that share the key/value head, token-major: row r of a tile is token r / group, head r % group.
struct tra_packed_launch {
  CUtensorMap map_q, map_k, map_v, map_do;   // boxes: 64 channels x (group heads x tile tokens | 1 head x 128 tokens)
  CUtensorMap map_q_stream, map_do_stream;   // backward, streamed tiles of stream_rows rows (then K and V boxes have that many, too)
  // window with first tokens: the key tile that holds the last of them and, behind them, the first keys of the window
  CUtensorMap map_k_first, map_v_first, map_k_rest, map_v_rest;
  const void *q, *k, *v, *o_in, *d_o;
  void *o, *dq, *dk, *dv;
  float* lse;                  // forward: written or NULL; backward: read
  void* o_rest;                // [total_q][heads][d] o minus its rounding, or NULL; forward: written (with lse); backward: read
  float* part_o;               // forward, split over the keys: [splits][total_q][heads][d]
  float* part_lse2;            //   [splits][total_q][heads] base-2 log of the sum the part was divided by
  float* part_exact;           //   [splits][total_q][heads] base-2 log of the unrounded sum (lse asked for) or NULL
  float* delta;                // backward: [total_q][heads] sum of dO O
  uint32_t* norms;             // backward, fp16: [2][kv_heads] bits of the largest squared norm of a row of dO, of V
  long long q_stride[2], k_stride[2], v_stride[2], o_stride[2], do_stride[2], dq_stride[2], dk_stride[2], dv_stride[2];
  const int32_t *cu_q, *k_begin, *k_end;
  int n_seq, total_q, total_k, max_q, max_k;
  int heads, kv_heads, group, tile_tokens;   // tile_tokens = 128 / group: query tokens of a 128-row tile
  int stream_rows, stream_tokens;            // backward: rows of a streamed tile, 128 or 64, and stream_rows / group
  int order, splits, n_units;                // n_units: query-tile pairs (forward) or key / query tiles (backward) launched
  int window, sinks, sink_rows;              // kOrderWindow; sink_rows: sinks rounded up to whole 8-row pieces of a tile
  int dq_tiles;                              // backward with a window: query tiles of a dQ block, one after the other
  int sink_steps, sink_slots;                // backward: see tra_find_sink_unit; 0: the first keys' tiles walk all their queries
  float* sink_part;                          //   [slot][kv_heads][sinks][dK, dV][d] fp32
  // fp16 products for bf16 tensors (kPieces = 0 of the forward kernel): Q, K and V are fp16 multiples of the elements
  const float* q_mul;                        // [total_q][heads]: Q's elements are these times what the map reads
  const uint32_t* kv_top;                    // [K, V][n_seq][kv_heads]: bits of the largest size, of which the multiple follows
  float sm_scale;
  int* status;
};

// Which keys a query at position p of its sequence's key axis sees (p of the last query = the last key): all; keys 0 .. p; of these, the
// last `window` and the first `sinks`.
constexpr int kOrderNone = 0, kOrderCausal = 1, kOrderWindow = 2;

struct tra_packed_ctx {
  const tra_packed_t* h;
  cudaStream_t stream;
};

int tra_packed_fwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_window_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_window_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_pieces_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_pieces_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_fp16_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_fp16_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_window_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_window_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_few_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_few_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_rows(const tra_packed_ctx& c, const tra_packed_launch& a, int chunk, bool clustered);

#ifdef __CUDACC__
namespace {

// The power of two that brings numbers of up to `top` below 2^15, where fp16 holds the most of them.
__device__ __forceinline__ float tra_fp16_mul(float top) {
  const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -100), 128);        // top < 2^e
  return __uint_as_float((uint32_t)(127 + 15 - e) << 23);
}
__device__ __forceinline__ float tra_inverse_pow2(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }

// Launch; after_last: may start while the stream's last kernel ends (see wait_last_launch); cluster: blocks along z that form
// a thread-block cluster.
template <typename... Params, typename... Args>
int tra_launch(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t stream, bool after_last, int cluster,
               const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  if (after_last) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = attr[cfg.numAttrs].val.clusterDim.y = 1;
    attr[cfg.numAttrs++].val.clusterDim.z = (unsigned)cluster;
  }
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? TRA_OK : TRA_ERR_CUDA;
}

// The token range of a sequence, brought inside the tensor and the stated maximum; what had to be cut is recorded.
struct tra_seq_range {
  int begin, len;
};
__device__ __forceinline__ tra_seq_range tra_clamp_range(int begin, int end, int total, int max_len, int* status) {
  const int b = min(max(begin, 0), total);
  const int e = min(max(end, b), total);
  const int len = min(e - b, max_len);
  if (b != begin || b + len != end) atomicCAS(status, 0, TRA_ERR_INVALID_ARG);
  return {b, len};
}

// The keys that a tile of queries walks.  With a window these are not one range: its first keys, [0, sink_rows), and the window's, from
// that of the tile's first query on.  They are walked as one axis v, closed up: key v below sink_rows, v + gap from there on, and a
// tile of keys may hold both.  (Tiles of their own for the first tokens and tiles that start at multiples of 128 keys take two more tiles
// per query tile.)  A query at position p sees v < p + 1 - gap, of these v < sinks and v > p - gap - window: gap > 0 only
// where the tile's first window starts behind sink_rows, and then every window of the tile does.
template <int kOrder>
struct tra_key_axis {
  int gap, len;                // len: of the axis, the sequence's last key included
  __device__ __forceinline__ tra_key_axis(const tra_packed_launch& p, int first_position, int k_len) {
    gap = kOrder == kOrderWindow ? max(first_position + 1 - p.window - p.sink_rows, 0) : 0;
    len = k_len - gap;
  }
};

// Loads `rows` keys from v0 on (a multiple of `rows`) into a tile of kAtoms 64-channel pieces, `atom_bytes` apart.
template <int kOrder, int kAtoms, typename Load>
__device__ __forceinline__ void tra_load_keys(const tra_packed_launch& p, int v0, int rows, int gap, bool v_side, uint32_t dst, int atom_bytes,
                                              Load load) {
  const CUtensorMap* whole = v_side ? &p.map_v : &p.map_k;
  if (kOrder == kOrderWindow && v0 < p.sink_rows && v0 + rows > p.sink_rows) {        // the last of the first tokens, and the window
    for (int a = 0; a < kAtoms; ++a) {
      load(dst + a * atom_bytes, v_side ? &p.map_v_first : &p.map_k_first, a * 64, v0);
      load(dst + a * atom_bytes + (p.sink_rows - v0) * 128, v_side ? &p.map_v_rest : &p.map_k_rest, a * 64, p.sink_rows + gap);
    }
    return;
  }
  const int key = kOrder == kOrderWindow && v0 >= p.sink_rows ? v0 + gap : v0;
  for (int a = 0; a < kAtoms; ++a) load(dst + a * atom_bytes, whole, a * 64, key);
}

// What a thread block works on: unit `index` of a sequence, of its `count`, and the sequence's token ranges.
struct tra_unit {
  int seq, index, count;   // seq = -1: nothing
  tra_seq_range q, k;
};

// Finds a unit: `unit_tokens` consecutive queries, or (by_keys) keys, of a sequence.  The units of sequence s are numbered from
// first(s) = floor(begin(s) / unit_tokens) + s on, which leaves room for all of them (some numbers mean nothing), and makes the
// sequence of a number a search in the ascending bounds, 32 at a time.  one_each: unit s is the whole of sequence s.
// One warp calls it; every lane gets the result.  There are at least as many numbers as sequences, and number s looks at the ranges of
// sequence s too, so that each is reported that runs backwards, which the search might never meet.
__device__ __forceinline__ tra_unit tra_find_unit(const tra_packed_launch& p, bool by_keys, bool one_each, int unit_tokens, int unit) {
  const int lane = threadIdx.x & 31;
  tra_unit u = {-1, 0, 1, {0, 0}, {0, 0}};
  if (one_each) {
    u.q = tra_clamp_range(p.cu_q[unit], p.cu_q[unit + 1], p.total_q, p.max_q, p.status);
    u.k = tra_clamp_range(p.k_begin[unit], p.k_end[unit], p.total_k, p.max_k, p.status);
    if ((by_keys ? u.k.len : u.q.len) > 0) u.seq = unit;
    return u;
  }
  if (unit < p.n_seq) {
    tra_clamp_range(p.cu_q[unit], p.cu_q[unit + 1], p.total_q, p.max_q, p.status);
    tra_clamp_range(p.k_begin[unit], p.k_end[unit], p.total_k, p.max_k, p.status);
  }
  int lo = 0, hi = p.n_seq;
  while (true) {
    const int stride = (hi - lo + 31) / 32;
    const int s = lo + lane * stride;
    int first = 0, q0 = 0, q1 = 0, k0 = 0, k1 = 0;
    if (s < hi) {
      if (stride == 1) q0 = p.cu_q[s], q1 = p.cu_q[s + 1], k0 = p.k_begin[s], k1 = p.k_end[s];
      const int begin = stride == 1 ? (by_keys ? k0 : q0) : (by_keys ? p.k_begin[s] : p.cu_q[s]);
      first = min(max(begin, 0), by_keys ? p.total_k : p.total_q) / unit_tokens + s;
    }
    const unsigned hits = __ballot_sync(0xffffffffu, s < hi && first <= unit);
    if (!hits) return u;                       // in front of the first sequence
    const int l = 31 - __clz(hits);
    if (stride == 1) {
      u.q = tra_clamp_range(__shfl_sync(0xffffffffu, q0, l), __shfl_sync(0xffffffffu, q1, l), p.total_q, p.max_q, p.status);
      u.k = tra_clamp_range(__shfl_sync(0xffffffffu, k0, l), __shfl_sync(0xffffffffu, k1, l), p.total_k, p.max_k, p.status);
      u.index = unit - __shfl_sync(0xffffffffu, first, l);
      u.count = ((by_keys ? u.k.len : u.q.len) + unit_tokens - 1) / unit_tokens;
      if (u.index < u.count) u.seq = lo + l;
      return u;
    }
    hi = min(lo + (l + 1) * stride, hi);
    lo += l * stride;
  }
}

// Backward with a window: the first keys are seen by all queries behind them, the others by a window's.  So that their tiles do not
// walk on when all others are done, the queries of a sequence of more than sink_steps streamed tiles are cut into units of that many, whose
// sums of the first keys' gradients go to `sink_part` and are added by a kernel of their own, in order.  Unit c of a sequence from token b on has
// slot 2 floor(b / unit) + c, unit in tokens: a sequence longer than a unit ends in front of the next one's slots, and there are at most
// 2 floor(total_q / unit) + 2, however many sequences there are.
__device__ __forceinline__ int tra_sink_unit_tokens(const tra_packed_launch& p) { return p.sink_steps * p.stream_tokens; }

// The unit of a slot (seq = -1: none).  One warp calls it; every lane gets the result.
__device__ __forceinline__ tra_unit tra_find_sink_unit(const tra_packed_launch& p, int slot) {
  const int lane = threadIdx.x & 31, unit = tra_sink_unit_tokens(p);
  tra_unit u = {-1, 0, 1, {0, 0}, {0, 0}};
  int lo = 0, hi = p.n_seq;                    // the last sequence whose first slot is not behind this one
  while (hi - lo > 1) {
    const int stride = (hi - lo + 31) / 32, s = lo + lane * stride;
    const bool in = s < hi && 2 * (min(max(p.cu_q[s], 0), p.total_q) / unit) <= slot;
    const unsigned hits = __ballot_sync(0xffffffffu, in);
    if (!hits) return u;
    const int l = 31 - __clz(hits);
    hi = min(lo + (l + 1) * stride, hi);
    lo += l * stride;
  }
  u.q = tra_clamp_range(p.cu_q[lo], p.cu_q[lo + 1], p.total_q, p.max_q, p.status);
  u.k = tra_clamp_range(p.k_begin[lo], p.k_end[lo], p.total_k, p.max_k, p.status);
  u.index = slot - 2 * (u.q.begin / unit);
  u.count = (u.q.len + unit - 1) / unit;
  if (u.q.len > unit && u.index >= 0 && u.index < u.count) u.seq = lo;
  return u;
}

}  // namespace
#endif
