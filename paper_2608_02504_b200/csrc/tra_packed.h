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
  int causal, splits, n_units;               // n_units: query-tile pairs (forward) or key / query tiles (backward) launched
  float sm_scale;
  int* status;
};

struct tra_packed_ctx {
  const tra_packed_t* h;
  cudaStream_t stream;
};

int tra_packed_fwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_fwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_d128(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_bwd_d64(const tra_packed_ctx& c, const tra_packed_launch& a);
int tra_packed_rows(const tra_packed_ctx& c, const tra_packed_launch& a, int chunk, bool clustered);

#ifdef __CUDACC__
namespace {

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

}  // namespace
#endif
