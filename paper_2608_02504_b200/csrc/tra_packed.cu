// Packed attention: handle, argument checks, the choice of the launch, the join of split launches.
#include <string.h>

#include <new>

#include "tra_cache4.h"
#include "tra_packed_ptx.cuh"

namespace {

constexpr int kMaxSplits = 256;       // parts of a split launch

// O = sum_s w_s O_s, w_s = 2^(lse2_s - lse2), lse2 = log2 sum_s 2^lse2_s over the parts of a split launch; lse from the
// unrounded sums in the same way.  kWarps warps per (token, head): first the weights, all parts' logarithms read at once and
// kept by the lanes, then every warp adds its parts, four loads in flight.  Four warps per row where there are few rows (the
// serial loads count), one where there are many (12,000 rows of two parts: 42 us a call with a block each, 29 with a warp each).
template <typename T, int D, int kWarps>
__global__ void __launch_bounds__(128) tra_packed_join_kernel(const __grid_constant__ tra_packed_launch p) {
  constexpr int kPer = D / 32, kLogs = kMaxSplits / 32;
  __shared__ __align__(16) float s_o[kWarps > 1 ? kWarps : 1][kWarps > 1 ? D : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long stride = (long long)p.total_q * p.heads;
  const long long row = kWarps > 1 ? blockIdx.x : (long long)blockIdx.x * 4 + warp;
  wait_last_launch();
  if (row >= stride) return;
  const int tok = (int)(row / p.heads), head = (int)(row - (long long)tok * p.heads);
  // rows in front of the first and behind the last sequence stay as they are
  if (tok < p.cu_q[0] || tok >= p.cu_q[p.n_seq]) return;
  float v[kLogs], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kLogs; ++i) {
    const int s = i * 32 + lane;
    v[i] = s < p.splits ? p.part_lse2[s * stride + row] : -INFINITY;
    top = v[i] != v[i] ? v[i] : fmaxf(top, v[i]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, top, o);
    top = top != top ? top : other != other ? other : fmaxf(top, other);
  }
  const float ref = top == -INFINITY ? 0.f : top;        // no part holds a key: every weight is 0
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kLogs; ++i) {
    v[i] = ex2(v[i] - ref);                              // parts without a key: 0
    sum += v[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  float o[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) o[i] = 0.f;
  const int first = kWarps > 1 ? warp : 0;
  const float* src = p.part_o + row * D + lane * kPer;
#pragma unroll
  for (int k = 0; k < kLogs; ++k) {
    for (int s0 = k * 32 + first; s0 < min(p.splits, k * 32 + 32); s0 += 4 * kWarps) {
      float part[4][kPer], w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int s = s0 + j * kWarps;
        const float w_s = __shfl_sync(0xffffffffu, v[k], s & 31);
        w[j] = s < k * 32 + 32 ? w_s : 0.f;              // (past the last part the weights are 0)
#pragma unroll
        for (int i = 0; i < kPer; ++i) part[j][i] = 0.f;
        if (w[j] != 0.f) {                               // a part without a key has no row to read
          if constexpr (kPer == 4) {
            const float4 x = *reinterpret_cast<const float4*>(src + s * stride * D);
            part[j][0] = x.x, part[j][1] = x.y, part[j][2] = x.z, part[j][3] = x.w;
          } else {
            const float2 x = *reinterpret_cast<const float2*>(src + s * stride * D);
            part[j][0] = x.x, part[j][1] = x.y;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] = fmaf(w[j], part[j][i], o[i]);
    }
  }
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  T* dst = (T*)p.o + tok * p.o_stride[0] + head * p.o_stride[1];
  if constexpr (kWarps > 1) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) s_o[warp][lane * kPer + i] = o[i];
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        o[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) o[i] += s_o[w][lane * kPer + i];
      }
    }
  }
  if (kWarps == 1 || warp == 0) {
    uint32_t y[kPer / 2], rest[kPer / 2];
#pragma unroll
    for (int i = 0; i < kPer / 2; ++i) {
      y[i] = pack_pair<T>(o[2 * i] * inv, o[2 * i + 1] * inv);
      rest[i] = rest_pair<T>(o[2 * i] * inv, o[2 * i + 1] * inv, y[i]);
    }
    T* dst_rest = p.o_rest ? (T*)p.o_rest + row * D : nullptr;
    if constexpr (kPer == 4) {
      reinterpret_cast<uint2*>(dst)[lane] = make_uint2(y[0], y[1]);
      if (dst_rest) reinterpret_cast<uint2*>(dst_rest)[lane] = make_uint2(rest[0], rest[1]);
    } else {
      reinterpret_cast<uint32_t*>(dst)[lane] = y[0];
      if (dst_rest) reinterpret_cast<uint32_t*>(dst_rest)[lane] = rest[0];
    }
  }
  if (p.lse && (kWarps == 1 || warp == kWarps - 1)) {
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < kLogs; ++i) {
      const int s = i * 32 + lane;
      if (s < p.splits) total += ex2(p.part_exact[s * stride + row] - ref);
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) total += __shfl_xor_sync(0xffffffffu, total, k);
    if (lane == 0) p.lse[row] = total != 0.f ? (ref + log2f(total)) * kLn2 : -INFINITY;
  }
}

// How a call runs: rows = the kernel for few rows (at most 16 per sequence and key/value head), with `splits` parts
// of `chunk` keys, joined inside a thread-block cluster (clustered) or by the join kernel; else the 128-row tiles, with
// `splits` ranges of key blocks and the join kernel.
struct Choice {
  bool rows, clustered;
  int splits, chunk;
};

constexpr int kClusterMax = 8;        // the largest portable cluster

// Whether a window hides anything from sequences of up to max_k keys: the last position has all but `window` in front of it, and the first
// tokens stay.
bool window_hides(const tra_packed* h, int max_k) { return h->cfg.window > 0 && (long long)h->cfg.window + h->cfg.sinks < max_k; }

// Keys that a tile of `tokens` queries walks at most (tra_key_axis).
int longest_axis(const tra_packed* h, int max_k, int tokens) {
  if (!window_hides(h, max_k)) return max_k;
  const long long n = (long long)(h->cfg.sinks + 7) / 8 * 8 + h->cfg.window + tokens - 1;
  return n < max_k ? (int)n : max_k;
}

Choice choose(const tra_packed* h, int n_seq, int total_q, int max_q, int max_k) {
  const int group = h->cfg.heads / h->cfg.kv_heads;
  Choice c = {(long long)max_q * group <= 16, false, 1, 64};
  if (max_q == 0) return c;                                // nothing to attend to: the launch looks at the ranges alone
  max_k = longest_axis(h, max_k, c.rows ? max_q : 2 * (kTileM / group));
  if (c.rows) {
    // Two blocks fit an SM: as many parts as fill them once (a second wave costs its ramp-up: 1,024 blocks of 256 keys
    // took 41 us over a 32K cache of eight heads, 128 blocks of 2,048 keys 27 us), each of at least 128 keys.
    const long long units = (long long)n_seq * h->cfg.kv_heads;
    long long parts = 2ll * h->sm_count / units;
    const long long most = ((long long)max_k + 127) / 128;
    if (parts > most) parts = most;
    // More parts than a cluster holds pay off only over long caches, where the join's launch and workspace are small.
    if (parts > kClusterMax && max_k <= 512 * kClusterMax) parts = kClusterMax;
    if (parts > kClusterMax) {
      parts = h->sm_count / units;                          // one block per SM: fewer and longer parts for the join
      if (parts < kClusterMax) parts = kClusterMax;
    }
    if (parts > kMaxSplits) parts = kMaxSplits;
    // Enough sequences to fill the GPU: long caches in two parts all the same, since their lengths differ (64 caches of up to
    // 32K keys, eight heads: 640 us against 700 when the lengths are spread evenly, 1,175 against 1,162 when they are equal).
    if (parts <= 1) parts = max_k >= 8192 ? 2 : 1;
    c.chunk = (int)(((max_k + parts - 1) / parts + 63) / 64 * 64);
    if (c.chunk < 64) c.chunk = 64;
    c.splits = max_k > 0 ? (int)(((long long)max_k + c.chunk - 1) / c.chunk) : 1;
    c.clustered = c.splits > 1 && c.splits <= kClusterMax;
  } else {
    const int tile = kTileM / group;
    const long long blocks = ((max_q <= 2 * tile ? 0 : total_q / (2 * tile)) + n_seq) * (long long)h->cfg.kv_heads;
    const long long nb = (max_k + 127) / 128;
    long long s = h->sm_count / blocks;
    if (s > nb / 2) s = nb / 2;                            // parts of two key blocks at least
    if (s > kMaxSplits) s = kMaxSplits;
    c.splits = s > 1 ? (int)s : 1;
  }
  return c;
}

size_t workspace_of(const tra_packed* h, const Choice& c, int total_q) {
  return c.splits > 1 && !c.clustered ? sizeof(float) * (size_t)c.splits * total_q * h->cfg.heads * (h->cfg.head_dim + 2) : 0;
}

bool bad_sizes(const tra_packed* h, int n_seq, int total_q, int max_q, int max_k) {
  return !h || n_seq < 1 || total_q < 0 || max_q < 0 || max_k < 0 || max_q > total_q;
}

// [tokens, heads, d] behind strides, viewed with the channels innermost; box = 64 channels x box_heads x box_tokens.
int make_packed_map(CUtensorMap* map, const tra_packed* h, const void* base, const int64_t* stride, int heads, long long tokens,
                    int box_heads, int box_tokens, bool fp16 = false) {
  encode_tiled_fn enc = get_encode_tiled();
  if (!enc) return TRA_ERR_CUDA;
  cuuint64_t dims[3] = {(cuuint64_t)h->cfg.head_dim, (cuuint64_t)heads, (cuuint64_t)tokens};
  // the stride of a dimension of one entry is never used; a legal value keeps the encoder content
  cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)stride[1] * 2 : 128u, tokens > 1 ? (cuuint64_t)stride[0] * 2 : 128u};
  cuuint32_t box[3] = {64u, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
  cuuint32_t estr[3] = {1u, 1u, 1u};
  const CUresult r = enc(map, h->cfg.dtype == TRA_BF16 && !fp16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                         const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? TRA_OK : TRA_ERR_CUDA;
}

// The stride of a dimension of one entry is never used; the others are positive multiples of 16 bytes.
bool bad_tensor(const void* ptr, const int64_t* stride, long long tokens, int heads) {
  if (tokens == 0) return false;
  if (!ptr || ((uintptr_t)ptr & 15)) return true;
  const long long n[2] = {tokens, heads};
  for (int i = 0; i < 2; ++i)
    if (n[i] > 1 && (stride[i] < 8 || (stride[i] & 7) || stride[i] >= (1ll << 38))) return true;
  return false;
}

// Checks what the forward and the backward call share and fills the launch.
int begin_launch(const tra_packed* h, const tra_packed_args_t* a, tra_packed_launch* p, bool keys = true) {
  if (!h || !a || bad_sizes(h, a->n_seq, a->total_q, a->max_q, a->max_k) || a->total_k < 0 || a->max_k > a->total_k)
    return TRA_ERR_INVALID_ARG;
  if (!a->cu_q || !a->k_begin || !a->k_end || !(a->sm_scale > 0.f) || a->sm_scale > 1e30f) return TRA_ERR_INVALID_ARG;
  if (((uintptr_t)a->cu_q | (uintptr_t)a->k_begin | (uintptr_t)a->k_end | (uintptr_t)a->lse) & 3) return TRA_ERR_INVALID_ARG;
  if (((uintptr_t)a->o_rest & 15) || (a->o_rest && !a->lse)) return TRA_ERR_INVALID_ARG;
  if (a->total_q > (1 << 30) || a->total_k > (1 << 30)) return TRA_ERR_UNSUPPORTED;
  const int heads = h->cfg.heads, kv = h->cfg.kv_heads;
  if (bad_tensor(a->q, a->q_stride, a->total_q, heads) || bad_tensor(a->o, a->o_stride, a->total_q, heads) ||
      (keys && (bad_tensor(a->k, a->k_stride, a->total_k, kv) || bad_tensor(a->v, a->v_stride, a->total_k, kv))))
    return TRA_ERR_INVALID_ARG;
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return TRA_ERR_CUDA;
  if (device != h->device) return TRA_ERR_INVALID_ARG;
  memset(p, 0, sizeof(*p));
  p->q = a->q, p->k = a->k, p->v = a->v;
  p->lse = a->lse;
  p->o_rest = a->o_rest;
  for (int i = 0; i < 2; ++i) {
    p->q_stride[i] = a->q_stride[i];
    p->k_stride[i] = a->k_stride[i];
    p->v_stride[i] = a->v_stride[i];
    p->o_stride[i] = a->o_stride[i];
  }
  p->cu_q = a->cu_q, p->k_begin = a->k_begin, p->k_end = a->k_end;
  p->n_seq = a->n_seq, p->total_q = a->total_q, p->total_k = a->total_k, p->max_q = a->max_q, p->max_k = a->max_k;
  p->heads = h->cfg.heads, p->kv_heads = h->cfg.kv_heads, p->group = h->cfg.heads / h->cfg.kv_heads;
  p->tile_tokens = kTileM / p->group;
  p->order = !h->cfg.causal ? kOrderNone : window_hides(h, a->max_k) ? kOrderWindow : kOrderCausal;
  p->window = h->cfg.window, p->sinks = h->cfg.sinks, p->sink_rows = (h->cfg.sinks + 7) / 8 * 8;
  p->splits = 1;
  p->sm_scale = a->sm_scale;
  p->status = h->d_status;
  return TRA_OK;
}

// The maps of K and V, in boxes of `rows` keys and, for the tile where the first tokens end, of its two parts.
int make_key_maps(tra_packed_launch* p, const tra_packed* h, const void* k, const int64_t* ks, const void* v, const int64_t* vs, long long tokens,
                  int rows, int pieces = 1) {
  int rc;
  const int heads = p->kv_heads * (pieces == 2 ? 2 : 1);
  const bool fp16 = pieces == 0;
  if ((rc = make_packed_map(&p->map_k, h, k, ks, heads, tokens, 1, rows, fp16)) != TRA_OK) return rc;
  if ((rc = make_packed_map(&p->map_v, h, v, vs, heads, tokens, 1, rows, fp16)) != TRA_OK) return rc;
  const int first = p->order == kOrderWindow ? p->sink_rows % rows : 0;
  if (first == 0) return TRA_OK;
  if ((rc = make_packed_map(&p->map_k_first, h, k, ks, heads, tokens, 1, first, fp16)) != TRA_OK) return rc;
  if ((rc = make_packed_map(&p->map_v_first, h, v, vs, heads, tokens, 1, first, fp16)) != TRA_OK) return rc;
  if ((rc = make_packed_map(&p->map_k_rest, h, k, ks, heads, tokens, 1, rows - first, fp16)) != TRA_OK) return rc;
  return make_packed_map(&p->map_v_rest, h, v, vs, heads, tokens, 1, rows - first, fp16);
}

template <typename T, int D>
int launch_join_shape(const tra_packed* h, const tra_packed_launch& p, cudaStream_t stream) {
  const long long rows = (long long)p.total_q * p.heads;
  if (rows >= 16ll * h->sm_count)
    return tra_launch(tra_packed_join_kernel<T, D, 1>, dim3((unsigned)((rows + 3) / 4)), 128, 0, stream, true, 1, p);
  return tra_launch(tra_packed_join_kernel<T, D, 4>, dim3((unsigned)rows), 128, 0, stream, true, 1, p);
}
template <typename T>
int launch_join(const tra_packed* h, const tra_packed_launch& p, cudaStream_t stream) {
  return h->cfg.head_dim == 128 ? launch_join_shape<T, 128>(h, p, stream) : launch_join_shape<T, 64>(h, p, stream);
}

}  // namespace

int tra_packed_join(const tra_packed_ctx& c, const tra_packed_launch& p) {
  return c.h->cfg.dtype == TRA_BF16 ? launch_join<__nv_bfloat16>(c.h, p, c.stream) : launch_join<__half>(c.h, p, c.stream);
}
int tra_packed_begin(const tra_packed_t* h, const tra_packed_args_t* a, bool keys, tra_packed_launch* p) { return begin_launch(h, a, p, keys); }
int tra_packed_longest_axis(const tra_packed_t* h, int max_k, int tokens) { return longest_axis(h, max_k, tokens); }

extern "C" int tra_packed_create(tra_packed_t** out, const tra_packed_config_t* cfg) {
  if (!out || !cfg) return TRA_ERR_INVALID_ARG;
  *out = nullptr;
  if (cfg->heads < 1 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads) return TRA_ERR_INVALID_ARG;
  if (cfg->dtype != TRA_BF16 && cfg->dtype != TRA_FP16) return TRA_ERR_INVALID_ARG;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return TRA_ERR_UNSUPPORTED;
  if (cfg->window < 0 || cfg->sinks < 0 || (cfg->sinks > 0 && cfg->window == 0)) return TRA_ERR_INVALID_ARG;
  if (cfg->window > 0 && !cfg->causal) return TRA_ERR_UNSUPPORTED;
  if (cfg->window > (1 << 30) || cfg->sinks > (1 << 30)) return TRA_ERR_UNSUPPORTED;
  if (cfg->heads > 4096 || cfg->heads / cfg->kv_heads > kTileM) return TRA_ERR_UNSUPPORTED;
  tra_packed* h = new (std::nothrow) tra_packed;
  if (!h) return TRA_ERR_CAPACITY;
  memset(h, 0, sizeof(*h));
  h->cfg = *cfg;
  h->cfg.causal = cfg->causal != 0;
  if (cudaGetDevice(&h->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess ||
      cudaMalloc(&h->d_status, sizeof(int)) != cudaSuccess || cudaMemset(h->d_status, 0, sizeof(int)) != cudaSuccess ||
      cudaStreamSynchronize(nullptr) != cudaSuccess) {
    cudaFree(h->d_status);
    delete h;
    return TRA_ERR_CUDA;
  }
  *out = h;
  return TRA_OK;
}

extern "C" int tra_packed_destroy(tra_packed_t* h) {
  if (!h) return TRA_ERR_INVALID_ARG;
  cudaFree(h->d_status);
  delete h;
  return TRA_OK;
}

extern "C" int tra_packed_status(tra_packed_t* h, void* stream_) {
  if (!h) return TRA_ERR_INVALID_ARG;
  cudaStream_t stream = (cudaStream_t)stream_;
  int code = 0;
  TRA_CUDA_CHECK(cudaMemcpyAsync(&code, h->d_status, sizeof(int), cudaMemcpyDeviceToHost, stream));
  TRA_CUDA_CHECK(cudaMemsetAsync(h->d_status, 0, sizeof(int), stream));
  TRA_CUDA_CHECK(cudaStreamSynchronize(stream));
  return code;
}

extern "C" size_t tra_packed_attn_workspace_bytes(const tra_packed_t* h, int n_seq, int total_q, int max_q, int max_k) {
  if (bad_sizes(h, n_seq, total_q, max_q, max_k)) return 0;
  return workspace_of(h, choose(h, n_seq, total_q, max_q, max_k), total_q);
}

static int attend(const tra_packed_t* h, const tra_packed_args_t* a, void* workspace, size_t workspace_bytes, void* stream_, int pieces,
                  const float* q_mul = nullptr, const uint32_t* kv_top = nullptr) {
  tra_packed_launch p;
  int rc = begin_launch(h, a, &p);
  if (rc != TRA_OK) return rc;
  const tra_packed_ctx ctx = {h, (cudaStream_t)stream_};
  p.o = a->o;
  const Choice c = choose(h, a->n_seq, a->total_q, a->max_q, a->max_k);
  p.splits = c.splits;
  const bool join = c.splits > 1 && !c.clustered;
  if (join) {
    if ((long long)a->total_q * p.heads > 0x7fffffffll) return TRA_ERR_UNSUPPORTED;
    if (!workspace || ((uintptr_t)workspace & 15)) return TRA_ERR_INVALID_ARG;
    if (workspace_bytes < workspace_of(h, c, a->total_q)) return TRA_ERR_CAPACITY;
    const long long rows = (long long)c.splits * a->total_q * p.heads;
    p.part_o = (float*)workspace;
    p.part_lse2 = p.part_o + rows * h->cfg.head_dim;
    p.part_exact = a->lse ? p.part_lse2 + rows : nullptr;
  }
  if (a->max_q == 0) return tra_packed_rows(ctx, p, c.chunk, false);       // (no row, no tile: the maps stay empty)
  const int key_box = c.rows ? 64 : 128;
  // without keys no tile is loaded; the maps then describe the queries
  const void *kk = a->total_k > 0 ? a->k : a->q, *vv = a->total_k > 0 ? a->v : a->q;
  const int64_t *ks = a->total_k > 0 ? a->k_stride : a->q_stride, *vs = a->total_k > 0 ? a->v_stride : a->q_stride;
  const long long tk = a->total_k > 0 ? a->total_k : a->total_q;
  if ((rc = make_key_maps(&p, h, kk, ks, vv, vs, tk, key_box, pieces)) != TRA_OK) return rc;
  if (c.rows) {
    rc = tra_packed_rows(ctx, p, c.chunk, c.clustered);
  } else {
    if ((rc = make_packed_map(&p.map_q, h, a->q, a->q_stride, p.heads, a->total_q, p.group, p.tile_tokens, pieces == 0)) != TRA_OK) return rc;
    p.n_units = (a->max_q <= 2 * p.tile_tokens ? 0 : a->total_q / (2 * p.tile_tokens)) + a->n_seq;
    if (pieces != 1) {
      if (p.order != kOrderWindow) p.window = 1 << 30, p.sinks = p.sink_rows = 0;
      p.q_mul = q_mul, p.kv_top = kv_top;
      if (pieces == 2)
        rc = h->cfg.head_dim == 128 ? tra_packed_fwd_pieces_d128(ctx, p) : tra_packed_fwd_pieces_d64(ctx, p);
      else
        rc = h->cfg.head_dim == 128 ? tra_packed_fwd_fp16_d128(ctx, p) : tra_packed_fwd_fp16_d64(ctx, p);
    } else if (p.order == kOrderWindow)
      rc = h->cfg.head_dim == 128 ? tra_packed_fwd_window_d128(ctx, p) : tra_packed_fwd_window_d64(ctx, p);
    else
      rc = h->cfg.head_dim == 128 ? tra_packed_fwd_d128(ctx, p) : tra_packed_fwd_d64(ctx, p);
  }
  if (rc != TRA_OK || !join) return rc;
  return tra_packed_join(ctx, p);
}

extern "C" int tra_packed_attn(const tra_packed_t* h, const tra_packed_args_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  return attend(h, a, workspace, workspace_bytes, stream, 1);
}
int tra_packed_attn_read_back(const tra_packed_t* h, const tra_packed_args_t* a, const float* q_mul, const uint32_t* kv_top, void* workspace,
                              size_t workspace_bytes, void* stream) {
  return attend(h, a, workspace, workspace_bytes, stream, h->cfg.dtype == TRA_BF16 ? 0 : 2, q_mul, kv_top);
}

namespace {

// Streamed tiles of 64 rows let two blocks share an SM where head_dim leaves the room; not where they would hold less than
// nine tenths of the rows of 128 (groups of 22 heads and more that do not divide 64).
int backward_stream_rows(const tra_packed* h) {
  const int group = h->cfg.heads / h->cfg.kv_heads;
  return h->cfg.head_dim == 64 && 20 * (64 / group) >= 9 * (kTileM / group) ? 64 : 128;
}

// Units of the first keys' gradients (tra_find_sink_unit): as many streamed tiles as another key tile walks, 16 at least, or a 32nd of all
// queries, or more where the sums would take over a quarter of a gigabyte.  slots = 0: not cut.
struct SinkPlan {
  int steps;
  long long slots;
};
SinkPlan sink_plan(const tra_packed* h, int total_q) {
  SinkPlan s = {0, 0};
  if (h->cfg.window == 0 || h->cfg.sinks == 0) return s;
  const long long tokens = backward_stream_rows(h) / (h->cfg.heads / h->cfg.kv_heads);
  long long steps = ((long long)h->cfg.window + kTileM) / tokens;
  if (steps > 64) steps = 64;
  if (steps < 16) steps = 16;
  if (steps < total_q / (32 * tokens)) steps = total_q / (32 * tokens);
  // not where one block that walks all queries is done before the others: these walk a window each, and the dQ blocks about as much
  const long long tiles = (total_q + kTileM - 1) / kTileM, walk = total_q / tokens, window = h->cfg.window < total_q ? h->cfg.window : total_q;
  const long long sink_tiles = ((h->cfg.sinks < total_q ? h->cfg.sinks : total_q) + kTileM - 1) / kTileM;
  const long long blocks = h->cfg.head_dim == 64 ? 2 : 1;
  if (10 * walk * blocks * h->sm_count < 6 * h->cfg.kv_heads * (2 * tiles * (window + kTileM) / tokens + sink_tiles * walk)) return s;
  for (; steps * tokens < total_q; steps *= 2) {
    const long long slots = 2 * (total_q / (steps * tokens)) + 2;
    if (slots * h->cfg.kv_heads * h->cfg.sinks > (256ll << 20) / (8 * h->cfg.head_dim)) continue;
    s.steps = (int)steps, s.slots = slots;
    break;
  }
  return s;
}
// Whether no key tile walks streamed tiles of more than 384 rows (one of the first tokens may): all queries', or those that a window's length and
// the tile's cover.
bool few_steps(const tra_packed_launch& p) {
  const long long all = ((long long)p.max_q + p.stream_tokens - 1) / p.stream_tokens, seen = ((long long)p.window + kTileM - 2) / p.stream_tokens + 2;
  return (all < seen ? all : seen) * p.stream_rows <= 3 * kTileM;
}
size_t round16(size_t n) { return (n + 15) / 16 * 16; }
// delta, and (fp16) the largest norms behind it
size_t delta_bytes(const tra_packed* h, int total_q) {
  return sizeof(float) * ((size_t)total_q * h->cfg.heads + (h->cfg.dtype == TRA_FP16 ? 2 * (size_t)h->cfg.kv_heads : 0));
}

}  // namespace

extern "C" size_t tra_packed_attn_backward_workspace_bytes(const tra_packed_t* h, int total_q) {
  if (!h || total_q <= 0) return 0;
  const size_t n = delta_bytes(h, total_q), slots = (size_t)sink_plan(h, total_q).slots;
  return slots == 0 ? n : round16(n) + sizeof(float) * slots * h->cfg.kv_heads * (size_t)h->cfg.sinks * 2 * h->cfg.head_dim;
}

extern "C" int tra_packed_attn_backward(const tra_packed_t* h, const tra_packed_args_t* a, const tra_packed_grads_t* g,
                                        void* workspace, size_t workspace_bytes, void* stream_) {
  tra_packed_launch p;
  int rc = begin_launch(h, a, &p);
  if (rc != TRA_OK) return rc;
  // packed keys only: a key that two sequences share would have two gradients
  if (!g || a->k_end != a->k_begin + 1 || (!a->lse && a->total_q > 0)) return TRA_ERR_INVALID_ARG;
  if (bad_tensor(g->d_o, g->do_stride, a->total_q, p.heads) || bad_tensor(g->dq, g->dq_stride, a->total_q, p.heads) ||
      bad_tensor(g->dk, g->dk_stride, a->total_k, p.kv_heads) || bad_tensor(g->dv, g->dv_stride, a->total_k, p.kv_heads))
    return TRA_ERR_INVALID_ARG;
  if ((long long)a->total_q * p.heads > 0x7fffffffll) return TRA_ERR_UNSUPPORTED;
  const tra_packed_ctx ctx = {h, (cudaStream_t)stream_};
  if (a->max_q == 0 && a->max_k == 0) return tra_packed_rows(ctx, p, 64, false);      // nothing to do: the ranges are looked at
  if (a->total_q > 0) {
    if (!workspace || ((uintptr_t)workspace & 15)) return TRA_ERR_INVALID_ARG;
    if (workspace_bytes < tra_packed_attn_backward_workspace_bytes(h, a->total_q)) return TRA_ERR_CAPACITY;
  }
  p.delta = (float*)workspace;
  p.norms = (uint32_t*)workspace + (long long)a->total_q * p.heads;
  p.o_in = a->o, p.d_o = g->d_o;
  p.dq = g->dq, p.dk = g->dk, p.dv = g->dv;
  for (int i = 0; i < 2; ++i) {
    p.do_stride[i] = g->do_stride[i];
    p.dq_stride[i] = g->dq_stride[i];
    p.dk_stride[i] = g->dk_stride[i];
    p.dv_stride[i] = g->dv_stride[i];
  }
  // Sequences that the window hides nothing of take the window's kernels too, whose dq has second pieces of dS (dq_tiles_block): 1.2 times the error of
  // rounding dq alone, against 1.51 to 1.53 at d 64, where it costs nothing over long sequences (four of 8,190 tokens: 1.89 ms, causal order 1.90), and
  // up to 1.58 over a few keys.  Not long ones at d 128 (40 / 8 heads, the window's kernels and the others: four of
  // 4,096 tokens 2.40 ms and 2.20, eight of 2,048 1.43 and 1.27, ten of 1,536 1.10 and 1.02, 16 of 1,024 0.87 and 0.84, 32 of 512 0.58 and 0.62, 54 of 300 0.45 and 0.51;
  // 16 heads: 1,035 us and 939, 641 and 565, 505 and 441, 412 and 374, 300 and 297, 361 and 355).  (Precision sets the border: rows of few keys need it.)
  if (h->cfg.window > 0 && p.order == kOrderCausal && (h->cfg.head_dim == 64 || p.max_k <= 1024))
    p.order = kOrderWindow, p.window = 1 << 30, p.sinks = p.sink_rows = 0;
  p.stream_rows = backward_stream_rows(h);
  p.stream_tokens = p.stream_rows / p.group;
  // dQ blocks of about 24 steps, as long as there are three for every SM (times two where two share one)
  const long long most = (long long)p.sink_rows + p.window + p.tile_tokens, walked = (most < a->max_k ? most : a->max_k) / p.stream_rows + 1;
  const long long tiles = ((long long)a->total_q / p.tile_tokens + 1) * p.kv_heads, three = 3ll * h->sm_count * (p.stream_rows == 64 ? 2 : 1);
  p.dq_tiles = (int)(walked >= 24 ? 1 : 24 / walked);
  while (p.dq_tiles > 1 && tiles / p.dq_tiles < three) --p.dq_tiles;
  const SinkPlan sinks = sink_plan(h, a->total_q);
  if (p.order == kOrderWindow && p.sinks > 0 && sinks.slots > 0) {
    p.sink_steps = sinks.steps, p.sink_slots = (int)sinks.slots;
    p.sink_part = (float*)((uint8_t*)workspace + round16(delta_bytes(h, a->total_q)));
  }
  // a side without tokens is never loaded; its maps then describe the other side
  const bool q = a->total_q > 0, k = a->total_k > 0;
  const void *qq = q ? a->q : a->k, *oo = q ? g->d_o : a->k, *kk = k ? a->k : a->q, *vv = k ? a->v : a->q;
  const int64_t *qs = q ? a->q_stride : a->k_stride, *os = q ? g->do_stride : a->k_stride;
  const int64_t *ks = k ? a->k_stride : a->q_stride, *vs = k ? a->v_stride : a->q_stride;
  const int q_heads = q ? p.heads : p.kv_heads, q_box = q ? p.group : 1, nq = q ? a->total_q : a->total_k, nk = k ? a->total_k : a->total_q;
  if ((rc = make_packed_map(&p.map_q, h, qq, qs, q_heads, nq, q_box, p.tile_tokens)) != TRA_OK) return rc;
  if ((rc = make_packed_map(&p.map_do, h, oo, os, q_heads, nq, q_box, p.tile_tokens)) != TRA_OK) return rc;
  if ((rc = make_key_maps(&p, h, kk, ks, vv, vs, nk, p.stream_rows)) != TRA_OK) return rc;
  p.map_q_stream = p.map_q, p.map_do_stream = p.map_do;
  if (p.stream_rows != kTileM) {
    if ((rc = make_packed_map(&p.map_q_stream, h, qq, qs, q_heads, nq, q_box, p.stream_tokens)) != TRA_OK) return rc;
    if ((rc = make_packed_map(&p.map_do_stream, h, oo, os, q_heads, nq, q_box, p.stream_tokens)) != TRA_OK) return rc;
  }
  if (p.order == kOrderWindow) {
    if (few_steps(p)) return h->cfg.head_dim == 128 ? tra_packed_bwd_few_d128(ctx, p) : tra_packed_bwd_few_d64(ctx, p);
    return h->cfg.head_dim == 128 ? tra_packed_bwd_window_d128(ctx, p) : tra_packed_bwd_window_d64(ctx, p);
  }
  return h->cfg.head_dim == 128 ? tra_packed_bwd_d128(ctx, p) : tra_packed_bwd_d64(ctx, p);
}
