// Penalties, biases and allowed-token masks on the logits of the mask rows, alone (wedlm_logits_adjust) or inside the
// confidence pass (wedlm_confidence_commit_adjusted), and the upkeep of the token histories that the penalties read.
//
// Work is cut like the plain confidence pass: (row, chunk) items, here one warp per item.
#include <math_constants.h>

#include "adjust.cuh"

namespace wedlm {
namespace {

constexpr int kWarpsPerBlock = 4;
constexpr int kNoToken = 0x7fffffff;

// Running softmax statistics of some tokens: m = reference (their maximum so far), s = sum 2^d, t = sum d 2^d with
// d = (x - m) log2(e); the best token and its value beside them.
struct Stats {
  float m, s, t;
  float best;
  int token;
  __device__ void clear() { m = -CUDART_INF_F; s = 0.f; t = 0.f; best = -CUDART_INF_F; token = kNoToken; }
  // tokens come in ascending order, so a strict comparison keeps the lowest of equal ones
  __device__ void add(float x, int v) {
    if (x > best) { best = x; token = v; }
    if (!(x > -CUDART_INF_F)) return;
    constexpr float kLog2e = 1.4426950408889634f;
    if (x > m) {
      const float d = (m - x) * kLog2e, f = exp2f(d);
      t = f > 0.f ? (t + d * s) * f : 0.f;      // d may be -inf where f is 0
      s *= f;
      m = x;
    }
    const float d = fmaxf((x - m) * kLog2e, -200.f), e = exp2f(d);
    s += e;
    t = fmaf(d, e, t);
  }
};

// Joins the lanes' statistics; the same result in every lane.  t comes back in units of the natural logarithm.
__device__ __forceinline__ float4 join_lanes(const Stats& z) {
  constexpr float kLog2e = 1.4426950408889634f;
  float best = z.best;
  int token = z.token;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float ob = __shfl_xor_sync(0xffffffffu, best, o);
    const int ot = __shfl_xor_sync(0xffffffffu, token, o);
    if (ob > best || (ob == best && ot < token)) { best = ob; token = ot; }
  }
  float s = 0.f, t = 0.f;
  if (z.s > 0.f) {
    const float d = (z.m - best) * kLog2e, f = exp2f(d);
    s = z.s * f;
    t = f > 0.f ? (z.t + d * z.s) * f : 0.f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  return make_float4(best, s, t * 0.6931471805599453f, __int_as_float(best > -CUDART_INF_F ? token : kNoToken));
}

// The item of this warp, or false when it has none (past the end, or the row is no active mask).
__device__ __forceinline__ bool warp_item(int W, int n_chunks, long long n_items, const int32_t* n_filled,
                                          const int32_t* window_len, int& row, int& b, int& chunk) {
  const long long item = (long long)blockIdx.x * kWarpsPerBlock + (threadIdx.x >> 5);
  if (item >= n_items) return false;
  row = (int)(item / n_chunks);
  chunk = (int)(item - (long long)row * n_chunks);
  b = row / W;
  const int i = row - b * W;
  const int L = window_len ? min(max(window_len[b], 0), W) : W;
  return i >= n_filled[b] && i < L;
}

template <typename T>
__global__ void __launch_bounds__(32 * kWarpsPerBlock)
conf_adjusted_kernel(AdjustView a, int n_chunks, int chunk_len, long long n_items, const T* __restrict__ logits,
                     const int32_t* __restrict__ perm, const int32_t* __restrict__ n_filled,
                     const int32_t* __restrict__ window_len, float4* __restrict__ part, int32_t* status) {
  int row, b, chunk;
  if (!warp_item(a.W, n_chunks, n_items, n_filled, window_len, row, b, chunk)) return;
  const int lane = threadIdx.x & 31;
  const RowRules r = row_rules(a, b, min(max(perm[row], 0), a.W - 1), chunk == 0 && lane == 0 ? status : nullptr);
  const T* src = logits + (size_t)row * a.V;
  const int end = min(a.V, (chunk + 1) * chunk_len);
  Stats z;
  z.clear();
  for (int v = chunk * chunk_len + lane; v < end; v += 32) z.add(adjusted_logit(src, v, r), v);
  const float4 p = join_lanes(z);
  if (lane == 0) part[(size_t)row * n_chunks + chunk] = p;
}

template <typename T>
__global__ void __launch_bounds__(32 * kWarpsPerBlock)
logits_adjust_kernel(AdjustView a, int n_chunks, int chunk_len, long long n_items, const T* logits, T* out,
                     const int32_t* __restrict__ perm, const int32_t* __restrict__ n_filled,
                     const int32_t* __restrict__ window_len, int32_t* status) {
  int row, b, chunk;
  if (!warp_item(a.W, n_chunks, n_items, n_filled, window_len, row, b, chunk)) return;
  const int lane = threadIdx.x & 31;
  const RowRules r = row_rules(a, b, min(max(perm[row], 0), a.W - 1), chunk == 0 && lane == 0 ? status : nullptr);
  const T* src = logits + (size_t)row * a.V;
  T* dst = out + (size_t)row * a.V;
  const int end = min(a.V, (chunk + 1) * chunk_len);
  for (int v = chunk * chunk_len + lane; v < end; v += 32) st_from_float(dst, (size_t)v, adjusted_logit(src, v, r));
}

// One thread per token.  Integer atomics only: the result does not depend on their order.
__global__ void __launch_bounds__(256)
history_add_kernel(AdjustView a, int length, int blocks_per_seq, const int32_t* __restrict__ tokens,
                   const int32_t* __restrict__ count, int in_prompt, int32_t* status) {
  const int b = blockIdx.x / blocks_per_seq;
  const int n = min(max(count[b], 0), length);
  const int i = (blockIdx.x - b * blocks_per_seq) * 256 + threadIdx.x;
  if (i >= n) return;
  const int v = tokens[(size_t)b * length + i];
  if (v < 0 || v >= a.V) {
    if (status) atomicOr(status, WEDLM_STATUS_BAD_TOKEN);
    return;
  }
  if (in_prompt) {
    atomicOr(&a.record[(size_t)b * a.V + v].x, 1);
    atomicOr(a.bits + (size_t)b * a.words + (v >> 5), 1u << (v & 31));
  } else {
    count_token(a, b, v);
  }
}

// One block per sequence.  Of equal ids the one listed last counts.
__global__ void __launch_bounds__(256)
history_bias_kernel(AdjustView a, int n_ids, const int32_t* __restrict__ ids, const float* __restrict__ values,
                    int32_t* status) {
  extern __shared__ int32_t id_s[];
  const int b = blockIdx.x;
  for (int k = threadIdx.x; k < n_ids; k += 256) id_s[k] = ids[(size_t)b * n_ids + k];
  __syncthreads();
  for (int k = threadIdx.x; k < n_ids; k += 256) {
    const int v = id_s[k];
    if (v < 0) continue;                                    // unused entry
    if (v >= a.V) {
      if (status) atomicOr(status, WEDLM_STATUS_BAD_TOKEN);
      continue;
    }
    bool last = true;
    for (int o = k + 1; o < n_ids && last; ++o) last = id_s[o] != v;
    if (!last) continue;
    a.record[(size_t)b * a.V + v].y = __float_as_int(values[(size_t)b * n_ids + k]);
    atomicOr(a.bits + (size_t)b * a.words + (v >> 5), 1u << (v & 31));
  }
}

}  // namespace

int launch_conf_adjusted_pass1(const Shape& s, const AdjustView& a, int n_chunks, int chunk, const void* logits,
                               const int32_t* perm, const int32_t* n_filled, const int32_t* window_len, void* partials,
                               int32_t* status, cudaStream_t st) {
  const long long items = (long long)s.B * s.W * n_chunks;
  const long long blocks = (items + kWarpsPerBlock - 1) / kWarpsPerBlock;
  if (blocks > 0x7fffffffLL) return WEDLM_ERR_UNSUPPORTED;
  float4* part = reinterpret_cast<float4*>(partials);
  if (s.dtype == WEDLM_DTYPE_BF16)
    conf_adjusted_kernel<<<(unsigned)blocks, 32 * kWarpsPerBlock, 0, st>>>(a, n_chunks, chunk, items, (const __nv_bfloat16*)logits,
                                                                           perm, n_filled, window_len, part, status);
  else
    conf_adjusted_kernel<<<(unsigned)blocks, 32 * kWarpsPerBlock, 0, st>>>(a, n_chunks, chunk, items, (const float*)logits, perm,
                                                                           n_filled, window_len, part, status);
  count_launch();
  return cuda_ok(cudaGetLastError());
}

int launch_logits_adjust(const Shape& s, const AdjustView& a, const void* logits, void* out, const int32_t* perm,
                         const int32_t* n_filled, const int32_t* window_len, int32_t* status, cudaStream_t st) {
  constexpr int chunk = 8192;
  const int n_chunks = (s.V + chunk - 1) / chunk;
  const long long items = (long long)s.B * s.W * n_chunks;
  const long long blocks = (items + kWarpsPerBlock - 1) / kWarpsPerBlock;
  if (blocks > 0x7fffffffLL) return WEDLM_ERR_UNSUPPORTED;
  if (s.dtype == WEDLM_DTYPE_BF16)
    logits_adjust_kernel<<<(unsigned)blocks, 32 * kWarpsPerBlock, 0, st>>>(a, n_chunks, chunk, items, (const __nv_bfloat16*)logits,
                                                                           (__nv_bfloat16*)out, perm, n_filled, window_len, status);
  else
    logits_adjust_kernel<<<(unsigned)blocks, 32 * kWarpsPerBlock, 0, st>>>(a, n_chunks, chunk, items, (const float*)logits,
                                                                           (float*)out, perm, n_filled, window_len, status);
  count_launch();
  return cuda_ok(cudaGetLastError());
}

int launch_history_add(const Shape& s, const AdjustView& a, int length, const int32_t* tokens, const int32_t* count,
                       int in_prompt, int32_t* status, cudaStream_t st) {
  const int per_seq = (length + 255) / 256;
  const long long blocks = (long long)s.B * per_seq;
  if (blocks > 0x7fffffffLL) return WEDLM_ERR_UNSUPPORTED;
  history_add_kernel<<<(unsigned)blocks, 256, 0, st>>>(a, length, per_seq, tokens, count, in_prompt, status);
  count_launch();
  return cuda_ok(cudaGetLastError());
}

int launch_history_bias(const Shape& s, const AdjustView& a, int n_ids, const int32_t* ids, const float* values,
                        int32_t* status, cudaStream_t st) {
  history_bias_kernel<<<s.B, 256, (size_t)n_ids * sizeof(int32_t), st>>>(a, n_ids, ids, values, status);
  count_launch();
  return cuda_ok(cudaGetLastError());
}

}  // namespace wedlm
