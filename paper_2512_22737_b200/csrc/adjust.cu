// Penalties, biases and allowed-token masks on the logits of the mask rows, alone (wedlm_logits_adjust) or inside the
// confidence pass (wedlm_confidence_commit_adjusted), and the upkeep of the token histories that the penalties read.
//
// Work is cut like the plain confidence pass: (row, chunk) items, a block per item in the confidence pass, a warp per item where the
// rules are applied alone.
#include <math_constants.h>

#include <type_traits>

#include "adjust.cuh"
#include "tc_ptx.cuh"

namespace wedlm {
namespace {

using namespace ptx;

constexpr int kWarpsPerBlock = 4;
constexpr int kNoToken = 0x7fffffff;
constexpr float kLog2e = 1.4426950408889634f;

// Running softmax statistics of some tokens: m = reference (their maximum so far), s = sum 2^d, t = sum d 2^d with
// d = (x - m) log2(e); the best token and its value beside them.
struct Stats {
  float m, s, t;
  float best;
  int token;
  __device__ void clear() { m = -CUDART_INF_F; s = 0.f; t = 0.f; best = -CUDART_INF_F; token = kNoToken; }
  __device__ void add(float x, int v) {
    if (x > best || (x == best && v < token)) { best = x; token = v; }
    if (!(x > -CUDART_INF_F)) return;
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

// ---------------------------------------------------------------------------------------------- confidence pass 1
// A token is either plain (allowed, no record) or touched (has a record) or excluded by the row's mask.
//
// touched_list_kernel lists the touched tokens of every (sequence, chunk), ascending, with their offsets: a few per hundred,
// but a third of the low ids of a long history.  conf_adjusted_kernel then takes (row, chunk) items, six blocks on an SM,
// each with a slot of 16 KB that its producer warp keeps filled by bulk copies.  The listed tokens are taken out of the slot
// one by one (their adjusted values join the sums, kFloor takes their place), the rest moves to registers, the slot is
// handed back, and the sums are formed.  Rows with a mask get its bits applied in registers, unless it allows only a few
// tokens of the chunk: those are gathered, and nothing else of it is read.
//
// Values at or below kFloor in the stream count as nothing.  A share of a row whose largest logit is not above kLow is
// computed again token by token, so that rows at the lowest value of the type are still the uniform rows that they are.
//
// Bound: the logits, 2 bytes each, once; measured 121 us for the 414 MB of the 1364 mask rows of a 64 x 32 window (151 936
// tokens, 5250 of them touched per sequence; 3.4 TB/s; 140 us with the lists and the commit), at 64 % of the issue slots: of 80 M
// instructions 27 M are the exponentials and sums of the plain tokens, the rest what the touched ones and the hand-overs cost.
// Under grammars the latency of the gathered items comes to that, and of the masks' words: 96 us for 48 x 32 rows, nine in ten
// masked, of which 480 are streamed (146 MB, 55 us: 2.7 TB/s) and 426 gathered (26 us).  Tried and slower: a warp per item with its own
// slot, or with its vectors masked in registers instead of taken out of the slot (145 us); lists made by every block
// (144 us); a warp of its own for the gathered items (150 us).
constexpr int kConfThreads = 128, kConfWarps = kConfThreads / 32;      // consumers of a block; one producer warp beside them
constexpr int kConfBlocksPerSM = 6;           // 4, 5, 7, 8: 140, 139, 142, 166 us where 6 takes 139 (64 x 32 rows of 151 936)
constexpr int kAdjustVecs = 8;                // vectors per lane of the kernel that applies the rules alone
constexpr uint32_t kChunkBytes = kConfThreads * 8 * 16;       // eight 16-byte vectors per thread
constexpr int kListMost = 4096;               // with more touched tokens the chunk has no list, and they are found by their bits
constexpr int kListNear = 1024;               // a list no longer than this comes to shared memory with its chunk
constexpr uint32_t kSeen = 0x8000u;           // flag of a listed token that the sequence has (not only a bias for it)
// Allowed tokens of a masked row's chunk that are gathered rather than streamed.  48 x 32 rows of 151 936 bf16 logits, nine in ten
// masked, every mask with so many tokens of each chunk: 4 gathered 75, streamed 106 us; 20: 89, 108; 41: 97, 108; 82: 107, 109;
// 123: 116, 109; 246: 130, 109; 983: 197, 110.  The border for such a batch lies near 90; with the mixed masks of a serving
// batch, 4 or 82 tokens in the narrow ones, both gathered take 96, the 82 streamed 99, both streamed 107.
constexpr int kGatherMost = 256;
constexpr float kFloor = -1.0e30f;
constexpr uint32_t kFloorBf16x2 = 0xF149F149u;
constexpr float kLow = -1.0e20f;

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t sel) {       // selector 8 + i replicates the sign of byte i
  uint32_t d;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(d) : "r"(a), "r"(sel));
  return d;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}

// 32 bits of a bitmap from any bit position on, possibly before its start; bits outside the bitmap are zero.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* __restrict__ bits, int pos, int words) {
  const int k = pos >> 5, sh = pos & 31;
  const uint32_t lo = k >= 0 && k < words ? bits[k] : 0u;
  if (sh == 0) return lo;
  return __funnelshift_r(lo, k + 1 >= 0 && k + 1 < words ? bits[k + 1] : 0u, sh);
}

__device__ __forceinline__ void consumer_sync() {     // the consumer threads only
  asm volatile("bar.sync 1, %0;" ::"n"(kConfThreads) : "memory");
}

// A thread's part of a chunk: the 16-byte vectors k * kConfThreads + tid, k < 8.
template <typename T> struct Part;
template <> struct Part<__nv_bfloat16> {
  static constexpr int VL = 8, kPairs = 32;
  uint32_t w[32];
  __device__ __forceinline__ void load(const uint8_t* stage, int tid) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint4 v = *reinterpret_cast<const uint4*>(stage + (k * kConfThreads + tid) * 16);
      w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
    }
  }
  // tokens whose bit is clear -> kFloor; on[k]: the bits of vector k
  __device__ __forceinline__ void mask(const uint32_t (&bits)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t on = bits[k];
      const uint32_t z0 = (on & 15u) * 0x10204080u, z1 = (on >> 4) * 0x10204080u;     // one bit to each byte's sign
      const uint32_t m[4] = {prmt(z0, 0x9988), prmt(z0, 0xBBAA), prmt(z1, 0x9988), prmt(z1, 0xBBAA)};
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * k + e] = (w[4 * k + e] & m[e]) | (kFloorBf16x2 & ~m[e]);
    }
  }
  uint32_t top[4];                            // maxima of the words i with i % 4 == 0, 1, 2, 3
  __device__ __forceinline__ float clamp_and_maximum() {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      w[i] = max_bf16x2(w[i], kFloorBf16x2);
      top[i & 3] = i < 4 ? w[i] : max_bf16x2(top[i & 3], w[i]);
    }
    const uint32_t m = max_bf16x2(max_bf16x2(top[0], top[1]), max_bf16x2(top[2], top[3]));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  // lowest token that holds m, which one of the thread's has; first: token 0 of the thread's first vector
  __device__ __forceinline__ int find(float m, int first) const {
    int at = kNoToken;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (__uint_as_float(top[q] << 16) == m || __uint_as_float(top[q] & 0xffff0000u) == m) {
#pragma unroll
        for (int k = 7; k >= 0; --k) {
          const int v = first + k * kConfThreads * VL + 2 * q;
          if (__uint_as_float(w[4 * k + q] & 0xffff0000u) == m) at = min(at, v + 1);
          if (__uint_as_float(w[4 * k + q] << 16) == m) at = min(at, v);
        }
      }
    return at;
  }
  __device__ __forceinline__ void pair(int i, float& lo, float& hi) const {
    lo = __uint_as_float(w[i] << 16);
    hi = __uint_as_float(w[i] & 0xffff0000u);
  }
};
template <> struct Part<float> {
  static constexpr int VL = 4, kPairs = 16;
  float x[32];
  __device__ __forceinline__ void load(const uint8_t* stage, int tid) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(stage + (k * kConfThreads + tid) * 16);
      x[4 * k] = v.x; x[4 * k + 1] = v.y; x[4 * k + 2] = v.z; x[4 * k + 3] = v.w;
    }
  }
  __device__ __forceinline__ void mask(const uint32_t (&bits)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t on = bits[k];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!((on >> e) & 1u)) x[4 * k + e] = kFloor;
    }
  }
  float top[4];                               // maxima of the values i with i % 4 == 0, 1, 2, 3
  __device__ __forceinline__ float clamp_and_maximum() {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      x[i] = fmaxf(x[i], kFloor);
      top[i & 3] = i < 4 ? x[i] : fmaxf(top[i & 3], x[i]);
    }
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  }
  __device__ __forceinline__ int find(float m, int first) const {
    int at = kNoToken;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (top[q] == m) {
#pragma unroll
        for (int k = 7; k >= 0; --k)
          if (x[4 * k + q] == m) at = min(at, first + k * kConfThreads * VL + q);
      }
    return at;
  }
  __device__ __forceinline__ void pair(int i, float& lo, float& hi) const { lo = x[2 * i]; hi = x[2 * i + 1]; }
};

// A lane's running sums relative to its largest logit m: r = m log2(e) as rounded, s = sum 2^d, t = sum d 2^d with
// d = x log2(e) - r (one fused operation, so that its error is relative to d).
struct Lane {
  float m, r, s, t;
  __device__ __forceinline__ void raise(float to) {
    const float r_new = to * kLog2e, d = r - r_new, f = ex2_approx(d);
    t = f > 0.f ? fmaf(d, s, t) * f : 0.f;
    s *= f;
    m = to;
    r = r_new;
  }
  __device__ __forceinline__ void add(float x) {
    if (x > m) raise(x);
    const float d = fmaxf(fmaf(x, kLog2e, -r), -200.f), e = ex2_approx(d);
    s += e;
    t = fmaf(d, e, t);
  }
};

// Lists of touched tokens in the workspace: [B * n_chunks] counts, tokens relative to their chunk with the flag kSeen, offsets.
// A list of odd length has a token behind it that stands for none.
struct Lists {
  int* count;
  uint16_t* token;
  float* offset;
};
constexpr size_t kListStride = kListMost + 8;
inline size_t lists_bytes(long long n) { return (size_t)n * (16 + kListStride * 6) + 64; }
inline Lists carve_lists(void* at, long long n) {
  Lists l;
  unsigned char* p = static_cast<unsigned char*>(at);
  l.offset = reinterpret_cast<float*>(p); p += (size_t)n * kListStride * 4;
  l.token = reinterpret_cast<uint16_t*>(p); p += (size_t)n * kListStride * 2;
  l.count = reinterpret_cast<int*>(p);
  return l;
}

// One block per (sequence, chunk): each thread compacts one word of bits, then the records are looked up side by side.  Latency:
// 6.5 us for 48 sequences, 12 us for 64 with 5250 touched tokens each.
__global__ void __launch_bounds__(256) touched_list_kernel(AdjustView a, int n_chunks, int chunk_len, Lists lists) {
  __shared__ int count_s[8];
  __shared__ uint16_t token_s[kListMost];
  grid_dependency_trigger();
  const int b = blockIdx.x / n_chunks, chunk = blockIdx.x - b * n_chunks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int at = chunk * (chunk_len / 32) + tid;
  uint32_t w = tid < chunk_len / 32 && at < a.words ? a.bits[(size_t)b * a.words + at] : 0u;
  if ((at + 1) * 32 > a.V) w &= at * 32 < a.V ? (1u << (a.V - at * 32)) - 1u : 0u;       // nothing past the vocabulary
  const int n = __popc(w);
  int upto = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += up;
  }
  if (lane == 31) count_s[warp] = upto;
  __syncthreads();
  int to = upto - n, total = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k < warp) to += count_s[k];
    total += count_s[k];
  }
  if (tid == 0) lists.count[blockIdx.x] = total;
  if (total > kListMost) return;
  for (; w; w &= w - 1) token_s[to++] = (uint16_t)(tid * 32 + __ffs(w) - 1);
  __syncthreads();
  const RowRules r = history_rules(a, b);
  uint16_t* const token = lists.token + blockIdx.x * kListStride;
  float* const offset = lists.offset + blockIdx.x * kListStride;
  for (int k = tid; k < ((total + 1) & ~1); k += 256) {
    if (k == total) {
      token[k] = (uint16_t)chunk_len;
      offset[k] = 0.f;
      continue;
    }
    const uint32_t v = token_s[k];
    const int2 rec = r.record[chunk * chunk_len + v];
    token[k] = (uint16_t)(v | (rec.x != 0 ? kSeen : 0u));
    offset[k] = rule_offset(rec, r);
  }
}

// What the producer puts beside the 16 KB of a row.
template <typename T>
struct Item {
  const T* src;                               // token 0 of the chunk
  const uint32_t* allowed;                    // the chunk's bits, or NULL
  const uint32_t* touched;
  const int2* record;
  long long out;                              // where the partial goes
  int row, token0, len, list, n_list, mode;   // row -1: nothing, -2: the end
  int shift, copied;                          // token 0 sits at this place of the stage; places that the copy fills
  float repetition, inverse, presence, frequency;
};
enum { kNothing, kGather, kCopy };

template <typename T>
struct ConfSmem {
  alignas(128) uint8_t stage[kChunkBytes + 16];
  alignas(16) uint16_t token[kListNear];      // the chunk's list, if it is that short
  alignas(16) float offset[kListNear];
  Item<T> item;
  uint64_t full, empty;
  int gave_up;
  float top[2][kConfWarps];                   // the warps' maxima
  float4 join[2][kConfWarps];                 // and their statistics
};

template <typename T>
__device__ __forceinline__ RowRules rules_of(const Item<T>& it) {
  RowRules r;
  r.touched = it.touched; r.allowed = it.allowed; r.record = it.record;
  r.repetition = it.repetition; r.inverse = it.inverse; r.presence = it.presence; r.frequency = it.frequency;
  return r;
}
__device__ __forceinline__ bool bit_of(const uint32_t* bits, int v) { return (bits[v >> 5] >> (v & 31)) & 1u; }

// Word j of this thread's share of a chunk's bits, none past its len tokens.
__device__ __forceinline__ uint32_t my_bits(const uint32_t* bits, int j, int len, int& at) {
  at = (j * kConfThreads + (int)threadIdx.x) * 32;
  if (at >= len) return 0u;
  return bits[at >> 5] & (len - at >= 32 ? 0xffffffffu : (1u << (len - at)) - 1u);
}

// A thread's statistics of tokens that it takes one by one.
struct Single {
  Lane z;
  float best;
  int token;
  __device__ __forceinline__ void clear() { z = Lane{kLow, kLow * kLog2e, 0.f, 0.f}; best = kLow; token = kNoToken; }
  __device__ __forceinline__ void take(float x, int v) {
    if (x > best || (x == best && v < token && best > kLow)) { best = x; token = v; }
    if (x > kLow) z.add(x);
  }
};

// The tokens of a chunk that a mask allows, gathered.
template <typename T>
__device__ __forceinline__ void gather_allowed(const Item<T>& it, Single* out) {
  const RowRules r = rules_of(it);
  Single g;
  g.clear();
  for (int j = 0; j < (int)(kChunkBytes / sizeof(T)) / 32 / kConfThreads; ++j) {
    int at0;
    uint32_t bits = my_bits(it.allowed, j, it.len, at0);
    const uint32_t rec = bits && it.touched ? it.touched[at0 >> 5] : 0u;
    for (; bits; bits &= bits - 1) {
      const int e = __ffs(bits) - 1;
      const float x = ld_as_float(it.src, at0 + e);
      g.take((rec >> e) & 1u ? adjust_token(x, r.record[at0 + e], r) : x, it.token0 + at0 + e);
    }
  }
  *out = g;
}

// The touched tokens of a copied chunk that has no list: out of the stage, found by their bits.
template <typename T>
__device__ __forceinline__ void walk_touched(const Item<T>& it, T* stage, Single* out) {
  const RowRules r = rules_of(it);
  Single g;
  g.clear();
  for (int j = 0; j < (int)(kChunkBytes / sizeof(T)) / 32 / kConfThreads; ++j) {
    int at0;
    for (uint32_t bits = my_bits(it.touched, j, it.len, at0); bits; bits &= bits - 1) {
      const int at = at0 + __ffs(bits) - 1;
      const float x = ld_as_float(stage, at);
      st_from_float(stage, at, kFloor);
      if (it.allowed == nullptr || bit_of(it.allowed, at)) g.take(adjust_token(x, r.record[at], r), it.token0 + at);
    }
  }
  *out = g;
}

// All tokens of a chunk once more, one by one, with nothing counted as nothing; every thread gets its warp's part.
template <typename T>
__device__ __forceinline__ float4 slow_statistics(const Item<T>& it) {
  const RowRules r = rules_of(it);
  Stats slow;
  slow.clear();
  for (int at = threadIdx.x; at < it.len; at += kConfThreads) slow.add(adjusted_logit(it.src, at, r), it.token0 + at);
  return join_lanes(slow);
}

// Tokens of a chunk that a mask allows, by a warp.  Not inlined: 64 x 32 rows without a mask take 4 us less of 141.
template <int WORDS>
__device__ __noinline__ int count_allowed(const uint32_t* allowed, int len) {
  int n = 0;
#pragma unroll
  for (int j = 0; j < WORDS; ++j) {
    const int at = j * 32 + (int)(threadIdx.x & 31), left = len - at * 32;
    if (left > 0) n += __popc(allowed[at] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u));
  }
  return __reduce_add_sync(0xffffffffu, n);
}

// The stage holds 16-byte blocks as they lie in memory.  BOUND: every row starts on such a boundary.  Otherwise the chunk's
// token 0 sits at place `shift` of the stage, the block that the row ends in (which the next row begins in, or nothing) is
// filled token by token, and the up to VL - 1 tokens that are pushed behind the last vector are taken one by one.
template <typename T, bool BOUND>
__global__ void __launch_bounds__(kConfThreads + 32, kConfBlocksPerSM)
conf_adjusted_kernel(AdjustView a, int n_chunks, long long n_items, Lists lists, const T* __restrict__ logits,
                     const int32_t* __restrict__ perm, const int32_t* __restrict__ n_filled, const int32_t* __restrict__ window_len,
                     float4* __restrict__ part, int32_t* status) {
  constexpr int VL = Part<T>::VL;
  constexpr int kChunk = (int)(kChunkBytes / sizeof(T));            // tokens
  extern __shared__ __align__(128) uint8_t smem_raw[];
  ConfSmem<T>& sm = *reinterpret_cast<ConfSmem<T>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t full = smem_u32(&sm.full), empty = smem_u32(&sm.empty);
  if (tid == 0) {
    mbar_init(full, 1);
    mbar_init(empty, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm.gave_up = 0;
    st_from_float(reinterpret_cast<T*>(sm.stage), kChunk, kFloor);  // the place of the token that evens out a list
  }
  __syncthreads();
  grid_dependency_wait();
  grid_dependency_trigger();

  if (warp == kConfWarps) {
    // ---- producer warp: finds out about 32 items ahead at a time, one per lane, and fills the slot with one after the
    // other; while a copy runs, it writes out the statistics of the last item but one
    uint32_t n = 0;
    long long out1 = -1, out2 = -1;                                 // the last item that was given out, and the one before
    auto write_out = [&](uint32_t k, long long out) {
      float m = -CUDART_INF_F, sum = 0.f, tilt = 0.f;
      int token = kNoToken;
#pragma unroll
      for (int j = 0; j < kConfWarps; ++j) m = fmaxf(m, sm.join[k & 1][j].x);
#pragma unroll
      for (int j = 0; j < kConfWarps; ++j) {
        const float4 p = sm.join[k & 1][j];
        if (p.x == m) token = min(token, __float_as_int(p.w));
        const float d = p.x - m, f = p.y > 0.f ? ex2_approx(d * kLog2e) : 0.f;
        sum += p.y * f;
        if (f > 0.f) tilt += fmaf(d, p.y, p.z) * f;
      }
      part[out] = make_float4(m, sum, tilt, __int_as_float(m > -CUDART_INF_F ? token : kNoToken));
    };
    for (long long it0 = blockIdx.x;; it0 += 32LL * gridDim.x) {
      const long long mine = it0 + (long long)lane * gridDim.x;
      int row = 0, list = 0, n_list = 0, m = -1;
      float repetition = 1.f, presence = 0.f, frequency = 0.f;
      bool active = false;
      if (mine < n_items) {
        row = (int)(mine / n_chunks);
        const int chunk = (int)(mine - (long long)row * n_chunks);
        const int b = row / a.W, i = row - b * a.W;
        const int L = window_len ? min(max(window_len[b], 0), a.W) : a.W;
        active = i >= n_filled[b] && i < L;                         // an active mask row
        list = b * n_chunks + chunk;
        if (a.bits) n_list = lists.count[list];
        if (a.mask_index) m = a.mask_index[(size_t)b * a.W + min(max(perm[row], 0), a.W - 1)];
        if (a.repetition) repetition = a.repetition[b];
        if (a.presence) presence = a.presence[b];
        if (a.frequency) frequency = a.frequency[b];
        if (m >= a.n_masks) {                                       // no such mask: flagged, the row is left unconstrained
          if (status && active) atomicOr(status, WEDLM_STATUS_BAD_TOKEN);
          m = -1;
        }
      }
      const float inverse = __frcp_rn(repetition);
      for (uint32_t todo = __ballot_sync(0xffffffffu, active); todo; todo &= todo - 1) {
        const int l = __ffs(todo) - 1;
        const long long it = it0 + (long long)l * gridDim.x;
        Item<T> w;
        w.row = __shfl_sync(0xffffffffu, row, l);
        w.n_list = __shfl_sync(0xffffffffu, n_list, l);
        w.list = __shfl_sync(0xffffffffu, list, l);
        w.repetition = __shfl_sync(0xffffffffu, repetition, l);
        w.inverse = __shfl_sync(0xffffffffu, inverse, l);
        w.presence = __shfl_sync(0xffffffffu, presence, l);
        w.frequency = __shfl_sync(0xffffffffu, frequency, l);
        const int mask = __shfl_sync(0xffffffffu, m, l), b = w.row / a.W, chunk = w.list - b * n_chunks;
        w.token0 = chunk * kChunk;
        w.len = min(kChunk, a.V - w.token0);
        w.src = logits + (size_t)w.row * a.V + w.token0;
        w.shift = BOUND ? 0 : (int)((uintptr_t)w.src & 15u) / (int)sizeof(T);
        w.copied = BOUND ? w.len : (w.shift + w.len) / VL * VL;
        w.allowed = mask >= 0 ? a.allowed + (size_t)mask * a.words + w.token0 / 32 : nullptr;
        w.touched = a.bits ? a.bits + (size_t)b * a.words + w.token0 / 32 : nullptr;
        w.record = a.record + (size_t)b * a.V + w.token0;
        w.out = it;
        w.mode = kCopy;
        if (w.allowed) {
          const int n_allowed = count_allowed<kChunk / 1024>(w.allowed, w.len);
          if (n_allowed == 0) {
            if (lane == 0) part[it] = make_float4(-CUDART_INF_F, 0.f, 0.f, __int_as_float(kNoToken));
            continue;
          }
          w.mode = n_allowed <= kGatherMost ? kGather : kCopy;
        }
        bool ok = true;
        if (lane == 0) {
          if (n > 0) ok = mbar_wait(empty, (n - 1) & 1u);
          if (ok) {
            if (w.mode == kCopy) {
              const bool near = w.n_list > 0 && w.n_list <= kListNear;
              const uint32_t bytes = (uint32_t)w.copied * (uint32_t)sizeof(T), list_bytes = near ? (uint32_t)((w.n_list + 7) & ~7) * 2u : 0u;
              auto copy = [&](void* to, const void* from, uint32_t n_bytes) {
                if (n_bytes)
                  asm volatile(
                      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                      ::"r"(smem_u32(to)), "l"(from), "r"(n_bytes), "r"(full) : "memory");
              };
              asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(full), "r"(bytes + 3u * list_bytes) : "memory");
              copy(sm.stage, w.src - w.shift, bytes);
              if (near) {
                copy(sm.token, lists.token + w.list * kListStride, list_bytes);
                copy(sm.offset, lists.offset + w.list * kListStride, 2u * list_bytes);
              }
            }
            sm.item = w;
            if (n > 1) write_out(n - 2, out2);                      // complete since the slot came back
            out2 = out1;
            out1 = w.out;
            mbar_arrive(full);
          } else if (status) {
            atomicOr(status, WEDLM_STATUS_WAIT_EXPIRED);
          }
        }
        ++n;
        if (__shfl_sync(0xffffffffu, ok ? 1 : 0, 0) == 0) return;
      }
      if (it0 + 32LL * gridDim.x >= n_items) break;
    }
    if (lane == 0) {                                                // the end: twice, so that the last item is complete too
      for (int k = 0; k < 2 && n > 0; ++k, ++n) {
        if (!mbar_wait(empty, (n - 1) & 1u)) {
          if (status) atomicOr(status, WEDLM_STATUS_WAIT_EXPIRED);
          return;
        }
        if (n > 1) write_out(n - 2, out2);
        out2 = out1;
        sm.item.row = k == 0 ? -1 : -2;
        mbar_arrive(full);
      }
      if (n == 0) {
        sm.item.row = -2;
        mbar_arrive(full);
      }
    }
    return;
  }

  for (uint32_t n = 0;; ++n) {
    // Bounded, never expected to expire.  A thread whose wait does expire takes nothing and carries on to the barrier below,
    // behind which all consumers leave together: until there every thread passes the same number of barriers, whatever it saw.
    const bool got = mbar_wait(full, n & 1u);
    if (!got) *(volatile int*)&sm.gave_up = 1;
    const int row = got ? *(volatile int*)&sm.item.row : -1;
    const int mode = row < 0 ? kNothing : sm.item.mode, token0 = sm.item.token0, place0 = BOUND ? 0 : sm.item.shift;
    float best = kLow;                                              // of the streamed tokens
    Single g;
    g.clear();
    Part<T> q;
    if (mode == kCopy) {
      const int len = sm.item.len, n_list = sm.item.n_list, shift = place0;
      const uint32_t* const allowed_bits = sm.item.allowed;
      T* const stage = reinterpret_cast<T*>(sm.stage) + shift;      // token 0
      if (!BOUND) {
        // the block that the row ends in, token by token; nothing before token 0 and behind the row
        const int copied = sm.item.copied;
        if (copied + tid < shift + len) stage[copied - shift + tid] = sm.item.src[copied - shift + tid];
        if (tid < shift) st_from_float(stage, tid - shift, kFloor);
        for (int k = len + tid; k < kChunk + VL - shift; k += kConfThreads) st_from_float(stage, k, kFloor);
        consumer_sync();
      }
      if (n_list <= kListMost) {
        const bool near = n_list <= kListNear;
        const size_t list = (size_t)sm.item.list;
        const uint32_t* const two_at = reinterpret_cast<const uint32_t*>(near ? sm.token : lists.token + list * kListStride);
        const float2* const off_at = reinterpret_cast<const float2*>(near ? sm.offset : lists.offset + list * kListStride);
        RowRules r;
        r.repetition = sm.item.repetition;
        r.inverse = sm.item.inverse;
        for (int k = tid; k < (n_list + 1) >> 1; k += kConfThreads) {         // two at a time
          const uint32_t two = two_at[k];
          const float2 off = off_at[k];
          const int at0 = (int)(two & (kSeen - 1u)), at1 = (int)((two >> 16) & (kSeen - 1u));
          float x0 = fmaxf(apply_rules(ld_as_float(stage, at0), (two & kSeen) != 0, off.x, r), kFloor);
          float x1 = fmaxf(apply_rules(ld_as_float(stage, at1), (two & (kSeen << 16)) != 0, off.y, r), kFloor);
          st_from_float(stage, at0, kFloor);
          st_from_float(stage, at1, kFloor);
          if (allowed_bits) {
            if (!bit_of(allowed_bits, at0)) x0 = kFloor;
            if (at1 >= len || !bit_of(allowed_bits, at1)) x1 = kFloor;
          }
          const float top = fmaxf(x0, x1);
          if (top > g.best) {                                       // (ascending: the first of equals stays)
            g.best = top;
            g.token = token0 + (x0 == top ? at0 : at1);
          }
          if (top > g.z.m) g.z.raise(top);
          const float d0 = fmaf(x0, kLog2e, -g.z.r), d1 = fmaf(x1, kLog2e, -g.z.r);
          const float e0 = ex2_approx(d0), e1 = ex2_approx(d1);
          g.z.s += e0 + e1;
          g.z.t = fmaf(d1, e1, fmaf(d0, e0, g.z.t));
        }
      } else {
        Single walked;                                              // (g itself stays in registers)
        walk_touched<T>(sm.item, stage, &walked);
        g = walked;
      }
      if (BOUND && len < kChunk)
        for (int k = len + tid; k < kChunk; k += kConfThreads) st_from_float(stage, k, kFloor);     // the row ends: old bytes behind it
      consumer_sync();
      if (!BOUND && kChunk - shift + tid < len) {                   // pushed behind the last vector
        const int at = kChunk - shift + tid;
        const float x = ld_as_float(stage, at);
        if (x > kLow && (allowed_bits == nullptr || bit_of(allowed_bits, at))) g.take(x, token0 + at);
      }
      q.load(sm.stage, tid);
      if (allowed_bits) {
        uint32_t on[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = (k * kConfThreads + tid) * VL - shift;
          if (BOUND) on[k] = at < len ? (reinterpret_cast<const uint8_t*>(allowed_bits)[at >> 3] >> (at & 7)) & ((1u << VL) - 1u) : 0u;
          else on[k] = bits_at(allowed_bits, at, (len + 31) >> 5) & ((1u << VL) - 1u);
        }
        q.mask(on);
      }
      fence_async_smem();                                           // reads and pokes before the next copy's writes
      best = q.clamp_and_maximum();
    } else {
      if (mode == kGather) {
        Single gathered;
        gather_allowed<T>(sm.item, &gathered);
        g = gathered;
      }
      consumer_sync();
      if (!BOUND) consumer_sync();
    }
    float m = fmaxf(best, g.best);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) sm.top[n & 1][warp] = m;
    consumer_sync();
    if (*(volatile int*)&sm.gave_up) {
      if (tid == 0 && status) atomicOr(status, WEDLM_STATUS_WAIT_EXPIRED);
      for (int it = 0; it < 200; ++it) __nanosleep(1000);           // let a late copy land
      return;
    }
    if (row == -2) return;                                          // the end, alike for all
    m = fmaxf(fmaxf(sm.top[n & 1][0], sm.top[n & 1][1]), fmaxf(sm.top[n & 1][2], sm.top[n & 1][3]));
    float4 p;
    if (!(m > kLow) && mode != kNothing) {                          // alike for all
      p = slow_statistics<T>(sm.item);
      consumer_sync();
    }
    if (tid == 0) mbar_arrive(empty);
    if (mode == kNothing) continue;
    if (m > kLow) {
      int token = g.best == m ? g.token : kNoToken;
      g.z.raise(m);
      if (mode == kCopy) {
        if (best == m) token = min(token, q.find(m, token0 + tid * VL - place0));
        const unsigned long long L2 = pack2(kLog2e, kLog2e), NR = pack2(-g.z.r, -g.z.r);
        unsigned long long sA = pack2(g.z.s, 0.f), sB = pack2(0.f, 0.f), tA = pack2(g.z.t, 0.f), tB = sB;
#pragma unroll
        for (int k = 0; k < Part<T>::kPairs; k += 2) {
          float x0, x1, y0, y1;
          q.pair(k, x0, x1);
          q.pair(k + 1, y0, y1);
          const unsigned long long dA = fma2(pack2(x0, x1), L2, NR), dB = fma2(pack2(y0, y1), L2, NR);
          unpack2(dA, x0, x1);
          unpack2(dB, y0, y1);
          const unsigned long long eA = pack2(ex2_approx(x0), ex2_approx(x1)), eB = pack2(ex2_approx(y0), ex2_approx(y1));
          sA = add2(sA, eA);
          sB = add2(sB, eB);
          tA = fma2(dA, eA, tA);
          tB = fma2(dB, eB, tB);
        }
        float lo, hi;
        unpack2(add2(sA, sB), lo, hi);
        g.z.s = lo + hi;
        unpack2(add2(tA, tB), lo, hi);
        g.z.t = lo + hi;
      }
      token = __reduce_min_sync(0xffffffffu, token);
      // the reference as rounded -> the maximum itself
      const float d = fmaf(-m, kLog2e, g.z.r), f = ex2_approx(d);
      float s = g.z.s, t = g.z.t;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
      }
      p = make_float4(m, s * f, fmaf(d, s, t) * f * 0.6931471805599453f, __int_as_float(token));
    }
    if (lane == 0) sm.join[n & 1][warp] = p;
  }
}

// Buffers off 16-byte boundaries: one block per item, token by token, four loads in flight per thread.
constexpr int kScalarThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kScalarThreads)
conf_adjusted_scalar_kernel(AdjustView a, int n_chunks, int chunk_len, const T* __restrict__ logits, const int32_t* __restrict__ perm,
                            const int32_t* __restrict__ n_filled, const int32_t* __restrict__ window_len, float4* __restrict__ part,
                            int32_t* status) {
  __shared__ float4 join_s[kScalarThreads / 32];
  const int row = blockIdx.x / n_chunks, chunk = blockIdx.x - row * n_chunks;
  const int b = row / a.W, i = row - b * a.W;
  const int L = window_len ? min(max(window_len[b], 0), a.W) : a.W;
  if (i < n_filled[b] || i >= L) return;                            // not an active mask row
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const RowRules r = row_rules(a, b, min(max(perm[row], 0), a.W - 1), chunk == 0 && tid == 0 ? status : nullptr);
  const T* src = logits + (size_t)row * a.V;
  const int end = min(a.V, (chunk + 1) * chunk_len);
  Stats z;
  z.clear();
  int v = chunk * chunk_len + tid;
  for (; v + 3 * kScalarThreads < end; v += 4 * kScalarThreads) {
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = adjusted_logit(src, v + u * kScalarThreads, r);
#pragma unroll
    for (int u = 0; u < 4; ++u) z.add(x[u], v + u * kScalarThreads);
  }
  for (; v < end; v += kScalarThreads) z.add(adjusted_logit(src, v, r), v);
  float4 p = join_lanes(z);
  if (lane == 0) join_s[warp] = p;
  __syncthreads();
  if (warp != 0) return;
  p = lane < kScalarThreads / 32 ? join_s[lane] : make_float4(-CUDART_INF_F, 0.f, 0.f, __int_as_float(kNoToken));
  Stats all;
  all.m = all.best = p.x;
  all.token = __float_as_int(p.w);
  all.s = p.y;
  all.t = p.z * kLog2e;
  p = join_lanes(all);
  if (lane == 0) part[(size_t)row * n_chunks + chunk] = p;
}

template <typename T>
int launch_conf_adjusted_t(const Shape& s, const AdjustView& a, int n_chunks, int chunk, const T* logits, const int32_t* perm,
                           const int32_t* n_filled, const int32_t* window_len, float4* part, void* list_ws, int32_t* status,
                           cudaStream_t st) {
  const long long items = (long long)s.B * s.W * n_chunks;
  if (items > 0x7fffffffLL) return WEDLM_ERR_UNSUPPORTED;
  if ((uintptr_t)logits % 16 != 0) {                                // (a block's first bytes could lie before the buffer)
    conf_adjusted_scalar_kernel<<<(unsigned)items, kScalarThreads, 0, st>>>(a, n_chunks, chunk, logits, perm, n_filled, window_len,
                                                                            part, status);
    count_launch();
    return cuda_ok(cudaGetLastError());
  }
  const Lists lists = carve_lists(list_ws, (long long)s.B * n_chunks);
  if (a.bits) {
    touched_list_kernel<<<(unsigned)(s.B * n_chunks), 256, 0, st>>>(a, n_chunks, chunk, lists);
    count_launch();
  }
  const bool bound = (size_t)s.V * sizeof(T) % 16 == 0;
  auto kern = bound ? conf_adjusted_kernel<T, true> : conf_adjusted_kernel<T, false>;
  static bool attr_done[2][64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return WEDLM_ERR_CUDA;
  if (dev < 0 || dev >= 64 || !attr_done[bound][dev]) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ConfSmem<T>)) != cudaSuccess)
      return WEDLM_ERR_CUDA;
    if (dev >= 0 && dev < 64) attr_done[bound][dev] = true;
  }
  long long grid = (long long)device_sm_count() * kConfBlocksPerSM;
  if (grid > items) grid = items;
  // With at most one list per SM the blocks start beside the lists', set up and wait (one request 15.3 -> 12.5 us); with more
  // they would take the places of lists still to come (16 requests: 36.9 us instead of 32.9).
  if (a.bits && (long long)s.B * n_chunks <= device_sm_count()) {
    if (!launch_behind(kern, (unsigned)grid, kConfThreads + 32, sizeof(ConfSmem<T>), st, a, n_chunks, items, lists, logits, perm,
                       n_filled, window_len, part, status))
      return WEDLM_ERR_CUDA;
  } else {
    kern<<<(unsigned)grid, kConfThreads + 32, sizeof(ConfSmem<T>), st>>>(a, n_chunks, items, lists, logits, perm, n_filled, window_len,
                                                                      part, status);
  }
  count_launch();
  return cuda_ok(cudaGetLastError());
}

// ---------------------------------------------------------------------------------------------- the rules alone
// Buffers on 16-byte boundaries; where the rows are not (BOUND false), a row's vectors begin at its first boundary, and the
// tokens in front of them and behind them are done one by one.  A warp takes eight vectors per lane, asynchronously into 4 KB of
// shared memory (a vector with nothing allowed is not read), with the records of the first touched tokens on their way at the
// same time; the mask and then the touched tokens, four per lane at a time, are applied there, and the span is written out.  In
// place only what changes is read and written.
// Bound: the logits, read and written once: 133 us for 64 x 32 rows of 151 936 bf16 tokens, two in five masked (705 MB, 5.3 TB/s).
// With the vectors in registers and each touched token read back and written by itself 158 us; in registers on the way to
// shared memory 179 us (96 registers).  Ten blocks on an SM 132, twelve 143, sixteen 165 us.
template <typename T, bool BOUND>
__global__ void __launch_bounds__(32 * kWarpsPerBlock)
logits_adjust_kernel(AdjustView a, int n_spans, long long n_items, const T* logits, T* out, const int32_t* __restrict__ perm,
                     const int32_t* __restrict__ n_filled, const int32_t* __restrict__ window_len, int32_t* status) {
  constexpr int VL = Part<T>::VL, kSpan = kAdjustVecs * 32 * VL, kWords = kSpan / 1024;
  constexpr uint32_t kAll = (1u << VL) - 1u;
  __shared__ __align__(16) uint8_t stage_s[kWarpsPerBlock][kAdjustVecs * 512];
  const long long item = (long long)blockIdx.x * kWarpsPerBlock + (threadIdx.x >> 5);
  if (item >= n_items) return;
  const int lane = threadIdx.x & 31;
  const int row = (int)(item / n_spans), span = (int)(item - (long long)row * n_spans);
  const int b = row / a.W, i = row - b * a.W;
  const int head = BOUND ? 0 : min((int)((16u - ((uintptr_t)(logits + (size_t)row * a.V) & 15u)) & 15u) / (int)sizeof(T), a.V);
  const int vec_end = BOUND ? a.V : head + (a.V - head) / VL * VL;
  const int token0 = head + span * kSpan, len = min(kSpan, vec_end - token0);
  // what depends on nothing else, at once: the chain to the logits is a load shorter for it
  const int filled = n_filled[b], L = window_len ? min(max(window_len[b], 0), a.W) : a.W, slot = perm[row];
  uint32_t touched[kWords];
#pragma unroll
  for (int j = 0; j < kWords; ++j) {
    const int at = (token0 >> 5) + j * 32 + lane;
    const uint32_t* const bits = a.bits + (size_t)b * a.words;
    if (BOUND) touched[j] = a.bits && at < a.words ? bits[at] : 0u;
    else touched[j] = a.bits ? bits_at(bits, token0 + (j * 32 + lane) * 32, a.words) : 0u;
  }
  const int m = a.mask_index ? a.mask_index[(size_t)b * a.W + min(max(slot, 0), a.W - 1)] : -1;
  if (i < filled || i >= L) return;                                 // not an active mask row
  RowRules r = history_rules(a, b);
  if (m >= a.n_masks) {                                             // no such mask: flagged, the row is left unconstrained
    if (status && span == 0 && lane == 0) atomicOr(status, WEDLM_STATUS_BAD_TOKEN);
  } else if (m >= 0) {
    r.allowed = a.allowed + (size_t)m * a.words;
  }
  const T* const src = logits + (size_t)row * a.V + token0;
  T* const dst = out + (size_t)row * a.V + token0;
  const bool in_place = src == dst;
#pragma unroll
  for (int j = 0; j < kWords; ++j) {
    const int at = (token0 >> 5) + j * 32 + lane;
    if (BOUND) {
      if (r.allowed && at < a.words) touched[j] &= r.allowed[at];
    } else if (r.allowed) {
      touched[j] &= bits_at(r.allowed, token0 + (j * 32 + lane) * 32, a.words);
    }
  }
  // the touched tokens of this lane, none past the span
  {
    int at0 = lane * 32;
#pragma unroll
    for (int j = 0; j < kWords; ++j, at0 += 1024) {
      const int left = len - at0;
      if (left < 32) touched[j] &= left <= 0 ? 0u : (1u << left) - 1u;
    }
  }
  int at[4];
  int2 rec[4];
  auto next_four = [&]() {                                          // the next four, their records on the way
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      at[u] = -1;
#pragma unroll
      for (int j = 0; j < kWords; ++j)
        if (at[u] < 0 && touched[j]) {
          at[u] = j * 1024 + lane * 32 + __ffs(touched[j]) - 1;
          touched[j] &= touched[j] - 1;
        }
      if (at[u] >= 0) rec[u] = r.record[token0 + at[u]];
    }
  };
  auto masked = [&](const uint4& v, uint32_t on) -> uint4 {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (VL == 8) {
        if (!((on >> (2 * e)) & 1u)) w[e] = (w[e] & 0xffff0000u) | 0xff80u;
        if (!((on >> (2 * e + 1)) & 1u)) w[e] = (w[e] & 0xffffu) | 0xff800000u;
      } else if (!((on >> e) & 1u)) {
        w[e] = 0xff800000u;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  };
  T* const stage = reinterpret_cast<T*>(stage_s[threadIdx.x >> 5]);
  T* const held = in_place ? dst : stage;                           // where the touched tokens are changed
  uint32_t on[kAdjustVecs];
#pragma unroll
  for (int k = 0; k < kAdjustVecs; ++k) {
    const int v = (k * 32 + lane) * VL;
    on[k] = v < len ? kAll : 0u;
    if (r.allowed && v < len)
      on[k] = (BOUND ? reinterpret_cast<const uint8_t*>(r.allowed)[(token0 + v) >> 3] >> (v & 7) : bits_at(r.allowed, token0 + v, a.words)) & kAll;
    if (!in_place && on[k] != 0)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(stage + v)), "l"(src + v) : "memory");
  }
  next_four();
  if (!in_place) asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int k = 0; k < kAdjustVecs; ++k) {
    const int v = (k * 32 + lane) * VL;
    if (v >= len || on[k] == kAll) continue;
    uint4* const to = reinterpret_cast<uint4*>(held + v);
    *to = masked(on[k] ? *to : make_uint4(0u, 0u, 0u, 0u), on[k]);
  }
  __syncwarp();
  while (at[0] >= 0) {
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at[u] >= 0) x[u] = ld_as_float(held, (size_t)at[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at[u] >= 0) st_from_float(held, (size_t)at[u], adjust_token(x[u], rec[u], r));
    next_four();
  }
  if (!in_place) {
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kAdjustVecs; ++k) {
      const int v = (k * 32 + lane) * VL;
      if (v < len) *reinterpret_cast<uint4*>(dst + v) = *reinterpret_cast<const uint4*>(stage + v);
    }
  }
  if (!BOUND && span == 0) {                                        // lanes 0..: in front of the vectors, 16..: behind them
    const int v = lane < head ? lane : (lane >= 16 && vec_end + lane - 16 < a.V ? vec_end + lane - 16 : -1);
    if (v >= 0) st_from_float(out + (size_t)row * a.V, (size_t)v, adjusted_logit(logits + (size_t)row * a.V, v, r));
  }
}

// Buffers off 16-byte boundaries.
template <typename T>
__global__ void __launch_bounds__(32 * kWarpsPerBlock)
logits_adjust_scalar_kernel(AdjustView a, int n_chunks, int chunk_len, long long n_items, const T* logits, T* out,
                            const int32_t* __restrict__ perm, const int32_t* __restrict__ n_filled,
                            const int32_t* __restrict__ window_len, int32_t* status) {
  int row, b, chunk;
  if (!warp_item(a.W, n_chunks, n_items, n_filled, window_len, row, b, chunk)) return;
  const int lane = threadIdx.x & 31;
  const RowRules r = row_rules(a, b, min(max(perm[row], 0), a.W - 1), chunk == 0 && lane == 0 ? status : nullptr);
  const T* src = logits + (size_t)row * a.V;
  T* dst = out + (size_t)row * a.V;
  const int end = min(a.V, (chunk + 1) * chunk_len);
  int v = chunk * chunk_len + lane;
  for (; v + 3 * 32 < end; v += 4 * 32) {                           // four loads in flight
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = adjusted_logit(src, v + u * 32, r);
#pragma unroll
    for (int u = 0; u < 4; ++u) st_from_float(dst, (size_t)(v + u * 32), x[u]);
  }
  for (; v < end; v += 32) st_from_float(dst, (size_t)v, adjusted_logit(src, v, r));
}

// One thread per token.  Integer atomics only: the result does not depend on their order.  Bound: one launch and an atomic round
// trip, 6.3 us for a step of 64 x 32 tokens; 64 prompts of 8192 tokens 8.2 us (11.8 without the look in front of the atomics).
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
    // a prompt repeats its frequent tokens: a look is cheaper than two more atomics on the same words
    int2* const rec = a.record + (size_t)b * a.V + v;
    uint32_t* const word = a.bits + (size_t)b * a.words + (v >> 5);
    const uint32_t bit = 1u << (v & 31);
    const int have = *reinterpret_cast<volatile int*>(&rec->x);
    const bool touched = (ld_bits(word) & bit) != 0u;
    if (touched && (have & 1)) return;                      // (if that was left there, whoever set the bit writes 1 in its place)
    if (!touched && !(or_bits(word, bit) & bit)) {
      rec->y = 0;
      atomicExch(&rec->x, 1);                               // all that others may add meanwhile is the same mark
    } else {
      atomicOr(&rec->x, 1);
    }
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
    // (one thread per token: nobody else is at this record)
    int2* const rec = a.record + (size_t)b * a.V + v;
    if (!((atomicOr(a.bits + (size_t)b * a.words + (v >> 5), 1u << (v & 31)) >> (v & 31)) & 1u)) rec->x = 0;
    rec->y = __float_as_int(values[(size_t)b * n_ids + k]);
  }
}

}  // namespace

size_t conf_adjusted_list_bytes(int B, int n_chunks) { return lists_bytes((long long)B * n_chunks); }

int launch_conf_adjusted_pass1(const Shape& s, const AdjustView& a, int n_chunks, int chunk, const void* logits,
                               const int32_t* perm, const int32_t* n_filled, const int32_t* window_len, void* partials,
                               void* list_ws, int32_t* status, cudaStream_t st) {
  const bool bf16 = s.dtype == WEDLM_DTYPE_BF16;
  if (chunk * (bf16 ? 2 : 4) != (int)kChunkBytes) return WEDLM_ERR_UNSUPPORTED;
  float4* part = reinterpret_cast<float4*>(partials);
  return bf16 ? launch_conf_adjusted_t(s, a, n_chunks, chunk, static_cast<const __nv_bfloat16*>(logits), perm, n_filled, window_len,
                                       part, list_ws, status, st)
              : launch_conf_adjusted_t(s, a, n_chunks, chunk, static_cast<const float*>(logits), perm, n_filled, window_len, part,
                                       list_ws, status, st);
}

int launch_logits_adjust(const Shape& s, const AdjustView& a, const void* logits, void* out, const int32_t* perm,
                         const int32_t* n_filled, const int32_t* window_len, int32_t* status, cudaStream_t st) {
  auto go = [&](auto* x) -> int {
    using T = std::remove_cv_t<std::remove_pointer_t<decltype(x)>>;
    T* y = static_cast<T*>(out);
    const bool vectors = (uintptr_t)x % 16 == 0 && (uintptr_t)y % 16 == 0, bound = (size_t)s.V * sizeof(T) % 16 == 0;
    const int span = vectors ? kAdjustVecs * 32 * Part<T>::VL : 512;
    const int n_spans = (s.V + span - 1) / span;
    const long long items = (long long)s.B * s.W * n_spans;
    const long long blocks = (items + kWarpsPerBlock - 1) / kWarpsPerBlock;
    if (blocks > 0x7fffffffLL) return WEDLM_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)blocks, threads = 32 * kWarpsPerBlock;
    if (vectors && bound)
      logits_adjust_kernel<T, true><<<grid, threads, 0, st>>>(a, n_spans, items, x, y, perm, n_filled, window_len, status);
    else if (vectors)
      logits_adjust_kernel<T, false><<<grid, threads, 0, st>>>(a, n_spans, items, x, y, perm, n_filled, window_len, status);
    else
      logits_adjust_scalar_kernel<T><<<grid, threads, 0, st>>>(a, n_spans, span, items, x, y, perm, n_filled, window_len, status);
    count_launch();
    return cuda_ok(cudaGetLastError());
  };
  return s.dtype == WEDLM_DTYPE_BF16 ? go(static_cast<const __nv_bfloat16*>(logits)) : go(static_cast<const float*>(logits));
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
