// Window attention for sequences that share the leading pages of their cache (answers drawn from one prompt, a common
// system prompt): the shared keys are read and multiplied once for all members of a group.
//
// Members of a group see the shared keys [0, S) without any mask, so their query rows can be stacked: a shared unit is one
// (group, KV head, 128-row tile of the members' packed rows) over S, an own unit one (sequence, KV head, row tile) over
// [S, P + W).  Every row is the join of its two parts by (m, l, O), the running maximum, sum and accumulator of a softmax.
// With W * G < 128 stacking is what fills the 128 rows of a tensor-core tile: at W = 16, G = 4 it halves the tiles, at
// W = 1 it divides them by up to 32.
//
// Five launches:
//   shared_rank_kernel           orders the sequences by group and finds, per sequence, how many leading pages equal those of its
//                                group's first member
//   shared_plan_kernel           one block: lengths of all streams and the cut of their tiles into equal runs
//   rope_stage_kernel<.., true>  beside the two: rotates and stages as for wedlm_window_attn, the queries in group order
//   attn_shared_kernel           the pieces; tile loop as in the plain window kernel
//   shared_merge_kernel          joins the pieces of every row that has more than one
#include <cuda.h>
#include <cudaTypedefs.h>
#include <math_constants.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace wedlm {
namespace {

constexpr int kTileN = 64;            // keys per tile (4 pages)
constexpr int kD = 128;               // head size
constexpr int kPage = 16;
static_assert(kTileN == 4 * kPage, "a tile is four pages");
constexpr int kThreadsT = 224;        // 4 softmax warps + MMA issue warp + two TMA producer warps
constexpr float kLazyRescaleLog2 = 8.0f;   // keep the old reference while the max grew by < 2^8

// shared memory map (bytes, base 1024-aligned)
constexpr uint32_t kOffQ = 0;                       // 2 halves x [128 rows x 128 B]
constexpr uint32_t kOffK = 32768;                   // 2 stages x 2 halves x [64 rows x 128 B]
constexpr uint32_t kOffV = 65536;                   // 2 stages x 2 halves x [64 rows x 128 B]
constexpr uint32_t kOffP = 98304;                   // [128 rows x 128 B] bf16 probabilities
constexpr uint32_t kOffBar = 114688;
constexpr uint32_t kSmemBytes = kOffBar + 256;
constexpr uint32_t kStageBytes = 16384;
constexpr uint32_t kHalfKV = 8192;
constexpr uint32_t kHalfQ = 16384;

enum Bar { Q_FULL = 0, K_FULL0, K_FULL1, V_FULL0, V_FULL1, S_FULL0, S_FULL1, O_DONE, P_READY, K_FREE0, K_FREE1,
           V_FREE0, V_FREE1, N_BARS };

using namespace ptx;

// ---------------------------------------------------------------------------------------------- the cut
// A stream is the keys of one unit row: entry r < B is the shared part of the group whose first member has rank r (empty
// for other ranks, and where sharing does not pay), entry B + r the own part of the sequence of rank r.  Per KV head its
// tiles are split into nch chunks of C tiles; the linear order of work is (entry, head, chunk, row tile, tile), so the row
// tiles of one chunk sit next to each other: CTAs that read the same keys do so at about the same time, and the later
// readers find them in L2.  An interval (entry, head, chunk, row tile) costs its tiles + kUnitCost (starting a piece: Q
// load, write-out), and the line is cut into one run of L per CTA, wherever that falls.  An interval that a cut goes through
// leaves several pieces; piece number = interval number + run number, which is unique.
// us of the whole call for 4 x 8 rows on 1040 shared keys, 32 x 16 on three prompts of 4099, 64 x 16 on 16 384, 61 x 1 on two of
// 8200 (the long ones under the power cap): kUnitCost 3 takes 26.6, 80.0, 387, 50.8, 1 takes 26.6, 86.7, 434, 50.0, 6 takes
// 28.6, 80.6, 376, 51.5.  kMinRun, the tiles of a run at the least: 2, 3, 8 instead of 4 take 25.3, 26.5, 28.8 for the first
// shape, which alone has fewer tiles than would give every CTA one such run; the others stay within 0.5 %.
// kMinShared: fewer shared tiles than this stay with the sequences.  8 x 16, 64 x 16 rows with up to 700 keys of their own: 3 tiles
// shared 34.6, 73.0, kept 28.7, 57.4; 4 tiles 30.7, 74.0 and 28.7, 58.5; 8 tiles 34.9, 78.9 and 29.3, 68.8; 15 tiles 36.0, 84.4
// and 30.7, 84.0: sharing costs a second piece per row and its merge, and pays from 16 tiles on (1024 keys) at 64 sequences.
constexpr int kUnitCost = 3;
constexpr int kMinRun = 4 + kUnitCost;
constexpr int kMinShared = 4;

struct Entry {
  int T, t_first;            // tiles, index of the first in the cache line of the sequence
  int mt, nch, C;            // row tiles, chunks, tiles per chunk
  int q0;                    // intervals of all earlier entries
  int slot_begin, slot_end;  // packed window slots of its rows
  int P;                     // own part: prefix length
  int b;                     // sequence whose block table is read
  int base;                  // linear position of the first interval
};

struct Plan {
  int total, L, n_runs;
};

struct SharedParams {
  int B, W, Hq, Hkv, G, W_t, max_pages, num_pages, max_prefix, n_ctas;
  float scale_log2;
  const int32_t* block_table;
  const int32_t* prefix_len;
  const int32_t* seq_at;       // [B] sequence of each rank
  const int32_t* group_key;    // [B] by rank: equal keys = one group
  const int32_t* same_pages;   // [B] by rank: leading pages equal to those of the group's first member
  int32_t* first_of;           // [B] by rank: rank of the group's first member
  Entry* entries;              // [2B]
  int32_t* start;              // [n_ctas] entry of each run's first position
  Plan* plan;
  __nv_bfloat16* out;
  float* part_o;               // [pieces][128][128]
  float2* part_ml;             // [pieces][128]
  int32_t* status;
};

// Positions are 32-bit: shapes whose line could be longer (SharedLayout::too_large) are not planned here.
__device__ __forceinline__ int head_cost(const Entry& e) { return e.mt * (e.T + e.nch * kUnitCost); }

// chunks of a stream, given the run length that one chunk should have
__device__ __forceinline__ void set_chunks(Entry& e, int L0) {
  const int want = e.mt > 1 ? max(e.T / L0, 1) : 1;
  e.C = (e.T + want - 1) / want;
  e.nch = (e.T + e.C - 1) / e.C;
}
__device__ __forceinline__ Entry shared_entry(const SharedParams& p, int first, int n, int T, int b) {
  Entry e;
  e.T = T; e.t_first = 0;
  e.mt = T > 0 ? (n * p.W + p.W_t - 1) / p.W_t : 0;
  e.slot_begin = first * p.W; e.slot_end = (first + n) * p.W;
  e.P = 0; e.b = b;
  e.nch = 0; e.C = 1; e.q0 = 0; e.base = 0;
  return e;
}
__device__ __forceinline__ Entry own_entry(const SharedParams& p, int rank, int T_shared, int P, int b) {
  Entry e;
  e.t_first = T_shared;
  e.T = (P + p.W + kTileN - 1) / kTileN - T_shared;
  e.mt = (p.W + p.W_t - 1) / p.W_t;
  e.slot_begin = rank * p.W; e.slot_end = (rank + 1) * p.W;
  e.P = P; e.b = b;
  e.nch = 0; e.C = 1; e.q0 = 0; e.base = 0;
  return e;
}

// The plan of up to 1024 sequences, one thread per rank with its two entries in registers: what follows from what goes
// through shared memory, so that only two loads depend on each other (seq_at, prefix_len).  4 us, beside the rotation.
constexpr int kPlanMost = 1024;
__global__ void __launch_bounds__(kPlanMost) shared_plan_small_kernel(SharedParams p) {
  __shared__ int key_s[kPlanMost], pages_s[kPlanMost], n_s[kPlanMost], warp_i[32], warp_q[32];
  __shared__ int warp_c[32], base_s[2 * kPlanMost];
  const int r = threadIdx.x, lane = r & 31, warp = r >> 5;
  grid_dependency_wait();
  grid_dependency_trigger();
  const bool in = r < p.B;
  const int b = in ? p.seq_at[r] : 0, key = in ? p.group_key[r] : -1, pages = in ? p.same_pages[r] : 0;
  const int P = in ? checked_prefix(p.prefix_len, b, p.max_prefix, p.status, true) : 0;
  key_s[r] = key;
  pages_s[r] = 0x7fffffff;
  n_s[r] = 0;
  __syncthreads();
  // rank of the group's first member: the last change of key up to here
  int first = in && (r == 0 || key_s[r - 1] != key) ? r : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, first, o);
    if (lane >= o) first = max(first, up);
  }
  if (lane == 31) warp_i[warp] = first;
  __syncthreads();
  for (int k = 0; k < warp; ++k) first = max(first, warp_i[k]);
  if (in) {
    atomicMin(&pages_s[first], pages);
    atomicAdd(&n_s[first], 1);
  }
  __syncthreads();
  Entry es{}, eo{};
  if (in) {
    int T = n_s[first] > 1 ? pages_s[first] / 4 : 0;
    if (T < kMinShared) T = 0;
    p.first_of[r] = first;
    es = shared_entry(p, first, n_s[first], first == r ? T : 0, b);
    eo = own_entry(p, r, T, P, b);
  }
  int sum = es.mt * (es.T + kUnitCost) + eo.mt * (eo.T + kUnitCost);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) warp_c[warp] = sum;
  __syncthreads();
  sum = 0;
  for (int k = 0; k < (int)blockDim.x / 32; ++k) sum += warp_c[k];
  const int L0 = max((sum * p.Hkv + p.n_ctas - 1) / p.n_ctas, kMinRun);
  int total = 0, q_total = 0;
  for (int part = 0; part < 2; ++part) {                            // prefix sums: all shared parts, then all own parts
    Entry& e = part ? eo : es;
    int cost = 0, q = 0;
    if (e.mt > 0) {
      set_chunks(e, L0);
      cost = head_cost(e) * p.Hkv;
      q = e.mt * e.nch * p.Hkv;
    }
    int c_inc = cost;
    int q_inc = q;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int c_up = __shfl_up_sync(0xffffffffu, c_inc, o);
      const int q_up = __shfl_up_sync(0xffffffffu, q_inc, o);
      if (lane >= o) { c_inc += c_up; q_inc += q_up; }
    }
    __syncthreads();
    if (lane == 31) { warp_c[warp] = c_inc; warp_q[warp] = q_inc; }
    __syncthreads();
    int c_all = 0, q_all = 0;
    for (int k = 0; k < (int)blockDim.x / 32; ++k) {
      if (k == warp) { c_inc += c_all; q_inc += q_all; }
      c_all += warp_c[k];
      q_all += warp_q[k];
    }
    e.base = total + c_inc - cost;
    e.q0 = q_total + q_inc - q;
    total += c_all;
    q_total += q_all;
    if (in) {
      base_s[part * p.B + r] = e.base;
      p.entries[part * p.B + r] = e;
    }
  }
  __syncthreads();
  const int L = max((total + p.n_ctas - 1) / p.n_ctas, kMinRun);
  const int n_runs = (total + L - 1) / L;
  if (r == 0) {
    Plan pl;
    pl.total = total; pl.L = L; pl.n_runs = n_runs;
    *p.plan = pl;
  }
  for (int c = r; c < n_runs; c += (int)blockDim.x) {
    const int pos = c * L;
    int lo = 0, hi = 2 * p.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (base_s[mid] <= pos) lo = mid; else hi = mid - 1;
    }
    p.start[c] = lo;           // an empty entry begins where its successor begins, so the last of equals has work
  }
}

// Any number of sequences, in steps through global memory.  One block of 1024 threads.
__global__ void __launch_bounds__(1024) shared_plan_kernel(SharedParams p) {
  __shared__ int warp_sum[32];
  __shared__ int warp_q[32];
  __shared__ int carry;
  __shared__ int carry_q;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dependency_wait();
  grid_dependency_trigger();
  const int n_entries = 2 * p.B;
  // shared tiles of every group, by the warp that meets its first member
  for (int r = warp; r < p.B; r += 32) {
    const int key = p.group_key[r];
    if (r > 0 && p.group_key[r - 1] == key) continue;
    int n = 0, pages = 0x7fffffff;
    for (int at = r;; at += 32) {
      const bool in = at + lane < p.B && p.group_key[at + lane] == key;
      int mine = in ? p.same_pages[at + lane] : 0x7fffffff;
      pages = min(pages, __reduce_min_sync(0xffffffffu, mine));
      const int here = __popc(__ballot_sync(0xffffffffu, in));
      n += here;
      if (here < 32) break;
    }
    int T = n > 1 ? pages / 4 : 0;
    if (T < kMinShared) T = 0;
    for (int at = r + lane; at < r + n; at += 32) {
      p.first_of[at] = r;
      Entry e = shared_entry(p, r, n, at == r ? T : 0, p.seq_at[r]);
      p.entries[at] = e;
      const int b = p.seq_at[at];
      e = own_entry(p, at, T, checked_prefix(p.prefix_len, b, p.max_prefix, p.status, true), b);
      p.entries[p.B + at] = e;
    }
  }
  __syncthreads();
  // all tiles -> the run length that one chunk should have
  int sum = 0;
  for (int i = tid; i < n_entries; i += 1024) sum += p.entries[i].mt * (p.entries[i].T + kUnitCost);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) warp_sum[warp] = sum;
  __syncthreads();
  sum = 0;
  for (int i = 0; i < 32; ++i) sum += warp_sum[i];
  const int L0 = max((sum * p.Hkv + p.n_ctas - 1) / p.n_ctas, kMinRun);
  __syncthreads();
  if (tid == 0) { carry = 0; carry_q = 0; }
  __syncthreads();
  // chunks, and the prefix sums of costs and interval counts
  for (int i0 = 0; i0 < n_entries; i0 += 1024) {
    const int i = i0 + tid;
    int cost = 0, q = 0;
    Entry e;
    if (i < n_entries) {
      e = p.entries[i];
      if (e.mt > 0) {
        set_chunks(e, L0);
        cost = head_cost(e) * p.Hkv;
        q = e.mt * e.nch * p.Hkv;
      }
    }
    int c_inc = cost;
    int q_inc = q;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int c_up = __shfl_up_sync(0xffffffffu, c_inc, o);
      const int q_up = __shfl_up_sync(0xffffffffu, q_inc, o);
      if (lane >= o) { c_inc += c_up; q_inc += q_up; }
    }
    if (lane == 31) { warp_sum[warp] = c_inc; warp_q[warp] = q_inc; }
    __syncthreads();
    int c_before = carry;
    int q_before = carry_q;
    for (int k = 0; k < warp; ++k) { c_before += warp_sum[k]; q_before += warp_q[k]; }
    if (i < n_entries) {
      e.base = c_before + c_inc - cost;
      e.q0 = q_before + q_inc - q;
      p.entries[i] = e;
    }
    __syncthreads();
    if (tid == 1023) { carry = c_before + c_inc; carry_q = q_before + q_inc; }
    __syncthreads();
  }
  const int total = carry;
  const int L = max((total + p.n_ctas - 1) / p.n_ctas, kMinRun);
  const int n_runs = (total + L - 1) / L;
  if (tid == 0) {
    Plan pl;
    pl.total = total; pl.L = L; pl.n_runs = n_runs;
    *p.plan = pl;
  }
  // last entry that begins at or before the run's position and is not empty
  for (int c = tid; c < n_runs; c += 1024) {
    const int pos = c * L;
    int lo = 0, hi = n_entries - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.entries[mid].base <= pos) lo = mid; else hi = mid - 1;
    }
    p.start[c] = lo;           // an empty entry begins where its successor begins, so the last of equals has work
  }
}

// one piece of work: key tiles [t0, t1) for the 128 packed rows from slot0 * G on of KV head g
struct Piece {
  int b, g, slot0, slot_end, t0, t1, kv_end, first_limit, piece;
  bool shared, once, whole;    // once: nobody else reads its keys; whole: the rows have no other piece, the result is final
};

struct Walk {
  Entry e;
  int i, h, k, m, off, run;    // entry, head, chunk, row tile, offset inside the interval
  int pos, end;
};

__device__ __forceinline__ void walk_init(Walk& w, const SharedParams& p, int cta) {
  const Plan pl = *p.plan;
  w.run = cta;
  w.pos = min(cta, pl.n_runs) * pl.L;
  w.end = min(w.pos + pl.L, pl.total);
  if (w.pos >= w.end) return;
  w.i = p.start[cta];
  w.e = p.entries[w.i];
  int rem = w.pos - w.e.base;
  const int per_head = head_cost(w.e);
  w.h = rem / per_head;
  rem -= w.h * per_head;
  const int per_chunk = w.e.mt * (w.e.C + kUnitCost);
  w.k = rem / per_chunk;
  rem -= w.k * per_chunk;
  const int cost = min(w.e.C, w.e.T - w.k * w.e.C) + kUnitCost;
  w.m = rem / cost;
  w.off = rem - w.m * cost;
}

__device__ __forceinline__ bool walk_next(Walk& w, const SharedParams& p, Piece& sg) {
  while (w.pos < w.end) {
    const int c0 = w.k * w.e.C;
    const int cost = min(w.e.C, w.e.T - c0) + kUnitCost;
    const int take = min(cost - w.off, w.end - w.pos);
    sg.shared = w.i < p.B;
    sg.once = w.e.mt == 1;
    sg.b = w.e.b;
    sg.g = w.h;
    sg.slot0 = w.e.slot_begin + w.m * p.W_t;
    sg.slot_end = w.e.slot_end;
    sg.first_limit = w.e.P + w.m * p.W_t;
    sg.kv_end = sg.shared ? w.e.T * kTileN : w.e.P + min(p.W, (w.m + 1) * p.W_t);
    const int horizon = (sg.kv_end + kTileN - 1) / kTileN;       // this row tile's last key may lie before the stream's
    sg.t0 = w.e.t_first + c0 + max(w.off - kUnitCost, 0);
    sg.t1 = min(w.e.t_first + c0 + max(w.off + take - kUnitCost, 0), horizon);
    sg.piece = w.e.q0 + (w.h * w.e.nch + w.k) * w.e.mt + w.m + w.run;
    sg.whole = !sg.shared && w.e.nch == 1 && w.off == 0 && take == cost && w.e.t_first == 0;
    w.pos += take;
    w.off += take;
    if (w.off == cost) {
      w.off = 0;
      if (++w.m == w.e.mt) {
        w.m = 0;
        if (++w.k == w.e.nch) {
          w.k = 0;
          if (++w.h == p.Hkv) {
            w.h = 0;
            if (w.pos < w.end) {
              do w.e = p.entries[++w.i]; while (w.e.mt == 0);
            }
          }
        }
      }
    }
    if (sg.t1 > sg.t0) return true;
  }
  return false;
}

// Persistent, two blocks per SM, a run of pieces each.  The tile loop is that of the plain window kernel: S = Q K^T and O += P V on
// the tensor cores, one row of the softmax per thread, the running maximum moved only when it grew by 2^8.  Roundings: the
// rotated query and P are bf16, because the tensor cores take no more (half a step each, 2^-8 relative; l sums the unrounded
// probabilities); scores, maxima, sums and O are fp32, and so are the pieces that the merge joins.
// Time: a chain per 64 keys (S, softmax, P, P V) behind which tensor pipe and exponentials are each about half busy, so neither
// binds.  64 x 16 rows over 16 384 shared and 1024 own keys: 284 GFLOP in 287 us at 1.65 GHz (0.99 PFLOP/s; the whole call 335 us
// at that clock, 376-388 under the power cap).  32 x 16 rows on three prompts of 4099: 37 GFLOP, empty halves of the own parts'
// tiles included, in 49 us (0.76 PFLOP/s).  61 x 1 rows over two prompts of 8200: 114 MB in 30 us (3.8 TB/s).
// The comparisons below were made in short runs at about 1.65 GHz.
// Probabilities in tensor memory instead of shared memory: 349 against 349 us of the whole call.
__global__ void __launch_bounds__(kThreadsT, 2)
attn_shared_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const SharedParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float c = p.scale_log2;

  const uint32_t sbase = smem_u32(smem);
  if ((sbase & 1023u) != 0u) {     // the swizzled layouts need a 1024-byte aligned base
    if (p.status && tid == 0) atomicOr(p.status, WEDLM_STATUS_WAIT_EXPIRED);
    grid_dependency_wait();        // the merge takes this kernel's end for the plan's
    return;
  }
  const uint32_t bars = sbase + kOffBar;
  auto bar = [&](int i) -> uint32_t { return bars + 8u * (uint32_t)i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + kOffBar + 112);
  volatile uint32_t* abort_flag = tmem_slot + 1;

  if (tid == 0) {
    for (int i = 0; i < N_BARS; ++i) mbar_init(bar(i), i == P_READY ? 128u : 1u);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(256u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t tmem_S = tmem_base;            // columns [0,64) and [64,128)
  const uint32_t tmem_O = tmem_base + 128u;     // columns [128,256)
  grid_dependency_wait();
  grid_dependency_trigger();

  // Every role walks the same list of pieces.  Tiles are numbered through all pieces of the CTA (tt): the stage
  // rings and the barrier phases run on without a break from one piece to the next.
  Walk w;
  walk_init(w, p, (int)blockIdx.x);
  Piece sg;

  if (warp == 4) {
    // ------------------------------------------------------------------ MMA issue warp
    // All lanes run the loop and wait on the barriers; one elected lane issues (see elect_one()).  The warp
    // never waits for an MMA to finish: completion is signalled to the consumers of the result (S_FULL,
    // O_DONE) and to the producer of the operands (K_FREE, V_FREE) through tcgen05.commit.
    const bool leader = elect_one();
    bool ok = true;
    const uint32_t idesc_qk = make_idesc(kTileN, false);
    const uint32_t idesc_pv = make_idesc(kD, true);
    auto issue_qk = [&](uint32_t tt) {
      const uint32_t st = tt & 1u;
      tc_fence_after();
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const uint64_t ad = make_desc(sbase + kOffQ + (kk >> 2) * kHalfQ + (kk & 3) * 32u, 16u, 1024u);
        const uint64_t bd = make_desc(sbase + kOffK + st * kStageBytes + (kk >> 2) * kHalfKV + (kk & 3) * 32u, 16u, 1024u);
        if (leader) umma(tmem_S + st * 64u, ad, bd, idesc_qk, kk > 0);
      }
      if (leader) {
        umma_commit(bar(S_FULL0 + st));
        umma_commit(bar(K_FREE0 + st));
      }
    };
    uint32_t gt = 0, n_seg = 0;
    while (ok && walk_next(w, p, sg)) {
      const int T = sg.t1 - sg.t0;
      ok = mbar_wait(bar(Q_FULL), n_seg & 1u);
      if (ok) ok = mbar_wait(bar(K_FULL0 + (gt & 1u)), (gt >> 1) & 1u);
      if (ok) issue_qk(gt);
      for (int t = 0; ok && t < T; ++t) {
        const uint32_t tt = gt + (uint32_t)t, st = tt & 1u, ph = (tt >> 1) & 1u;
        if (t + 1 < T) {
          // S[(tt+1)&1] was last read by the softmax of tile tt-1, whose P_READY we saw one iteration ago
          ok = mbar_wait(bar(K_FULL0 + (st ^ 1u)), ((tt + 1u) >> 1) & 1u);
          if (!ok) break;
          issue_qk(tt + 1u);
        }
        ok = mbar_wait(bar(P_READY), tt & 1u);
        if (!ok) break;
        ok = mbar_wait(bar(V_FULL0 + st), ph);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t ad = make_desc(sbase + kOffP + j * 32u, 16u, 1024u);
          const uint64_t bd = make_desc(sbase + kOffV + st * kStageBytes + j * 2048u, kHalfKV, 1024u);
          if (leader) umma(tmem_O, ad, bd, idesc_pv, (t > 0) || (j > 0));
        }
        if (leader) {
          umma_commit(bar(O_DONE));
          umma_commit(bar(V_FREE0 + st));
        }
      }
      gt += (uint32_t)T;
      ++n_seg;
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      if (p.status) atomicOr(p.status, WEDLM_STATUS_WAIT_EXPIRED);
    }
  } else if (warp >= 5) {
    // ------------------------------------------------------------------ TMA producer warps
    // Warp 5 streams the K tiles (and loads Q), warp 6 the V tiles; each refills a stage as soon as the
    // MMAs that read it have completed.  A tile is 8 copies of 2 KB (4 pages x 2 column halves): lanes
    // 0..7 each look up their page and issue their copy, so a tile leaves in one warp instruction.
    const bool is_k = (warp == 5);
    // Keys that one row tile alone reads are the first to leave L2, which then keeps the pieces' sums for the merge and the
    // keys that others read again: 61 single tokens on two prompts of 8200 57.4 -> 52.7 us; for all keys, 64 answers over
    // 16384 shared keys go from 336 to 410 us.
    const uint64_t once = l2_evict_first();
    bool ok = true;
    const int oob_row = p.num_pages * p.Hkv * kPage;        // a row coordinate past the end: zero fill
    const int pg = (lane >> 1) & 3, half = lane & 1;
    const uint32_t lane_dst = (uint32_t)pg * 2048u + (uint32_t)half * kHalfKV;
    auto wait_all = [&](uint32_t barrier, uint32_t parity) -> bool {      // lane 0 waits, the warp follows
      int good = 1;
      if (lane == 0) good = mbar_wait(barrier, parity) ? 1 : 0;
      return __shfl_sync(0xffffffffu, good, 0) != 0;
    };
    const CUtensorMap* map = is_k ? &tm_k : &tm_v;
    const uint32_t stage0 = sbase + (is_k ? kOffK : kOffV);
    const int full0 = is_k ? K_FULL0 : V_FULL0, free0 = is_k ? K_FREE0 : V_FREE0;
    uint32_t gt = 0, n_seg = 0;
    while (ok && walk_next(w, p, sg)) {
      const int T = sg.t1 - sg.t0;
      // TMA row coordinate of this lane's page of tile t of the unit (same for K and V)
      auto page_row = [&](int t) -> int {
        const int key0 = t * kTileN + pg * kPage;
        const int lp = key0 / kPage;
        int pp = -1;
        if (lp < p.max_pages) pp = p.block_table[(size_t)sg.b * p.max_pages + lp];
        if (pp < 0 || pp >= p.num_pages) {
          if (is_k && key0 < sg.kv_end && p.status) atomicOr(p.status, lp < p.max_pages ? WEDLM_STATUS_BAD_PAGE : WEDLM_STATUS_BAD_LENGTH);
          return oob_row;
        }
        return (pp * p.Hkv + sg.g) * kPage;
      };
      if (is_k) {
        // the Q tile may only be replaced once every Q K^T of the previous piece has completed
        if (n_seg > 0) ok = wait_all(bar(K_FREE0 + ((gt - 1u) & 1u)), ((gt - 1u) >> 1) & 1u);
        if (!ok) break;
        if (lane == 0) {
          // Q tile: two 64-element halves of [W_t packed slots x G heads] rows
          mbar_expect_tx(bar(Q_FULL), 2u * kHalfQ);
          tma_load_3d(sbase + kOffQ, &tm_q, 0, sg.g * p.G, sg.slot0, bar(Q_FULL));
          tma_load_3d(sbase + kOffQ + kHalfQ, &tm_q, 64, sg.g * p.G, sg.slot0, bar(Q_FULL));
        }
      }
      int y_next = page_row(sg.t0);
      for (int t = 0; ok && t < T; ++t) {
        const uint32_t tt = gt + (uint32_t)t, st = tt & 1u;
        const int y = y_next;
        if (t + 1 < T) y_next = page_row(sg.t0 + t + 1);      // table entry of the next tile, used one iteration later
        if (tt >= 2u) ok = wait_all(bar(free0 + st), ((tt - 2u) >> 1) & 1u);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(bar(full0 + st), kStageBytes);
        __syncwarp();
        if (lane < 8) {
          const uint32_t dst = stage0 + st * kStageBytes + lane_dst;
          if (sg.once) tma_load_2d(dst, map, half * 64, y, bar(full0 + st), once);
          else tma_load_2d(dst, map, half * 64, y, bar(full0 + st));
        }
      }
      gt += (uint32_t)T;
      ++n_seg;
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      if (p.status) atomicOr(p.status, WEDLM_STATUS_WAIT_EXPIRED);
    }
  } else {
    // ------------------------------------------------------------------ softmax warps: one row per thread
    const uint32_t lane_sel = (uint32_t)(warp * 32) << 16;
    const int r = tid;                                         // row of the 128-row tile
    bool ok = true;
    uint32_t gt = 0;
    while (ok && walk_next(w, p, sg)) {
      const int T = sg.t1 - sg.t0;
      const int kv_end = sg.kv_end;
      const int slot = sg.slot0 + r / p.G;                     // packed window slot
      const bool row_valid = slot < sg.slot_end;
      // last visible key (inclusive): rows of a shared part see all of it
      const int limit = !row_valid ? -1 : (sg.shared ? kv_end - 1 : sg.first_limit + r / p.G);
      const int mask_from = sg.shared ? kv_end : sg.first_limit + 1;     // tiles that end at or before this need no mask
      float m_ref = -CUDART_INF_F;                             // reference maximum (raw score units)
      float l = 0.f;
      for (int t = 0; t < T; ++t) {
        const uint32_t tt = gt + (uint32_t)t, st = tt & 1u, ph = (tt >> 1) & 1u;
        ok = mbar_wait(bar(S_FULL0 + st), ph);
        if (!ok) break;
        tc_fence_after();
        uint32_t raw[64];
        {
          uint32_t (&lo)[32] = *reinterpret_cast<uint32_t (*)[32]>(&raw[0]);
          uint32_t (&hi)[32] = *reinterpret_cast<uint32_t (*)[32]>(&raw[32]);
          tmem_ld32(tmem_S + lane_sel + st * 64u, lo);
          tmem_ld32(tmem_S + lane_sel + st * 64u + 32u, hi);
          tmem_wait_ld();
        }
        const int tile0 = (sg.t0 + t) * kTileN;
        const bool need_mask = tile0 + kTileN > mask_from;                    // block-uniform
        float m_tile;
        if (need_mask) {
          m_tile = -CUDART_INF_F;
#pragma unroll
          for (int cc = 0; cc < 64; ++cc) {
            const int key = tile0 + cc;
            float x = __uint_as_float(raw[cc]);
            x = (key <= limit && key < kv_end) ? x : -CUDART_INF_F;
            raw[cc] = __float_as_uint(x);
            m_tile = fmaxf(m_tile, x);
          }
        } else {
          float m4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
          for (int cc = 0; cc < 64; cc += 8) {
            m4[0] = max3(m4[0], __uint_as_float(raw[cc + 0]), __uint_as_float(raw[cc + 1]));
            m4[1] = max3(m4[1], __uint_as_float(raw[cc + 2]), __uint_as_float(raw[cc + 3]));
            m4[2] = max3(m4[2], __uint_as_float(raw[cc + 4]), __uint_as_float(raw[cc + 5]));
            m4[3] = max3(m4[3], __uint_as_float(raw[cc + 6]), __uint_as_float(raw[cc + 7]));
          }
          m_tile = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
        }
        // lazy reference: only move it when the maximum grew by more than 2^kLazyRescaleLog2
        float alpha = 1.f;
        bool moved = false;
        if (m_tile > -CUDART_INF_F && (m_ref == -CUDART_INF_F || (m_tile - m_ref) * c > kLazyRescaleLog2)) {
          alpha = (m_ref == -CUDART_INF_F) ? 0.f : exp2f((m_ref - m_tile) * c);
          m_ref = m_tile;
          moved = true;
        }
        const float neg_mc = (m_ref == -CUDART_INF_F) ? 0.f : -m_ref * c;
        // p = 2^(s*c - m*c): the scale and the reference are folded into one packed FMA per two scores
        const unsigned long long C2 = pack2(c, c), NM2 = pack2(neg_mc, neg_mc);
        unsigned long long sumA = pack2(0.f, 0.f), sumB = sumA;
        uint32_t pk[32];
#pragma unroll
        for (int cc = 0; cc < 64; cc += 4) {
          float a0, a1, b0, b1;
          unpack2(fma2(pack2(__uint_as_float(raw[cc]), __uint_as_float(raw[cc + 1])), C2, NM2), a0, a1);
          unpack2(fma2(pack2(__uint_as_float(raw[cc + 2]), __uint_as_float(raw[cc + 3])), C2, NM2), b0, b1);
          const float p0 = ex2_approx(a0), p1 = ex2_approx(a1), p2 = ex2_approx(b0), p3 = ex2_approx(b1);
          sumA = add2(sumA, pack2(p0, p1));
          sumB = add2(sumB, pack2(p2, p3));
          pk[cc >> 1] = pack_bf16(p0, p1);
          pk[(cc >> 1) + 1] = pack_bf16(p2, p3);
        }
        float sum, sum2;
        {
          float x0, x1;
          unpack2(add2(sumA, sumB), x0, x1);
          sum = x0;
          sum2 = x1;
        }
        l = l * alpha + (sum + sum2);
        // P buffer and O are free / stable once P V of the previous tile has completed (at the first tile of a
        // later piece that was waited for when the previous piece's result was read)
        if (t > 0) {
          ok = mbar_wait(bar(O_DONE), (tt - 1u) & 1u);
          if (!ok) break;
          tc_fence_after();
          if (__any_sync(0xffffffffu, moved)) {
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              uint32_t o[32];
              tmem_ld32(tmem_O + lane_sel + ch * 32u, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st32(tmem_O + lane_sel + ch * 32u, o);
            }
            tmem_wait_st();
          }
        }
        // bf16 P row into the 128-byte-swizzled K-major tile: 16-byte chunk j of row r sits at j ^ (r & 7)
        {
          uint8_t* prow = smem + kOffP + r * 128;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint4 v = make_uint4(pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]);
            *reinterpret_cast<uint4*>(prow + ((j ^ (r & 7)) << 4)) = v;
          }
        }
        // last tile of the unit: V rows of keys beyond the horizon may hold anything (0 * NaN = NaN): zero them
        if (kv_end - tile0 < kTileN) {
          ok = mbar_wait(bar(V_FULL0 + st), ph);
          if (!ok) break;
          const int first_bad = kv_end - tile0;
          uint8_t* vst = smem + kOffV + st * kStageBytes;
          for (int idx = tid; idx < (kTileN - first_bad) * 16; idx += 128) {      // 16 x 16-byte chunks per key row
            const int row = first_bad + idx / 16, ch = idx % 16;
            *reinterpret_cast<uint4*>(vst + (ch >> 3) * kHalfKV + row * 128 + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
        }
        fence_async_smem();
        tc_fence_before();
        mbar_arrive(bar(P_READY));
      }
      if (!ok) break;
      gt += (uint32_t)T;
      ok = mbar_wait(bar(O_DONE), (gt - 1u) & 1u);
      if (!ok) break;
      tc_fence_after();
      const float inv = l > 0.f ? 1.f / l : 0.f;
      size_t orow = 0;
      if (sg.whole && row_valid) {
        const int rank = slot / p.W;
        orow = (((size_t)p.seq_at[rank] * p.W + (slot - rank * p.W)) * p.Hq + sg.g * p.G + r % p.G) * kD;
      }
      const size_t prow = (size_t)sg.piece * 128 + r;
#pragma unroll 1
      for (int ch = 0; ch < 4; ++ch) {
        uint32_t o[32];
        tmem_ld32(tmem_O + lane_sel + ch * 32u, o);
        tmem_wait_ld();
        if (!row_valid) continue;
        if (sg.whole) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + orow + ch * 32);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            uint4 v;
            v.x = pack_bf16(__uint_as_float(o[8 * q4 + 0]) * inv, __uint_as_float(o[8 * q4 + 1]) * inv);
            v.y = pack_bf16(__uint_as_float(o[8 * q4 + 2]) * inv, __uint_as_float(o[8 * q4 + 3]) * inv);
            v.z = pack_bf16(__uint_as_float(o[8 * q4 + 4]) * inv, __uint_as_float(o[8 * q4 + 5]) * inv);
            v.w = pack_bf16(__uint_as_float(o[8 * q4 + 6]) * inv, __uint_as_float(o[8 * q4 + 7]) * inv);
            dst[q4] = v;
          }
        } else {
          uint4* dst = reinterpret_cast<uint4*>(p.part_o + prow * kD + ch * 32);
#pragma unroll
          for (int q4 = 0; q4 < 8; ++q4) dst[q4] = make_uint4(o[4 * q4], o[4 * q4 + 1], o[4 * q4 + 2], o[4 * q4 + 3]);
        }
      }
      if (row_valid && !sg.whole)
        p.part_ml[prow] = make_float2((m_ref == -CUDART_INF_F) ? -CUDART_INF_F : m_ref * c, l);      // log2 domain
      // the accumulator has been read: order those loads before the next piece's first P V overwrites it
      tc_fence_before();
    }
    if (!ok) {
      *abort_flag = 1;
      if (p.status) atomicOr(p.status, WEDLM_STATUS_WAIT_EXPIRED);
    }
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0) {
    // a wait expired: give copies that may still be in flight a bounded time (about 0.2 ms) to land
    // before this CTA's shared memory is handed to another CTA
    for (int it = 0; it < 200; ++it) __nanosleep(1000);
  }
  __syncthreads();
  if (warp == 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
  }
}

// Joins the pieces of every row that has more than one.  One block per (rank, KV head) and kMergeRows query rows, half a warp
// per row: it works out from the plan which pieces the row has, of the shared and of the own part, and takes up to
// four at a time, with their (m, l) and accumulators on their way together.  m is in the log2 domain.
// Bound by the way to the sums: 4 us for 1024 rows, 13 us for 16 384 rows of about four pieces (33 MB, partly out of HBM).
constexpr int kMergeRows = 16, kMergeWarps = 8;       // 32, 64 rows: 359, 364 us of the whole call where 16 takes 334 (64 x 16k)

__global__ void __launch_bounds__(32 * kMergeWarps) shared_merge_kernel(const SharedParams p, int n_parts) {
  __shared__ Entry entry_s[2];
  const int unit = blockIdx.x / n_parts, row0 = (blockIdx.x - unit * n_parts) * kMergeRows;
  const int rank = unit / p.Hkv, g = unit - rank * p.Hkv;
  const int tid = threadIdx.x, half = tid >> 4, d = (tid & 15) * 8;  // (eight columns per thread)
  grid_dependency_wait();
  const int L = p.plan->L;
  if (tid < 2) entry_s[tid] = p.entries[tid == 0 ? p.first_of[rank] : p.B + rank];
  __syncthreads();
  const int row_end = min(row0 + kMergeRows, p.W * p.G);
  for (int row = row0 + half; row < row_end; row += 2 * kMergeWarps) {
    const int i = row / p.G, hg = row - i * p.G;
    float acc[8] = {};
    float m = -CUDART_INF_F, l = 0.f;
    int n = 0;
    size_t at[4] = {0, 0, 0, 0};
    auto join = [&]() {                                             // the collected pieces into the running result
      float2 ml[4];
      float4 o[4][2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        ml[u] = make_float2(-CUDART_INF_F, 0.f);
        o[u][0] = o[u][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (u < n) {
          ml[u] = p.part_ml[at[u]];
          o[u][0] = __ldcs(reinterpret_cast<const float4*>(p.part_o + at[u] * kD + d));
          o[u][1] = __ldcs(reinterpret_cast<const float4*>(p.part_o + at[u] * kD + d + 4));
        }
      }
      const float m_new = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m);
      if (m_new > -CUDART_INF_F) {
        const float keep = exp2f(m - m_new);                        // 0 where nothing was there
        l *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= keep;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float w = exp2f(ml[u].x - m_new);
          l += w * ml[u].y;
          if (w != 0.f) {
            acc[0] += w * o[u][0].x; acc[1] += w * o[u][0].y; acc[2] += w * o[u][0].z; acc[3] += w * o[u][0].w;
            acc[4] += w * o[u][1].x; acc[5] += w * o[u][1].y; acc[6] += w * o[u][1].z; acc[7] += w * o[u][1].w;
          }
        }
        m = m_new;
      }
      n = 0;
    };
    bool direct = false;
    for (int part = 0; part < 2; ++part) {
      const Entry& e = entry_s[part];
      if (e.mt == 0) continue;
      const int slot = part == 0 ? rank * p.W + i - e.slot_begin : i;           // among the entry's packed slots
      const int mt = slot / p.W_t, in_tile = (slot - mt * p.W_t) * p.G + hg;
      const int horizon = ((part == 0 ? e.T * kTileN : e.P + min(p.W, (mt + 1) * p.W_t)) + kTileN - 1) / kTileN;
      for (int k = 0; k < e.nch; ++k) {
        const int c0 = k * e.C;
        const int cost = min(e.C, e.T - c0) + kUnitCost;
        const int a = e.base + g * head_cost(e) + k * e.mt * (e.C + kUnitCost) + mt * cost;
        const int r0 = a / L, r1 = (a + cost - 1) / L;
        if (part == 1 && e.nch == 1 && r0 == r1 && e.t_first == 0) { direct = true; break; }    // written by the CTA that held it
        const int q = e.q0 + (g * e.nch + k) * e.mt + mt;
        for (int r = r0; r <= r1; ++r) {
          const int o0 = max(r * L - a, 0), o1 = min((r + 1) * L - a, cost);
          const int t0 = e.t_first + c0 + max(o0 - kUnitCost, 0);
          const int t1 = min(e.t_first + c0 + max(o1 - kUnitCost, 0), horizon);
          if (t1 <= t0) continue;
          const size_t from = (size_t)(q + r) * 128 + in_tile;
          if (n == 0) at[0] = from;
          else if (n == 1) at[1] = from;
          else if (n == 2) at[2] = from;
          else at[3] = from;
          if (++n == 4) join();
        }
      }
    }
    if (direct) continue;
    join();
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint4 v;
    v.x = pack_bf16(acc[0] * inv, acc[1] * inv);
    v.y = pack_bf16(acc[2] * inv, acc[3] * inv);
    v.z = pack_bf16(acc[4] * inv, acc[5] * inv);
    v.w = pack_bf16(acc[6] * inv, acc[7] * inv);
    *reinterpret_cast<uint4*>(p.out + (((size_t)entry_s[1].b * p.W + i) * p.Hq + g * p.G + hg) * kD + d) = v;
  }
}

// ---------------------------------------------------------------------------------------------- host
PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  if (fn) return fn;
  void* ptr = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
  return fn;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

SharedLayout plan_shared(const wedlm_config_t* c) {
  SharedLayout s{};
  const size_t B = c->batch, W = c->window, Hkv = c->n_kv_heads;
  const size_t w_t = 128 / (c->n_q_heads / c->n_kv_heads);
  s.n_ctas = 2 * device_sm_count();
  // every piece is an interval or the part of one behind a cut; a chunk is at least a run long, so chunking adds at most
  // one interval per run
  const size_t units = Hkv * ((B * W + w_t - 1) / w_t + B / 2 + B * ((W + w_t - 1) / w_t));
  s.n_pieces = units + 2 * (size_t)s.n_ctas + 2;
  const size_t tiles = ((size_t)c->max_prefix_len + W + kTileN - 1) / kTileN + 1;      // of one unit, at most
  s.too_large = units * (tiles + kUnitCost) + (size_t)s.n_ctas * (kUnitCost + kMinRun) * 2 > 0x3fffffffULL ||
                B * Hkv * ((W * (c->n_q_heads / c->n_kv_heads) + kMergeRows - 1) / kMergeRows) > 0x7fffffffULL;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes ? bytes : 1); return o; };
  s.off_q = take((B * W > w_t ? B * W : w_t) * c->n_q_heads * kD * 2);
  s.off_rank = take(4 * B * sizeof(int32_t));
  s.off_entries = take(2 * B * sizeof(Entry));
  s.off_start = take((size_t)s.n_ctas * sizeof(int32_t));
  s.off_plan = take(sizeof(Plan));
  s.off_ml = take(s.n_pieces * 128 * sizeof(float2));
  s.off_o = take(s.n_pieces * 128 * kD * sizeof(float));
  s.total = at;
  return s;
}

int launch_attn_shared(const Shape& s, const SharedLayout& lay, const int32_t* group, const void* q, const void* k, const void* v,
                       void* k_cache, void* v_cache, const int32_t* block_table, const int32_t* prefix_len,
                       const int32_t* pos_ids, void* out, int32_t* kv_slot_idx, void* workspace, int32_t* status,
                       cudaStream_t st) {
  auto encode = get_encode();
  if (!encode) return WEDLM_ERR_CUDA;
  char* ws = static_cast<char*>(workspace);
  SharedParams p;
  p.B = s.B; p.W = s.W; p.Hq = s.Hq; p.Hkv = s.Hkv; p.G = s.G; p.W_t = 128 / s.G;
  p.max_pages = s.max_pages; p.num_pages = s.num_pages; p.max_prefix = s.max_prefix; p.n_ctas = lay.n_ctas;
  p.scale_log2 = s.scale * 1.4426950408889634f;
  p.block_table = block_table; p.prefix_len = prefix_len;
  int32_t* ranks = reinterpret_cast<int32_t*>(ws + lay.off_rank);
  p.seq_at = ranks; p.group_key = ranks + s.B; p.same_pages = ranks + 2 * (size_t)s.B; p.first_of = ranks + 3 * (size_t)s.B;
  p.entries = reinterpret_cast<Entry*>(ws + lay.off_entries);
  p.start = reinterpret_cast<int32_t*>(ws + lay.off_start);
  p.plan = reinterpret_cast<Plan*>(ws + lay.off_plan);
  p.out = (__nv_bfloat16*)out;
  p.part_o = reinterpret_cast<float*>(ws + lay.off_o);
  p.part_ml = reinterpret_cast<float2*>(ws + lay.off_ml);
  p.status = status;
  void* q_rot = ws + lay.off_q;

  CUtensorMap tm_q, tm_k, tm_v;
  {
    // rotated queries [B*W packed slots][Hq][D] as (D, Hq, slots); box = (64, G, 128 / G).  Rows past the last slot fill
    // with zeros.
    const long long slots = (long long)s.B * s.W;
    cuuint64_t dims[3] = {(cuuint64_t)kD, (cuuint64_t)s.Hq, (cuuint64_t)(slots > p.W_t ? slots : p.W_t)};
    cuuint64_t strides[2] = {(cuuint64_t)kD * 2, (cuuint64_t)s.Hq * kD * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)s.G, (cuuint32_t)p.W_t};
    cuuint32_t estr[3] = {1, 1, 1};
    if (encode(&tm_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, q_rot, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return WEDLM_ERR_CUDA;
  }
  for (int which = 0; which < 2; ++which) {
    // cache [num_pages][Hkv][16][D] as (D, rows); box = one page of one head, 64 elements wide
    cuuint64_t dims[2] = {(cuuint64_t)kD, (cuuint64_t)s.num_pages * s.Hkv * kPage};
    cuuint64_t strides[1] = {(cuuint64_t)kD * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)kPage};
    cuuint32_t estr[2] = {1, 1};
    if (encode(which ? &tm_v : &tm_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, which ? v_cache : k_cache, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return WEDLM_ERR_CUDA;
  }
  // the opt-in to large dynamic shared memory is per device: done once for each device ordinal
  {
    static bool attr_done[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return WEDLM_ERR_CUDA;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
      if (cudaFuncSetAttribute(attn_shared_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes) != cudaSuccess)
        return WEDLM_ERR_CUDA;
      if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
  }
  // Each launch behind the first may start while its predecessor runs: it waits for it where it first reads what that wrote.
  // The rotation reads nothing of the plan and runs beside it.
  int rc = launch_shared_ranks(s, SharedRanks{group, ranks, ranks + s.B, ranks + 2 * (size_t)s.B}, block_table, prefix_len, st);
  if (rc != WEDLM_OK) return rc;
  // (320 threads where they do: 4 sequences take 26.6 us with 320 and 29.0 with 1024, 61 sequences 50.8 and 54.2)
  if (!launch_behind(s.B <= kPlanMost ? shared_plan_small_kernel : shared_plan_kernel, 1, s.B <= 320 ? 320 : kPlanMost, 0, st, p))
    return WEDLM_ERR_CUDA;
  rc = launch_rope_stage(s, q, k, v, q_rot, k_cache, v_cache, block_table, prefix_len, pos_ids, nullptr, kv_slot_idx, nullptr, status,
                         st, group);
  if (rc != WEDLM_OK) return rc;
  const int n_parts = (s.W * s.G + kMergeRows - 1) / kMergeRows;
  const bool ok = launch_behind(attn_shared_kernel, (unsigned)lay.n_ctas, kThreadsT, kSmemBytes, st, tm_q, tm_k, tm_v, p) &&
                  launch_behind(shared_merge_kernel, (unsigned)(s.B * s.Hkv * n_parts), 32 * kMergeWarps, 0, st, p, n_parts);
  if (!ok) return WEDLM_ERR_CUDA;
  count_launch(3);
  return cuda_ok(cudaGetLastError());
}

}  // namespace wedlm
