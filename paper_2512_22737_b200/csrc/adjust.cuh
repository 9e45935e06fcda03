// Rules that differ from request to request and change logits before the softmax: penalties for tokens the sequence
// already has, biases of single tokens, and allowed-token masks.  Device view of wedlm_adjust_t and the arithmetic of
// one token, shared by every kernel that applies them.
#pragma once
#include "common.cuh"

namespace wedlm {

// Words of a token bitmap: one bit per token, rows padded to 16 bytes.
__host__ __device__ constexpr int token_bits_words(int vocab) { return (vocab + 127) / 128 * 4; }

struct AdjustView {
  uint32_t* bits;               // [B][words] or NULL: tokens that have a record
  int2* record;                 // [B][V]: (2 * generated count | in the prompt, bits of the bias)
  const float* repetition;      // [B] or NULL
  const float* presence;
  const float* frequency;
  const uint32_t* allowed;      // [n_masks][words] or NULL
  const int32_t* mask_index;    // [B][W] logical slots
  int words, n_masks, V, W, count_fills;
};

inline AdjustView adjust_view(const wedlm_config_t* cfg, const wedlm_adjust_t* a) {
  AdjustView v;
  v.bits = a->token_bits;
  v.record = reinterpret_cast<int2*>(a->token_record);
  v.repetition = a->repetition; v.presence = a->presence; v.frequency = a->frequency;
  v.allowed = a->allowed; v.mask_index = a->mask_index;
  v.words = token_bits_words(cfg->vocab); v.n_masks = a->n_masks; v.V = cfg->vocab; v.W = cfg->window;
  v.count_fills = a->count_fills;
  return v;
}

// The rules of one window row: null bitmaps mean "no token touched" and "every token allowed".
struct RowRules {
  const uint32_t* touched;
  const uint32_t* allowed;
  const int2* record;
  float repetition, inverse;    // factor of logits <= 0 and of logits > 0 of a token that the sequence has
  float presence, frequency;
};

// The rules of a sequence, without a mask.
__device__ __forceinline__ RowRules history_rules(const AdjustView& a, int b) {
  RowRules r;
  r.touched = a.bits ? a.bits + (size_t)b * a.words : nullptr;
  r.record = a.record ? a.record + (size_t)b * a.V : nullptr;
  r.repetition = a.repetition ? a.repetition[b] : 1.f;
  r.inverse = __frcp_rn(r.repetition);
  r.presence = a.presence ? a.presence[b] : 0.f;
  r.frequency = a.frequency ? a.frequency[b] : 0.f;
  r.allowed = nullptr;
  return r;
}

__device__ __forceinline__ RowRules row_rules(const AdjustView& a, int b, int slot, int32_t* status) {
  RowRules r = history_rules(a, b);
  if (a.mask_index) {
    const int m = a.mask_index[(size_t)b * a.W + slot];
    if (m >= a.n_masks) {                                   // no such mask: flagged, the row is left unconstrained
      if (status) atomicOr(status, WEDLM_STATUS_BAD_TOKEN);
    } else if (m >= 0) {
      r.allowed = a.allowed + (size_t)m * a.words;
    }
  }
  return r;
}

// The rules on one touched token come down to x * scale + offset: one rounding each for the inverse and the offset's terms,
// one for the sum.  The same function serves every kernel, so equal logits with equal records stay equal everywhere.
__device__ __forceinline__ float rule_offset(int2 rec, const RowRules& r) {
  const int c = rec.x >> 1;
  const float off = __int_as_float(rec.y);
  return c > 0 ? off - fmaf(r.frequency, (float)c, r.presence) : off;
}
__device__ __forceinline__ float apply_rules(float x, bool seen, float offset, const RowRules& r) {
  return fmaf(x, seen ? (x > 0.f ? r.inverse : r.repetition) : 1.f, offset);
}
__device__ __forceinline__ float adjust_token(float x, int2 rec, const RowRules& r) {
  return apply_rules(x, rec.x != 0, rule_offset(rec, r), r);
}

// The same for any token of the row, with its bits looked up here.
template <typename T>
__device__ __forceinline__ float adjusted_logit(const T* __restrict__ row, int v, const RowRules& r) {
  const uint32_t bit = 1u << (v & 31);
  if (r.allowed && !(r.allowed[v >> 5] & bit)) return __int_as_float(0xff800000);
  const float x = ld_as_float(row, (size_t)v);
  if (r.touched && (r.touched[v >> 5] & bit)) return adjust_token(x, r.record[v], r);
  return x;
}

// A record counts only if its token's bit is set, and a history is emptied by clearing its bits, so what a record behind a
// clear bit holds is anything.  Writers therefore see the bit set, or set it, before they change the record: until the first
// of them has set it nobody else changes the record, so the one whose atomic found the bit clear knows what was left there and
// makes it count for nothing.  (Release and acquire on the word of bits order the look at the record before the others' changes.)
__device__ __forceinline__ uint32_t ld_bits(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t or_bits(uint32_t* p, uint32_t v) {
  uint32_t old;
  asm volatile("atom.acq_rel.gpu.global.or.b32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
  return old;
}

// A token that was written into a sequence: one more generated occurrence.  Sums of integers: the order does not matter.
__device__ __forceinline__ void count_token(const AdjustView& a, int b, int token) {
  if ((unsigned)token >= (unsigned)a.V) return;
  int2* const rec = a.record + (size_t)b * a.V + token;
  uint32_t* const word = a.bits + (size_t)b * a.words + (token >> 5);
  const uint32_t bit = 1u << (token & 31);
  const uint32_t left = *reinterpret_cast<volatile uint32_t*>(&rec->x);
  uint32_t add = 2u;
  if (!(ld_bits(word) & bit) && !(or_bits(word, bit) & bit)) {
    add -= left;
    rec->y = 0;
  }
  atomicAdd(reinterpret_cast<uint32_t*>(&rec->x), add);
}

// Brings what count_token looks at closer.
__device__ __forceinline__ void prefetch_count(const AdjustView& a, int b, int token) {
  if ((unsigned)token >= (unsigned)a.V) return;
  asm volatile("prefetch.global.L2 [%0];" ::"l"(a.record + (size_t)b * a.V + token));
  asm volatile("prefetch.global.L2 [%0];" ::"l"(a.bits + (size_t)b * a.words + (token >> 5)));
}

int launch_conf_adjusted_pass1(const Shape& s, const AdjustView& a, int n_chunks, int chunk, const void* logits,
                               const int32_t* perm, const int32_t* n_filled, const int32_t* window_len, void* partials,
                               void* list_ws, int32_t* status, cudaStream_t st);
size_t conf_adjusted_list_bytes(int B, int n_chunks);
size_t conf_adjusted_workspace_bytes(const wedlm_config_t* cfg);
int launch_logits_adjust(const Shape& s, const AdjustView& a, const void* logits, void* out, const int32_t* perm,
                         const int32_t* n_filled, const int32_t* window_len, int32_t* status, cudaStream_t st);
int launch_history_add(const Shape& s, const AdjustView& a, int length, const int32_t* tokens, const int32_t* count,
                       int in_prompt, int32_t* status, cudaStream_t st);
int launch_history_bias(const Shape& s, const AdjustView& a, int n_ids, const int32_t* ids, const float* values,
                        int32_t* status, cudaStream_t st);
int launch_confidence_adjusted(const Shape& s, const wedlm_config_t* cfg, const AdjustView& a, const void* logits,
                               const int32_t* perm, const int32_t* n_filled, const int32_t* n_commit, int32_t* window_tokens,
                               uint8_t* filled, int32_t* prefix_len, int32_t* window_len, int32_t* remaining_budget,
                               int32_t* argmax, float* maxprob, float* entropy, float* lse, int32_t* committed_tokens,
                               int32_t* committed_count, int32_t* filled_count, void* workspace, int32_t* status,
                               cudaStream_t st);

}  // namespace wedlm
