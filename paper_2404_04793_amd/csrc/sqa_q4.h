// What the calls on a cache in 4 bits share: where a sequence's tokens lie, argument checks, the numbers.
#pragma once
#include "sqa_chunk.h"

namespace sqa {

constexpr int kGroup = 32;                          // elements that share a power of two
constexpr int32_t kQ4MostSlots = 1 << 30;           // (slot numbers, rounded up to whole tiles, stay below 2^31)

struct Q4Args {                                     // (by value to the kernels)
  sqa_q4_cache L;
  ChunkArgs c;                                      // (c.L is not used)
};

// n tokens of a sequence at positions pos .. , in units of `slots` slots of which the first `sink` stay and the others are a ring
struct Q4Seq {
  int n, slots, sink, why;
  int64_t pos;
  __device__ __forceinline__ int64_t end() const { return pos + n; }                    // positions before it have been appended
  __device__ __forceinline__ int len() const { return (int)min(end(), (int64_t)slots); }
  __device__ __forceinline__ int slot(int64_t p) const {
    return p < slots ? (int)p : sink + (int)((uint32_t)(p - sink) % (uint32_t)(slots - sink));
  }
};
// n = 0: nothing to do; why: reported by the caller that owns the sequence
__device__ __forceinline__ Q4Seq q4_seq(const Q4Args& a, int b, bool report) {
  const ChunkSeq c = chunk_seq(a.c, b, report);
  Q4Seq s{c.n, a.L.capacity, a.L.n_sink, 0, c.pos};
  if (a.c.budget_seq) {
    s.slots = a.c.budget_seq[b];
    if (s.slots <= s.sink || s.slots > a.L.capacity) {
      if (report && s.n && a.c.status) *a.c.status = SQA_ERR_BUDGET;
      s.slots = a.L.capacity;
      s.n = 0;
    }
  }
  if (s.n > 0 && s.end() > s.slots && s.n > s.slots - s.sink) s.why = SQA_ERR_CAPACITY;
  if (s.end() > INT32_MAX) { s.why = SQA_ERR_SHAPE; }
  return s;
}

// The group's byte for the largest of its |x| as bits: e + 127 for the smallest 2^e with max |x| <= 7 * 2^e (7 = 1.75 * 2^2: the
// exponent less 2, one more where the significand is over 1.75); 255 for what is not finite.
__device__ __forceinline__ uint32_t q4_power(uint32_t top) {
  const int p = (int)((top + 0x1fffffu) >> 23) - 2;
  return top >= 0x7f800000u ? 255u : (uint32_t)min(max(p, 2), 252);
}

inline bool bad_q4(const sqa_q4_cache& c, int D, sqa_status* why) {
  *why = SQA_OK;
  if (!c.K || !c.V || !c.K_scale || !c.V_scale) *why = SQA_ERR_NULL;
  else if (!aligned16(c.K) || !aligned16(c.V) || (reinterpret_cast<uintptr_t>(c.K_scale) & 3u) || (reinterpret_cast<uintptr_t>(c.V_scale) & 3u))
    *why = SQA_ERR_SHAPE;
  else if (c.capacity < 1 || c.capacity > kQ4MostSlots) *why = SQA_ERR_CAPACITY;
  else if (c.n_sink < 0 || c.n_sink >= c.capacity) *why = SQA_ERR_BUDGET;
  else if (c.block_table && (c.n_blocks < 1 || c.blocks_per_unit < 1 || c.blocks_per_unit > SQA_MAX_BLOCKS_PER_UNIT ||
                             (int64_t)c.blocks_per_unit * SQA_BLOCK_SLOTS < c.capacity || (reinterpret_cast<uintptr_t>(c.block_table) & 3u)))
    *why = SQA_ERR_SHAPE;
  return *why != SQA_OK;
}

inline Q4Args q4_args(const sqa_q4_cache* layer, int B, int T, int Hq, int Hkv, int32_t new_pos, const sqa_batch_opts* opts) {
  Q4Args a{};
  a.L = *layer;
  a.c = chunk_args(nullptr, B, T, Hq, Hkv, new_pos, opts);
  return a;
}
inline int64_t q4_rows(const sqa_q4_cache& c, int B, int Hkv) {
  return c.block_table ? (int64_t)c.n_blocks * SQA_BLOCK_SLOTS : (int64_t)B * Hkv * c.capacity;
}
// Does memory that a call writes (n bytes at p, or NULL) lie in the cache or its table?
inline bool in_q4(const sqa_q4_cache& c, int B, int Hkv, int D, const void* p, size_t n) {
  const size_t codes = (size_t)q4_rows(c, B, Hkv) * D / 2, powers = codes / (kGroup / 2);
  return p && (overlap(p, n, c.K, codes) || overlap(p, n, c.V, codes) || overlap(p, n, c.K_scale, powers) || overlap(p, n, c.V_scale, powers) ||
               (c.block_table && overlap(p, n, c.block_table, (size_t)B * Hkv * c.blocks_per_unit * sizeof(int32_t))));
}

}  // namespace sqa
