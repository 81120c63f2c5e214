// What the calls on chunks of tokens (sqa_chunk_rows.hip, sqa_chunk_attention.hip, sqa_chunk_scores.hip) share: a chunk's
// place in a layer cache, argument checks, matrix products of 32 x 32 blocks.
#pragma once
#include "sqa_common.h"

namespace sqa {

__device__ __forceinline__ uint32_t pair(float lo, float hi) {                           // two bf16, round to nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

struct ChunkSeq { int n; int64_t pos; };            // tokens of a sequence in this call, position of the first

struct ChunkArgs {                                  // (by value to the kernels)
  sqa_layer_cache L;
  const int32_t* prompt_len;
  const int32_t* new_pos_seq;
  const int32_t* budget_seq;
  int32_t* status;
  int32_t new_pos;
  int B, T, Hq, Hkv, g;
};

// n = 0: the sequence takes no part (or brings a length outside 0..T: reported)
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& a, int b, bool report) {
  ChunkSeq s{a.T, a.new_pos};
  if (a.new_pos_seq) s.pos = a.new_pos_seq[b];
  if (a.prompt_len) s.n = a.prompt_len[b];
  if (s.n < 0 || s.n > a.T) {
    if (report && a.status) *a.status = SQA_ERR_SHAPE;
    s.n = 0;
  }
  if (s.pos < 0) s.n = 0;
  return s;
}

// where a unit's slots lie
struct ChunkUnit { int64_t first; int slots; const int32_t* table; };
__device__ __forceinline__ ChunkUnit chunk_unit(const sqa_layer_cache& L, int u) {
  ChunkUnit x{(int64_t)u * L.capacity, L.capacity, nullptr};
  if (L.unit_offset) {
    x.first = L.unit_offset[u];
    x.slots = (int)(L.unit_offset[u + 1] - x.first);
  } else if (L.block_table) {
    x.table = L.block_table + (int64_t)u * L.blocks_per_unit;
    x.slots = (int)min((int64_t)x.slots, (int64_t)L.blocks_per_unit * SQA_BLOCK_SLOTS);
  }
  return x;
}

// Does the unit hold the tokens of positions 0 .. end-1 in slots 0 .. end-1?  Exact while nothing was evicted; after that slot
// end-1 or the ring tells, unless heavy hitters have changed places.
__device__ __forceinline__ bool chunk_held(const sqa_layer_cache& L, const ChunkUnit& x, int u, int64_t end) {
  const int4 st = *reinterpret_cast<const int4*>(L.unit_state + (int64_t)u * SQA_ST_WORDS);        // (both asked for together)
  const int last = L.pos[x.first + max(min(end, (int64_t)x.slots), (int64_t)1) - 1];
  return end <= x.slots && st.x >= end && st.y == 0 && (end == 0 || last == end - 1);
}

// x / d for 32-bit x by one high product: off by one at most, put right
struct Divisor {
  uint32_t d, m;
  __device__ __forceinline__ explicit Divisor(uint32_t v) : d(v), m(0xffffffffu / v + (v > 1)) {}
  __device__ __forceinline__ void operator()(uint32_t x, uint32_t& q, uint32_t& r) const {
    q = d > 1 ? __umulhi(x, m) : x;
    r = x - q * d;
    if ((int32_t)r < 0) { --q; r += d; }
  }
};

inline bool bad_layer(const sqa_layer_cache& c, sqa_status* why) {
  *why = SQA_OK;
  if (!c.K || !c.V || !c.pos || !c.unit_state) *why = SQA_ERR_NULL;
  else if (!aligned16(c.K) || !aligned16(c.V) || !aligned16(c.unit_state)) *why = SQA_ERR_SHAPE;
  else if (c.budget < 1) *why = SQA_ERR_BUDGET;
  else if (c.capacity < 1) *why = SQA_ERR_CAPACITY;
  else if (c.block_table && (c.unit_offset || c.n_blocks < 1 || c.blocks_per_unit < 1 || c.blocks_per_unit > SQA_MAX_BLOCKS_PER_UNIT ||
                             (int64_t)c.blocks_per_unit * SQA_BLOCK_SLOTS < (c.budget < c.capacity ? c.budget : c.capacity)))
    *why = SQA_ERR_SHAPE;
  return *why != SQA_OK;
}

inline bool bad_chunk_shape(int B, int T, int Hq, int Hkv, int D, int32_t new_pos, const sqa_batch_opts* opts) {
  return B < 1 || T < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || (D != 64 && D != 128) || (int64_t)B * Hq > INT32_MAX / T ||
         (!(opts && opts->new_pos_seq) && (new_pos < 0 || (int64_t)new_pos + T > INT32_MAX));
}

inline ChunkArgs chunk_args(const sqa_layer_cache* layer, int B, int T, int Hq, int Hkv, int32_t new_pos, const sqa_batch_opts* opts) {
  ChunkArgs a{};
  if (layer) a.L = *layer;
  if (opts) { a.prompt_len = opts->prompt_len; a.new_pos_seq = opts->new_pos_seq; a.budget_seq = opts->budget_seq; a.status = opts->status; }
  a.new_pos = new_pos; a.B = B; a.T = T; a.Hq = Hq; a.Hkv = Hkv; a.g = Hq / Hkv;
  return a;
}

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// Data that one workgroup hands to another inside a launch: stored through to and loaded from where every XCD sees it (no
// cache is flushed), 16 bytes at a time by buffer instructions with the agent-scope bits set, or 8 by atomics.
struct HandOver {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ HandOver(float4* base /*the same in all lanes*/, uint32_t bytes)
      : r(__builtin_amdgcn_make_buffer_rsrc(base, 0, (int)bytes, 0x00027000)) {}
  static constexpr int kAgent = 16;                  // sc1
  __device__ __forceinline__ void put(uint32_t i, float4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u_t, v), r, (int)(i * 16), 0, kAgent);
  }
  __device__ __forceinline__ float4 get(uint32_t i) const {
    return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(i * 16), 0, kAgent));
  }
};
__device__ __forceinline__ void hand_over(float2* p, float2 v) {
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 handed_over(const float2* p) {
  return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// Every thread's stores have arrived, then one count: true in the whole workgroup if it is the last of `of`.
__device__ __forceinline__ bool last_to_arrive(int32_t* count, int of, int* s_word) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) *s_word = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*s_word != of - 1) return false;
  if (threadIdx.x == 0) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next launch
  return true;
}

constexpr int kChunkCounters = 1024;                // at the head of a workspace, whatever the call's shape
constexpr size_t kChunkCounterBytes = kChunkCounters * sizeof(int32_t);

size_t chunk_attention_scratch(int T, int Hq, int Hkv, int D);                          // bytes behind the counters
size_t chunk_scores_scratch();
struct ScoresPlan { int slots, tiles, splits; };     // slots of a workgroup, of which a unit has `tiles`, and the workgroups of each that share out the rows
ScoresPlan scores_plan(sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos, int32_t capacity, bool uniform);

}  // namespace sqa
