// Block tables brought up to date from the sequences' lengths (sqa_block_assign) and the rows that new tokens go to (sqa_slot_map).
// Bound by latency: a decode step changes a few entries of each table.  Prefix sums over the sequences of what they give back and of what they lack
// say which block goes where, so that nothing depends on the order in which threads arrive.  Small tables are one workgroup's work.  For others every
// workgroup of a first launch works out the sums for itself and moves its share of the blocks, and a second launch brings lengths and count up to
// date, which the first one reads: 64 sequences of 8 heads with up to 4000 tokens, an eighth of them leaving and an eighth joining, 7 + 3.3 us in place of 18
// for one workgroup, 256 with up to 2000 8 + 3.4 in place of 90.
#include "sqa_q4.h"

namespace sqa {

constexpr int kAssignThreads = 1024;
constexpr int kOneAssign = 4096;                    // entries of all tables that one workgroup sees to
constexpr int kMostAssign = 64;                     // workgroups of a launch
constexpr int kMostEntries = INT32_MAX - kMostAssign * kAssignThreads;                   // (a thread's next entry, past the last, is a 32-bit number too)

struct AssignArgs {
  int32_t* table;
  const int32_t* tokens;
  int32_t* held;
  int32_t* free_ids;
  int32_t* free_count;
  int32_t* status;
  int B, Hkv, per, capacity, n_blocks;
};

// exclusive prefix sums of v[0 .. n) in LDS, in place; v[n] = the sum.  Each thread a run of entries, then the runs' sums.
__device__ __forceinline__ void prefix_sums(int32_t* v, int n, int32_t* s_wave) {
  const int tid = threadIdx.x, each = (n + kAssignThreads - 1) / kAssignThreads, lo = min(tid * each, n), hi = min(lo + each, n);
  int sum = 0;
  for (int i = lo; i < hi; ++i) sum += v[i];
  int up = sum;
#pragma unroll
  for (int o = 1; o < SQA_WAVE; o *= 2) {
    const int x = __shfl_up(up, o, SQA_WAVE);
    if ((tid & 63) >= o) up += x;
  }
  if ((tid & 63) == 63) s_wave[tid >> 6] = up;
  __syncthreads();
  int before = up - sum;
  for (int w = 0; w < tid >> 6; ++w) before += s_wave[w];
  for (int i = lo; i < hi; ++i) { const int x = v[i]; v[i] = before; before += x; }
  if (hi == n && lo < n) v[n] = before;
  if (n == 0 && tid == 0) v[0] = 0;
  __syncthreads();
}
// the last b with v[b] <= i: whose run of numbers i lies in
__device__ __forceinline__ int owner(const int32_t* v, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (v[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

template <bool MOVE, bool UPDATE> __global__ __launch_bounds__(kAssignThreads) void block_assign_kernel(const AssignArgs a) {
  extern __shared__ int32_t s_mem[];                // what each gives, what each lacks (B + 1 each), blocks it needs
  __shared__ int32_t s_wave[kAssignThreads / SQA_WAVE];
  int32_t* const gives = s_mem;
  int32_t* const lacks = gives + a.B + 1;
  int32_t* const needs = lacks + a.B + 1;
  const int tid = threadIdx.x;
  const int count = *a.free_count;
  for (int b = tid; b < a.B; b += kAssignThreads) {
    const int tokens = a.tokens[b], has = a.held[b];
    int need = tokens < 0 ? has : (min(tokens, a.capacity) + SQA_BLOCK_SLOTS - 1) / SQA_BLOCK_SLOTS;
    if (has < 0 || has > a.per) {
      if (UPDATE && a.status) *a.status = SQA_ERR_STATE;
      need = has;
    }
    needs[b] = need;
    gives[b] = max(has - need, 0) * a.Hkv;
    lacks[b] = max(need - has, 0) * a.Hkv;
  }
  __syncthreads();
  prefix_sums(gives, a.B, s_wave);
  prefix_sums(lacks, a.B, s_wave);
  const int given = gives[a.B];
  if (count < 0 || count > a.n_blocks - given) {
    if (UPDATE && tid == 0 && a.status) *a.status = SQA_ERR_STATE;
    return;
  }
  const int there = count + given;
  // the first sequence that the list is too short for: lacks[first_out] <= there < lacks[first_out + 1]
  const int first_out = lacks[a.B] > there ? owner(lacks, a.B + 1, there) : a.B;
  const int taken = lacks[first_out];
  if constexpr (MOVE) {
    // where the i-th block that is taken goes
    auto entry_of = [&](int i) {
      const int b = owner(lacks, a.B, i), k = i - lacks[b], each = (lacks[b + 1] - lacks[b]) / a.Hkv;
      return a.table + ((int64_t)b * a.Hkv + k / each) * a.per + needs[b] - each + k % each;
    };
    // (what changes hands is a block's number, or reported: whether it is a number that nothing else holds cannot be seen from here)
    auto look = [&](int block) { if ((unsigned)block >= (unsigned)a.n_blocks && a.status) *a.status = SQA_ERR_STATE; };
    const int at = blockIdx.x * kAssignThreads + tid, all = gridDim.x * kAssignThreads;
    for (int i = at; i < given; i += all) {         // a block that comes back, to the list's end, and from there on where it is taken at once
      const int b = owner(gives, a.B, i), k = i - gives[b], each = (gives[b + 1] - gives[b]) / a.Hkv;
      int32_t* const entry = a.table + ((int64_t)b * a.Hkv + k / each) * a.per + needs[b] + k % each;
      const int block = *entry;
      look(block);
      *entry = -1;
      a.free_ids[count + i] = block;
      if (given - 1 - i < taken) *entry_of(given - 1 - i) = block;
    }
    for (int i = given + at; i < taken; i += all) { // (what the list held before)
      const int block = a.free_ids[there - 1 - i];
      look(block);
      *entry_of(i) = block;
    }
  }
  if constexpr (UPDATE) {
    if (MOVE) __syncthreads();
    for (int b = tid; b < a.B; b += kAssignThreads)
      if (b < first_out || lacks[b + 1] == lacks[b]) a.held[b] = needs[b];
    if (tid == 0) {
      *a.free_count = there - taken;
      if (first_out < a.B && a.status) *a.status = SQA_ERR_CAPACITY;
    }
  }
}

struct MapArgs { Q4Args a; int32_t* map; };
__global__ __launch_bounds__(256) void slot_map_kernel(const MapArgs m) {
  const Q4Args& a = m.a;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t u = i / a.c.T;
  const int t = (int)(i - u * a.c.T);
  if (u >= (int64_t)a.c.B * a.c.Hkv) return;
  const int b = (int)(u / a.c.Hkv);
  const Q4Seq s = q4_seq(a, b, t == 0 && u % a.c.Hkv == 0);
  int row = -1;
  if (t < s.n && s.why) {
    if (t == 0 && a.c.status) *a.c.status = s.why;
  } else if (t < s.n) {
    const int slot = s.slot(s.pos + t);
    int64_t r = u * a.L.capacity + slot;
    if (a.L.block_table) {
      const int block = a.L.block_table[u * a.L.blocks_per_unit + slot / SQA_BLOCK_SLOTS];
      r = block < 0 ? -1 : (int64_t)block * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS;
    }
    if (r > INT32_MAX) {
      r = -1;
      if (a.c.status) *a.c.status = SQA_ERR_SHAPE;
    }
    row = (int)r;
  }
  m.map[i] = row;
}

}  // namespace sqa

extern "C" sqa_status sqa_block_assign(int32_t* block_table, int B, int Hkv, int32_t blocks_per_unit, int32_t capacity, const int32_t* tokens,
                                       int32_t* held, int32_t* free_ids, int32_t* free_count, int32_t n_blocks, int32_t* status, void* stream) {
  if (!block_table || !tokens || !held || !free_ids || !free_count) return SQA_ERR_NULL;
  for (const void* p : {(const void*)block_table, (const void*)tokens, (const void*)held, (const void*)free_ids, (const void*)free_count, (const void*)status})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return SQA_ERR_SHAPE;
  if (B < 1 || B > SQA_MAX_ASSIGN || Hkv < 1 || blocks_per_unit < 1 || n_blocks < 1 || (int64_t)B * Hkv > sqa::kMostEntries / blocks_per_unit) return SQA_ERR_SHAPE;
  if (capacity < 1 || capacity > sqa::kQ4MostSlots || (int64_t)blocks_per_unit * SQA_BLOCK_SLOTS < capacity) return SQA_ERR_CAPACITY;
  sqa::AssignArgs a{block_table, tokens, held, free_ids, free_count, status, B, Hkv, blocks_per_unit, capacity, n_blocks};
  const size_t lds = (size_t)(3 * B + 2) * sizeof(int32_t);
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto launch = [&](void (*fn)(sqa::AssignArgs), int blocks) {
    if (sqa::allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds) != hipSuccess) return false;
    fn<<<blocks, sqa::kAssignThreads, lds, st>>>(a);
    return hipGetLastError() == hipSuccess;
  };
  const int64_t entries = (int64_t)B * Hkv * blocks_per_unit;
  const bool ok = entries <= sqa::kOneAssign ? launch(sqa::block_assign_kernel<true, true>, 1)
                                             : launch(sqa::block_assign_kernel<true, false>, (int)(entries / sqa::kOneAssign < sqa::kMostAssign ? entries / sqa::kOneAssign + 1 : sqa::kMostAssign)) &&
                                                   launch(sqa::block_assign_kernel<false, true>, 1);
  if (!ok) { (void)hipGetLastError(); return SQA_ERR_HIP; }
  return SQA_OK;
}

extern "C" sqa_status sqa_slot_map(const int32_t* block_table, int B, int T, int Hkv, int32_t blocks_per_unit, int32_t capacity, int32_t n_sink,
                                   int32_t new_pos, int32_t* map, void* stream, const sqa_batch_opts* opts) {
  if (!map) return SQA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(map) & 3u) || (reinterpret_cast<uintptr_t>(block_table) & 3u) || sqa::bad_chunk_shape(B, T, Hkv, Hkv, 64, new_pos, opts))
    return SQA_ERR_SHAPE;
  if (capacity < 1 || capacity > sqa::kQ4MostSlots || (block_table && (int64_t)blocks_per_unit * SQA_BLOCK_SLOTS < capacity)) return SQA_ERR_CAPACITY;
  if (n_sink < 0 || n_sink >= capacity) return SQA_ERR_BUDGET;
  sqa_q4_cache c{};
  c.block_table = block_table; c.blocks_per_unit = blocks_per_unit; c.capacity = capacity; c.n_sink = n_sink;
  const int64_t blocks = ((int64_t)B * Hkv * T + 255) / 256;
  sqa::MapArgs m{sqa::q4_args(&c, B, T, Hkv, Hkv, new_pos, opts), map};
  sqa::slot_map_kernel<<<(unsigned)blocks, 256, 0, static_cast<hipStream_t>(stream)>>>(m);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}
