// What a chunk of tokens gives to the accumulated attention of every slot of a layer cache (sqa_chunk_scores):
//   score[j] += sum over the unit's query heads and the tokens t with position >= j of exp(s_tj - lse_t),  s = q.K_j / sqrt(D)
// The normalisers are known, so this is one product and a sum down its columns.  A wave keeps the keys of one or two
// blocks of 32 slots in registers and walks the rows (head by head, only the tokens that see its workgroup's slots), 64 at a time in LDS
// with two buffers:
//   S^T = K.Q^T  a lane holds 16 of 32 slots of one row and adds up each by itself, over its rows: one normaliser per lane and
//                block, and no sum across lanes before the end.  The exponentials of one block of rows are independent of the next
//                one's products and are taken meanwhile
// Bound by how far a logit's vector instructions (multiply-add, exp2, add) and its product overlap: 32 heads over 8, 2048 tokens after 30000
// 1050 TFLOP/s; 64 over 8, 512 after 7680 80 us, 830, busy 0.47 and 0.36 (what a workgroup does before its first product weighs).
// One workgroup owns a slot, so nothing is added atomically; where there are few slots the rows are shared out over workgroups
// whose sums go through the workspace, and the last one to arrive adds them in order.
#include "sqa_chunk_mma.h"
#include <type_traits>

namespace sqa {

constexpr int kScoreThreads = 256;
constexpr int kScoreRows = 64;                      // of a tile in LDS
// slots of a wave in blocks of 32: two in bf16 with D = 128 (each row read from LDS feeds both), else one: in fp32 the products bound it
// either way; with D = 64 in bf16 a wave then needs 114 registers, four workgroups fit a CU, and 8 x 2048 tokens of 16 heads take 83 in place of 105 us
// (512 of 64 heads over 8 after 7680 68 in place of 65; with D = 128 201 against 219 and 89 against 85, 4096 tokens of 32 heads over 8 117
// against 95).  Whether the compiler is told of two, three or four workgroups changes neither registers nor time (83 to 84 us)
template <typename T, int D> constexpr int score_blocks() { return sizeof(T) == 2 && D == 128 ? 2 : 1; }
template <typename T, int D> constexpr int score_slots() { return 4 * 32 * score_blocks<T, D>(); }
constexpr int kScoreSlotsMost = 256;
constexpr int kScoreItems = 512;                    // workgroups that few slots are shared out to: two per CU

struct ScoresArgs {
  ChunkArgs c;
  const void* q;
  const float* lse;
  int32_t* count;                                   // [items]
  float2* part;                                     // [items][splits][slots of a workgroup / 2]
  float scale;                                      // log2(e) / sqrt(D)
  int tiles, splits;
};

template <typename T, int D>
__global__ __launch_bounds__(kScoreThreads, sizeof(T) == 2 && D == 64 ? 3 : 2) void chunk_scores_kernel(const ScoresArgs a) {
  using R = TileRows<T, D>;
  constexpr int TILE = kScoreRows * R::RB, KB = score_blocks<T, D>(), kScoreSlots = score_slots<T, D>(), NS = Frag<T, D>::NS;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // two tiles of rows
  __shared__ __attribute__((aligned(16))) float s_lse[4][kScoreRows];            // in powers of two; of rows that are none: infinity
  __shared__ __attribute__((aligned(16))) int s_see[4][kScoreRows];              // the last slot that a row sees
  __shared__ float s_sum[kScoreSlots];
  __shared__ int s_word;

  const int64_t items = (int64_t)a.c.B * a.c.Hkv * a.tiles;
  const int64_t work = xcd_item(items * a.splits);
  if (work < 0) return;
  const int split = (int)(work % a.splits);
  const int64_t item = work / a.splits;
  const int u = (int)(item / a.tiles), tile = (int)(item % a.tiles);
  const int b = u / a.c.Hkv, h = u % a.c.Hkv, g = a.c.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const ChunkSeq seq = chunk_seq(a.c, b, tid == 0 && h == 0 && tile == 0 && split == 0);
  if (seq.n == 0) return;
  const ChunkUnit unit = chunk_unit(a.c.L, u);
  const int64_t slot0 = (int64_t)tile * kScoreSlots;
  const int64_t held = seq.pos + seq.n;
  if (held > unit.slots) {
    if (tid == 0 && tile == 0 && split == 0 && a.c.status) *a.c.status = SQA_ERR_STATE;
    return;
  }
  const int end = __builtin_amdgcn_readfirstlane((int)held);
  if (slot0 >= end) return;
  // ---- the lane's slots.  (Asked for before it is known whether the unit holds the chunk: a block number outside the pools reads block 0.)
  const int slot = (int)slot0 + 32 * KB * wave + col;                    // ... whose keys it holds, and the first whose sums it holds
  const int slot_of = (int)slot0 + 32 * KB * wave + 4 * half;
  Frag<T, D> k[KB];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int s = min(slot + 32 * kb, end - 1);
    int64_t at = unit.first + s;
    if (unit.table) {
      const unsigned blk = (unsigned)unit.table[s / SQA_BLOCK_SLOTS];
      at = (int64_t)(blk < (unsigned)a.c.L.n_blocks ? blk : 0u) * SQA_BLOCK_SLOTS + s % SQA_BLOCK_SLOTS;
    }
    const char* src = static_cast<const char*>(a.c.L.K) + at * R::RB;
#pragma unroll
    for (int x = 0; x < k[kb].NS; ++x) k[kb].p[x] = ld16(src + (2 * x + half) * 16);
  }
  // the tokens that see any of the slots, and this workgroup's tiles of their rows
  const int t0 = __builtin_amdgcn_readfirstlane((int)max((int64_t)0, slot0 - seq.pos)), tv = __builtin_amdgcn_readfirstlane(seq.n) - t0, rows = g * tv;
  const int nt = (rows + kScoreRows - 1) / kScoreRows, per = (nt + a.splits - 1) / a.splits;
  const int parts = (nt + per - 1) / per;
  if (split >= parts) return;
  const int tile0 = split * per, tile1 = min(tile0 + per, nt);

  const int64_t head0 = (int64_t)b * a.c.Hq + h * g;
  const char* const Q = static_cast<const char*>(a.q) + head0 * a.c.T * R::RB;
  const Divisor by_tv((uint32_t)tv);
  constexpr int NI = kScoreRows / 4 / R::RPI;        // copies of a wave per tile
  uint32_t place[NI];                                // the lane's row and piece in each of them
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int rr = wave * (kScoreRows / 4) + i * R::RPI, row = rr + lane / R::PPR;
    place[i] = (uint32_t)(row * R::RB + (((lane % R::PPR) ^ R::k_swizzle(row)) << 4));
  }
  // where a tile's first row is: head of the unit, token (scalar arithmetic from tile to tile)
  struct Place { int gi, tt; };
  auto next = [&](Place p) {
    p.tt += kScoreRows;
    if (p.tt >= tv) {
      uint32_t more, tt;
      by_tv((uint32_t)p.tt, more, tt);
      p.gi += __builtin_amdgcn_readfirstlane((int)more);
      p.tt = __builtin_amdgcn_readfirstlane((int)tt);
    }
    return p;
  };
  auto fetch = [&](int tl, int buf, Place p) {
    const uint32_t dst = lds_at(s_stage) + (uint32_t)(buf * TILE + wave * (kScoreRows / 4) * R::RB);
    if (p.tt + kScoreRows <= tv) {                   // rows of one head, one after the other
      const char* const base = uniform(Q + ((int64_t)p.gi * a.c.T + t0 + p.tt) * R::RB);
#pragma unroll
      for (int i = 0; i < NI; ++i) fetch16(base, place[i], dst + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = wave * (kScoreRows / 4) + i * R::RPI + lane / R::PPR;
        uint32_t gi, tt;
        by_tv((uint32_t)min(tl * kScoreRows + row, rows - 1), gi, tt);
        fetch16(Q + ((int64_t)gi * a.c.T + t0 + tt - row) * R::RB + place[i], dst + i * 1024);
      }
    }
  };
  // a tile's normalisers wait in registers of the first wave for a round, so that nothing waits for them
  float lse_next = 0.f;
  int see_next = 0;
  auto ask = [&](int tl, Place p) {
    if (wave == 0 && tl < tile1) {
      uint32_t gi = (uint32_t)p.gi, tt = (uint32_t)(p.tt + tid);
      if (p.tt + kScoreRows > tv) by_tv((uint32_t)min(tl * kScoreRows + tid, rows - 1), gi, tt);
      lse_next = a.lse[(head0 + gi) * a.c.T + t0 + tt];
      see_next = (int)seq.pos + t0 + (int)tt;
    }
  };
  auto keep = [&](int tl) {
    if (wave == 0) {
      s_lse[tl & 3][tid] = tl * kScoreRows + tid < rows ? lse_next * 1.4426950408889634f : INFINITY;
      s_see[tl & 3][tid] = see_next;
    }
  };
  // rows of a tile that are of one head and all see the workgroup's last slot need no look at what each one sees
  const int last_slot = (int)slot0 + kScoreSlots - 1;
  float sum[KB][16] = {};                            // of a lane's rows
  f32x16_t s[2][KB];                                 // a block's products, and the one before it
  int q_at[NS];                                      // the lane's row and pieces in a block of 32 rows
#pragma unroll
  for (int x = 0; x < NS; ++x) q_at[x] = col * R::RB + (((2 * x + half) ^ R::k_swizzle(col)) << 4);
  // Logits of slots that a row does not see, of the rows 32 rb .. of tile tl.  (Their exponential is 0 unless the row's normaliser is NaN
  // or -inf: that goes into the logits that the row sees.)
  auto hide = [&](f32x16_t (&e)[KB], int tl, int rb, float& ref) {
    const int sees = s_see[tl & 3][32 * rb + col] - slot_of;
    if (__any(!(ref > -INFINITY))) {
      const float odd = ref > -INFINITY ? 0.f : ref;
      ref = ref > -INFINITY ? ref : 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) e[kb] -= odd;
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) e[kb][i] = sees >= 32 * kb + c_row(i, 0) ? e[kb][i] : -INFINITY;
  };
  // 16 / NS of a block's logits of each block of slots, x of NS
  auto add = [&](const f32x16_t (&e)[KB], int x, float ref) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 16 * x / NS; i < 16 * (x + 1) / NS; ++i) sum[kb][i] += exp2_fast(fmaf(e[kb][i], a.scale, -ref));
  };
  // The two blocks of rows of a tile, the exponentials of the block before each between its products (a product of bf16 takes the matrix
  // core as long as five multiply-adds or two exponentials take), its rows read from LDS some steps ahead.  The steps are kept apart: left
  // to itself the compiler gathers the products.
  auto rows_of = [&](const char* Qt, int tl, bool look_before, bool look) {
    constexpr int AHEAD = 3;
    uint4 q[2 * NS];
    auto read = [&](int y) { q[y] = *reinterpret_cast<const uint4*>(Qt + q_at[y % NS] + (y / NS) * 32 * R::RB); };
#pragma unroll
    for (int y = 0; y < AHEAD; ++y) read(y);
    float ref[2] = {s_lse[(tl - 1) & 3][32 + col], s_lse[tl & 3][col]};
    if (look_before) hide(s[1], tl - 1, 1, ref[0]);
#pragma unroll
    for (int y = 0; y < 2 * NS; ++y) {
      const int rb = y / NS, x = y % NS;
      if (y == NS) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(sum[kb][i]));      // (the branch is no reason to add them up later)
        if (look) hide(s[0], tl, 0, ref[1]);
      }
      if (y + AHEAD < 2 * NS) read(y + AHEAD);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if (x == 0) s[rb][kb] = f32x16_t{};
        mma_piece<T>(k[kb].p[x], q[y], s[rb][kb]);
      }
      add(s[1 - rb], x, ref[rb]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  bool look_before = false;                          // (s[1] holds the last block of the tile before, whose exponentials are still to come)
  Place now, soon, later;                            // of this tile, the next one and the one after
  {
    uint32_t gi, tt;
    by_tv((uint32_t)(tile0 * kScoreRows), gi, tt);
    now = {__builtin_amdgcn_readfirstlane((int)gi), __builtin_amdgcn_readfirstlane((int)tt)};
  }
  soon = later = next(now);
  ask(tile0, now);
  fetch(tile0, 0, now);
  int why = chunk_held(a.c.L, unit, u, held) ? 0 : SQA_ERR_STATE;
  if (!why && unit.table) {                          // a unit is left untouched as a whole: all of its blocks are looked at
    int outside = 0;
    for (int i = tid; i < (end + SQA_BLOCK_SLOTS - 1) / SQA_BLOCK_SLOTS; i += kScoreThreads) outside |= (unsigned)unit.table[i] >= (unsigned)a.c.L.n_blocks;
    if (__syncthreads_or(outside)) why = SQA_ERR_SHAPE;
  }
  if (why) {
    if (tid == 0 && tile == 0 && split == 0 && a.c.status) *a.c.status = why;
    fetched();                                       // (copies in flight would arrive in another workgroup's LDS)
    return;
  }
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) arrived(k[kb]);
  keep(tile0);
  if (wave == 0) s_lse[(tile0 - 1) & 3][tid] = INFINITY;              // what comes before the first block adds nothing
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) s[1][kb] = f32x16_t{};
  ask(tile0 + 1, soon);
  for (int tl = tile0; tl < tile1; ++tl) {
    const int buf = (tl - tile0) & 1;
    fetched();
    __syncthreads();
    if (tl + 1 < tile1) {
      keep(tl + 1);
      fetch(tl + 1, buf ^ 1, soon);
      later = next(soon);
      ask(tl + 2, later);
    }
    const char* const Qt = s_stage + buf * TILE;
    const bool look = now.tt + kScoreRows > tv || (int)seq.pos + t0 + now.tt < last_slot;
    now = soon;
    soon = later;
    rows_of(Qt, tl, look_before, look);
    look_before = look;
  }
  float ref = s_lse[(tile1 - 1) & 3][32 + col];
  if (look_before) hide(s[1], tile1 - 1, 1, ref);
#pragma unroll
  for (int x = 0; x < NS; ++x) add(s[1], x, ref);
  // the 32 rows of a slot's lanes: each exchange halves what a lane holds, the last leaves it one slot
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = sum[kb][i];
    auto exchange = [&](auto n_) {
      constexpr int n = decltype(n_)::value;
      const bool upper = (lane & (2 * n)) != 0;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float give = upper ? v[i] : v[i + n], mine = upper ? v[i + n] : v[i];
        v[i] = mine + __shfl_xor(give, 2 * n);
      }
    };
    exchange(std::integral_constant<int, 8>{});
    exchange(std::integral_constant<int, 4>{});
    exchange(std::integral_constant<int, 2>{});
    exchange(std::integral_constant<int, 1>{});
    const float all = v[0] + __shfl_xor(v[0], 1);
    if ((lane & 1) == 0) s_sum[32 * (KB * wave + kb) + c_row((lane & 31) >> 1, half)] = all;
  }
  __syncthreads();

  if (parts > 1) {
    float2* const rec = a.part + item * a.splits * (kScoreSlots / 2);
    if (tid < kScoreSlots / 2) hand_over(rec + (int64_t)split * (kScoreSlots / 2) + tid, make_float2(s_sum[2 * tid], s_sum[2 * tid + 1]));
    if (!last_to_arrive(a.count + item, parts, &s_word)) return;
    if (tid < kScoreSlots / 2) {
      float2 v = make_float2(0.f, 0.f);
      for (int p = 0; p < parts; ++p) {
        const float2 x = handed_over(rec + (int64_t)p * (kScoreSlots / 2) + tid);
        v.x += x.x; v.y += x.y;
      }
      s_sum[2 * tid] = v.x; s_sum[2 * tid + 1] = v.y;
    }
    __syncthreads();
  }
  if (tid < kScoreSlots && slot0 + tid < end) a.c.L.score_acc[unit.first + slot0 + tid] += s_sum[tid];
  if (tid == 0 && tile == 0) a.c.L.unit_state[(int64_t)u * SQA_ST_WORDS + SQA_ST_EVICT_HINT] = -2;   // what was decided by the old scores
}

ScoresPlan scores_plan(sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos, int32_t capacity, bool uniform) {
  ScoresPlan p;
  p.slots = dt == SQA_F32 || D == 64 ? score_slots<float, 64>() : score_slots<bf16_t, 128>();
  p.tiles = (int)(((uniform ? (int64_t)new_pos + T : capacity) + p.slots - 1) / p.slots);
  const int64_t items = (int64_t)B * Hkv * p.tiles, row_tiles = ((int64_t)T * (Hq / Hkv) + kScoreRows - 1) / kScoreRows;
  int64_t s = kScoreItems / items;
  s = s > row_tiles ? row_tiles : s;
  p.splits = s < 1 ? 1 : (int)s;
  return p;
}
// (any length: items x splits <= kScoreItems where there are splits)
size_t chunk_scores_scratch() { return (size_t)kScoreItems * kScoreSlotsMost * sizeof(float); }

template <typename T, int D>
static sqa_status launch_scores(const ScoresArgs& a, hipStream_t st) {
  const auto fn = chunk_scores_kernel<T, D>;
  const size_t lds = 2 * kScoreRows * TileRows<T, D>::RB;
  if (lds > 48 * 1024) SQA_HIP_CHECK(allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds));
  fn<<<(unsigned)xcd_grid((int64_t)a.c.B * a.c.Hkv * a.tiles * a.splits), kScoreThreads, lds, st>>>(a);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}

}  // namespace sqa

extern "C" sqa_status sqa_chunk_scores(const void* q, const float* lse, sqa_dtype dt, int B, int T, int Hq, int Hkv, int D,
                                       int32_t new_pos, const sqa_layer_cache* layer, void* workspace, size_t ws_bytes, void* stream,
                                       const sqa_batch_opts* opts) {
  if (!q || !lse || !layer || !workspace) return SQA_ERR_NULL;
  sqa_status why;
  if (sqa::bad_layer(*layer, &why)) return why;
  if (!layer->score_acc) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (sqa::bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  if (!sqa::aligned16(q) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return SQA_ERR_SHAPE;
  if (ws_bytes < sqa_chunk_workspace_bytes(layer, B, T, Hq, Hkv, D)) return SQA_ERR_CAPACITY;
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  if (uniform && (int64_t)new_pos + T > layer->capacity) return SQA_ERR_CAPACITY;
  sqa::ScoresArgs a{};
  a.c = sqa::chunk_args(layer, B, T, Hq, Hkv, new_pos, opts);
  a.q = q; a.lse = lse;
  a.count = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float2*>(static_cast<char*>(workspace) + sqa::kChunkCounterBytes);
  a.scale = (float)(1.4426950408889634 / sqrt((double)D));
  const sqa::ScoresPlan p = sqa::scores_plan(dt, B, T, Hq, Hkv, D, new_pos, layer->capacity, uniform);
  if ((int64_t)B * Hkv > (INT32_MAX - 8) / p.tiles) return SQA_ERR_SHAPE;
  a.tiles = p.tiles;
  a.splits = p.splits;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? sqa::launch_scores<float, 64>(a, st) : sqa::launch_scores<float, 128>(a, st);
  return D == 64 ? sqa::launch_scores<sqa::bf16_t, 64>(a, st) : sqa::launch_scores<sqa::bf16_t, 128>(a, st);
}
