// What a chunk of tokens gives to the accumulated attention of every slot of a layer cache (sqa_chunk_scores):
//   score[j] += sum over the unit's query heads and the tokens t with position >= j of exp(s_tj - lse_t),  s = q.K_j / sqrt(D)
// The normalisers are known, so this is one product and a sum down its columns.  A wave keeps 32 slots' keys in registers and
// walks the rows (head by head, only the tokens that see its workgroup's 128 slots), 64 at a time in LDS with two buffers:
//   S = Q.K^T    a lane holds 16 of 32 rows of one slot and adds them up by itself; the two lane halves meet at the end
// One workgroup owns a slot, so nothing is added atomically; where there are few slots the rows are shared out over workgroups
// whose sums go through the workspace, and the last one to arrive adds them in order.
#include "sqa_chunk_mma.h"

namespace sqa {

constexpr int kScoreThreads = 256;
constexpr int kScoreSlots = 128;                    // of a workgroup
constexpr int kScoreRows = 64;                      // of a tile in LDS
constexpr int kScoreItems = 1024;                   // workgroups that few slots are shared out to

struct ScoresArgs {
  ChunkArgs c;
  const void* q;
  const float* lse;
  int32_t* count;                                   // [items]
  float2* part;                                     // [items][splits][kScoreSlots / 2]
  float scale;                                      // log2(e) / sqrt(D)
  int tiles, splits;
};

template <typename T, int D>
__global__ __launch_bounds__(kScoreThreads, 2) void chunk_scores_kernel(const ScoresArgs a) {
  using R = TileRows<T, D>;
  constexpr int TILE = kScoreRows * R::RB;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // two tiles of rows
  __shared__ float s_lse[2][kScoreRows];            // in powers of two; of rows that are none: infinity
  __shared__ int s_see[2][kScoreRows];              // the last slot that a row sees
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
  if (!chunk_held(a.c.L, unit, u, seq.pos + seq.n)) {
    if (tid == 0 && tile == 0 && split == 0 && a.c.status) *a.c.status = SQA_ERR_STATE;
    return;
  }
  const int end = (int)(seq.pos + seq.n);
  if (unit.table) {                                  // a unit is left untouched as a whole: all of its blocks are looked at
    int outside = 0;
    for (int i = tid; i < (end + SQA_BLOCK_SLOTS - 1) / SQA_BLOCK_SLOTS; i += kScoreThreads) outside |= (unsigned)unit.table[i] >= (unsigned)a.c.L.n_blocks;
    if (__syncthreads_or(outside)) {
      if (tid == 0 && tile == 0 && split == 0 && a.c.status) *a.c.status = SQA_ERR_SHAPE;
      return;
    }
  }
  if (slot0 >= end) return;
  // the tokens that see any of the slots, and this workgroup's tiles of their rows
  const int t0 = (int)max((int64_t)0, slot0 - seq.pos), tv = seq.n - t0, rows = g * tv;
  const int nt = (rows + kScoreRows - 1) / kScoreRows, per = (nt + a.splits - 1) / a.splits;
  const int parts = (nt + per - 1) / per;
  if (split >= parts) return;
  const int tile0 = split * per, tile1 = min(tile0 + per, nt);

  // ---- the lane's slot
  const int slot = (int)slot0 + 32 * wave + col;
  Frag<T, D> k;
  {
    const int s = min(slot, end - 1);
    const int64_t at = unit.table ? (int64_t)unit.table[s / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + s % SQA_BLOCK_SLOTS : unit.first + s;
    const char* src = static_cast<const char*>(a.c.L.K) + at * R::RB;
#pragma unroll
    for (int x = 0; x < k.NS; ++x) k.p[x] = ld16(src + (2 * x + half) * 16);
    arrived(k);
  }
  const int64_t head0 = (int64_t)b * a.c.Hq + h * g;
  const char* const Q = static_cast<const char*>(a.q) + head0 * a.c.T * R::RB;
  auto fetch = [&](int tl, int buf) {
    const uint32_t dst = lds_at(s_stage) + (uint32_t)(buf * TILE);
#pragma unroll
    for (int i = 0; i < kScoreRows / 4 / R::RPI; ++i) {
      const int rr = wave * (kScoreRows / 4) + i * R::RPI, row = rr + lane / R::PPR;
      const int x = min(tl * kScoreRows + row, rows - 1);
      fetch16(Q + ((int64_t)(x / tv) * a.c.T + t0 + x % tv) * R::RB + (((lane % R::PPR) ^ R::k_swizzle(row)) << 4), dst + rr * R::RB);
    }
    if (tid < kScoreRows) {
      const int x = tl * kScoreRows + tid, y = min(x, rows - 1);
      const float v = a.lse[(head0 + y / tv) * a.c.T + t0 + y % tv];
      s_lse[buf][tid] = x < rows ? v * 1.4426950408889634f : INFINITY;
      s_see[buf][tid] = (int)seq.pos + t0 + y % tv;
    }
  };
  float sum = 0.f;
  fetch(tile0, 0);
  for (int tl = tile0; tl < tile1; ++tl) {
    const int buf = (tl - tile0) & 1;
    fetched();
    __syncthreads();
    if (tl + 1 < tile1) fetch(tl + 1, buf ^ 1);
    const char* const Qt = s_stage + buf * TILE;
#pragma unroll
    for (int rb = 0; rb < kScoreRows / 32; ++rb) {
      f32x16_t s{};
      const int row = 32 * rb + col;
#pragma unroll
      for (int x = 0; x < k.NS; ++x) {
        const uint4 q = *reinterpret_cast<const uint4*>(Qt + row * R::RB + (((2 * x + half) ^ R::k_swizzle(row)) << 4));
        mma_piece<T>(q, k.p[x], s);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = 32 * rb + c_row(i, half);
        const float p = exp2_fast(fmaf(s[i], a.scale, -s_lse[buf][at]));
        sum += s_see[buf][at] >= slot ? p : 0.f;
      }
    }
  }
  sum = other_half_sum(sum);

  if (parts > 1) {
    if (half == 0) s_sum[32 * wave + col] = sum;
    __syncthreads();
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
    sum = s_sum[32 * wave + col];
  }
  if (half == 0 && slot < end) a.c.L.score_acc[unit.first + slot] += sum;
  if (tid == 0 && tile == 0) a.c.L.unit_state[(int64_t)u * SQA_ST_WORDS + SQA_ST_EVICT_HINT] = -2;   // what was decided by the old scores
}

static int scores_splits(int B, int T, int Hq, int Hkv, int tiles) {
  const int64_t items = (int64_t)B * Hkv * tiles, row_tiles = ((int64_t)T * (Hq / Hkv) + kScoreRows - 1) / kScoreRows;
  int64_t s = kScoreItems / items;
  s = s > row_tiles ? row_tiles : s;
  return s < 1 ? 1 : (int)s;
}
// (any length: items x splits <= kScoreItems where there are splits)
size_t chunk_scores_scratch() { return (size_t)kScoreItems * kScoreSlots * sizeof(float); }

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
  const int64_t slots = uniform ? (int64_t)new_pos + T : layer->capacity;
  const int64_t tiles = (slots + sqa::kScoreSlots - 1) / sqa::kScoreSlots;
  if ((int64_t)B * Hkv > (INT32_MAX - 8) / tiles) return SQA_ERR_SHAPE;
  a.tiles = (int)tiles;
  a.splits = sqa::scores_splits(B, T, Hq, Hkv, a.tiles);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? sqa::launch_scores<float, 64>(a, st) : sqa::launch_scores<float, 128>(a, st);
  return D == 64 ? sqa::launch_scores<sqa::bf16_t, 64>(a, st) : sqa::launch_scores<sqa::bf16_t, 128>(a, st);
}
