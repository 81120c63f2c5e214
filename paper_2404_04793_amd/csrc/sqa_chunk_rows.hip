// Heads of queries and keys normalised and rotated, laid out head by head (sqa_qk_norm_rope) or, for a chunk's
// keys and values, written into the slots of a layer cache (sqa_chunk_append).
//   y = x / sqrt(mean(x^2) + eps) * w ;  (a, b) <- (a cos - b sin, b cos + a sin) over the leading rot_dim elements
// Bound by memory: every element is read once and written once, the angles come from a table of rot_dim floats per position.
// (4 x 2048 tokens of 32 + 8 heads of 128, bf16: 34.4 us, 4.9 TB/s, a large copy's 5.1; 8 x 512 into blocks after 2048 23.8 us, 4.3 TB/s: with what a
// projection has just written still in the last-level cache.  From HBM 45 and 30 us.)
// A row of one head is 16 bytes per lane (8 to 32 lanes); a wave takes as many heads as fit side by side and U tokens of them, all
// requested before the first is used: what it writes is U consecutive rows of each head.  The sum of squares and the rotation's
// partners (rot_dim / 2 elements away: a whole number of lanes) stay inside a row's lanes.  fp32 throughout, rounded once.
#include "sqa_chunk.h"

namespace sqa {

constexpr int kRowsThreads = 256;
enum { kQuery = 0, kKeyOut = 1, kKeyValue = 2 };    // what a wave's heads are: queries, keys to k_out, keys and values to the cache

struct RowsArgs {
  ChunkArgs c;
  sqa_token_rows q, k, v;
  void* q_out;
  void* k_out;                                      // NULL: to the cache
  sqa_head_prep prep;
  int q_groups, kv_groups, t_blocks;                // items of a sequence: head groups x blocks of U tokens
};

template <typename T> struct Piece;                 // 16 bytes of a row as floats
template <> struct Piece<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void open(uint4 w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Piece<bf16_t> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void open(uint4 w, float* x) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]); }
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(x[2 * i], x[2 * i + 1]);
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
};

// the value of the lane half a row away, rows of LPR lanes: where a whole head is rotated
template <int LPR> __device__ __forceinline__ float half_row_away(float v) {
  if constexpr (LPR == 16) return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, true));      // row_ror:8
  else return __shfl_xor(v, LPR / 2, LPR);
}

// May a unit take the chunk?  What its LPR lanes (lane c of them) have to know is asked for before the rows are worked on, all at
// once, and judged afterwards.  Other waves of the launch may have set the unit's state meanwhile: what is asked holds before and
// after that alike.
struct UnitAsked { ChunkUnit x; int4 state; int last, newest, block, budget; };
__device__ __forceinline__ UnitAsked ask_unit(const ChunkArgs& a, int b, int u, const ChunkSeq& s, int c) {
  UnitAsked k;
  k.x = chunk_unit(a.L, u);
  k.state = *reinterpret_cast<const int4*>(a.L.unit_state + (int64_t)u * SQA_ST_WORDS);
  k.last = s.pos > 0 && s.pos <= k.x.slots ? a.L.pos[k.x.first + s.pos - 1] : 0;
  k.budget = a.budget_seq ? a.budget_seq[b] : a.L.budget;
  const int limit = min(k.budget, k.x.slots);
  k.newest = limit > 0 ? a.L.pos[k.x.first + limit - 1] : 0;
  const int64_t entry = s.pos / SQA_BLOCK_SLOTS + c;
  k.block = k.x.table && entry <= (s.pos + s.n - 1) / SQA_BLOCK_SLOTS && entry < a.L.blocks_per_unit ? k.x.table[entry] : 0;
  return k;
}
// 0 or an error code, the same in all LPR lanes
template <int LPR>
__device__ __forceinline__ int judge_unit(const ChunkArgs& a, const UnitAsked& k, const ChunkSeq& s, int c) {
  if (a.budget_seq && (k.budget < 1 || k.budget > a.L.budget)) return SQA_ERR_BUDGET;
  const int limit = min(k.budget, k.x.slots), len = k.state.x;
  if (s.pos > k.x.slots || len < s.pos || k.state.y != 0 || (s.pos > 0 && k.last != s.pos - 1)) return SQA_ERR_STATE;
  if (s.pos + s.n > limit) return SQA_ERR_CAPACITY;
  // A full unit may have evicted, and then be taken back to its first tokens.  None of the slots from budget / 2 on then holds its own
  // position: `last` tells if it is one of them, and the newest if this call does not write it; the slots before, one by one.
  int bad = 0, outside = 0;
  if (len >= limit) {
    if (s.pos + s.n < limit) bad = k.newest != limit - 1;
    if (2 * s.pos <= limit)
      for (int64_t i = c; i < s.pos; i += LPR) bad |= a.L.pos[k.x.first + i] != i;
  }
  if (k.x.table) {
    outside = (unsigned)k.block >= (unsigned)a.L.n_blocks;
    for (int i = (int)(s.pos / SQA_BLOCK_SLOTS) + LPR + c; i <= (int)((s.pos + s.n - 1) / SQA_BLOCK_SLOTS); i += LPR)
      outside |= (unsigned)k.x.table[i] >= (unsigned)a.L.n_blocks;
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) { bad |= __shfl_xor(bad, o, LPR); outside |= __shfl_xor(outside, o, LPR); }
  return bad ? SQA_ERR_STATE : (outside ? SQA_ERR_SHAPE : 0);
}

template <typename T, int D, int U>
__global__ __launch_bounds__(kRowsThreads) void chunk_rows_kernel(const RowsArgs a) {
  constexpr int E = Piece<T>::E, LPR = D / E, HPW = SQA_WAVE / LPR;
  const int lane = threadIdx.x & (SQA_WAVE - 1), c = lane % LPR;
  const int64_t item = (int64_t)blockIdx.x * (kRowsThreads / SQA_WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / SQA_WAVE);
  const int groups = a.q_groups + a.kv_groups;
  const int tb = (int)(item % a.t_blocks);
  const int64_t bg = item / a.t_blocks;
  const int b = (int)(bg / groups), group = (int)(bg % groups);
  if (b >= a.c.B) return;
  const ChunkSeq s = chunk_seq(a.c, b, group == 0 && tb == 0 && lane == 0);
  const int t0 = tb * U;
  if (t0 >= s.n) return;
  const bool turn = a.prep.rope != nullptr;
  if (turn && s.pos + s.n > a.prep.n_pos) {
    if (group == 0 && tb == 0 && lane == 0 && a.c.status) *a.c.status = SQA_ERR_SHAPE;
    return;
  }
  const int kind = group < a.q_groups ? kQuery : (a.k_out ? kKeyOut : kKeyValue);
  const int heads = kind == kQuery ? a.c.Hq : a.c.Hkv;
  const int h = (kind == kQuery ? group : group - a.q_groups) * HPW + lane / LPR;
  const bool there = h < heads;
  const int nt = min(U, s.n - t0);

  const sqa_token_rows& src = kind == kQuery ? a.q : a.k;
  const int64_t at = (int64_t)b * src.seq_stride + (int64_t)t0 * src.row_stride + (int64_t)(there ? h : 0) * D + c * E;
  uint4 x[U], v[U];
#pragma unroll
  for (int i = 0; i < U; ++i) x[i] = ld16(static_cast<const T*>(src.data) + at + min(i, nt - 1) * src.row_stride);
  if (kind == kKeyValue) {
    const int64_t vat = (int64_t)b * a.v.seq_stride + (int64_t)t0 * a.v.row_stride + (int64_t)(there ? h : 0) * D + c * E;
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = ld16(static_cast<const T*>(a.v.data) + vat + min(i, nt - 1) * a.v.row_stride);
  }
  const int u = b * a.c.Hkv + min(h, heads - 1);
  UnitAsked asked;
  if (kind == kKeyValue) asked = ask_unit(a.c, b, u, s, c);

  // ---- norm and rotation
  const void* wp = kind == kQuery ? a.prep.q_weight : a.prep.k_weight;
  float w[E];
  if (wp) Piece<T>::open(ld16(static_cast<const T*>(wp) + c * E), w);
  const int half = a.prep.rot_dim / 2, e0 = c * E, step = a.prep.interleaved ? 0 : half / E;
  const bool mine = turn && e0 < a.prep.rot_dim, first = e0 < half;
  const int partner = mine ? (first ? lane + step : lane - step) : lane;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    float y[E];
    Piece<T>::open(x[i], y);
    if (wp) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, LPR);
      const float r = 1.f / sqrtf(ss * (1.f / D) + a.prep.eps);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = y[e] * r * w[e];
    }
    if (turn) {
      const float* row = a.prep.rope + (s.pos + t0 + min(i, nt - 1)) * a.prep.rot_dim;
      if (a.prep.interleaved) {
        if (mine) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float cs = row[(e0 + e) / 2], sn = row[half + (e0 + e) / 2];
            const float p = y[e], q = y[e + 1];
            y[e] = p * cs - q * sn;
            y[e + 1] = q * cs + p * sn;
          }
        }
      } else {
        float cs[E], sn[E];
        const float* from = row + (mine ? (first ? e0 : e0 - half) : 0);
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          *reinterpret_cast<float4*>(cs + e) = *reinterpret_cast<const float4*>(from + e);
          *reinterpret_cast<float4*>(sn + e) = *reinterpret_cast<const float4*>(from + half + e);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float other = step == LPR / 2 ? half_row_away<LPR>(y[e]) : __shfl(y[e], partner);
          const float z = fmaf(y[e], cs[e], first ? -other * sn[e] : other * sn[e]);
          y[e] = mine ? z : y[e];
        }
      }
    }
    if (wp || turn) x[i] = Piece<T>::close(y);
  }

  // ---- where they go
  if (kind != kKeyValue) {
    T* out = static_cast<T*>(kind == kQuery ? a.q_out : a.k_out) + (((int64_t)b * heads + h) * a.c.T + t0) * D + e0;
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (there && i < nt) st16(out + (int64_t)i * D, x[i]);
    return;
  }
  const ChunkUnit& unit = asked.x;
  const int why = judge_unit<LPR>(a.c, asked, s, c);
  if (!there) return;
  if (why) {
    if (c == 0 && tb == 0 && a.c.status) *a.c.status = why;
    return;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (i >= nt) break;
    const int64_t slot = s.pos + t0 + i;
    const int64_t row = unit.table ? (int64_t)unit.table[slot / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : unit.first + slot;
    st16(static_cast<T*>(a.c.L.K) + row * D + e0, x[i]);
    st16(static_cast<T*>(a.c.L.V) + row * D + e0, v[i]);
    if (c == 0) {
      a.c.L.pos[unit.first + slot] = (int32_t)slot;
      if (a.c.L.score_acc) a.c.L.score_acc[unit.first + slot] = 0.f;
    }
  }
  if (tb == 0 && c == 0)
    *reinterpret_cast<int4*>(a.c.L.unit_state + (int64_t)u * SQA_ST_WORDS) = make_int4((int)(s.pos + s.n), 0, -2, 0);
}

static bool bad_rows(const sqa_token_rows& r, int B, int T, size_t es) {
  const int64_t per16 = (int64_t)(16 / es);
  return !aligned16(r.data) || (B > 1 && (r.seq_stride < 0 || r.seq_stride % per16)) || (T > 1 && (r.row_stride < 0 || r.row_stride % per16));
}

static bool rows_overlap(const sqa_token_rows* r, int B, int T, int H, int D, size_t es, const void* p, size_t n) {
  if (!r) return false;
  const int64_t last = (B > 1 ? (int64_t)(B - 1) * r->seq_stride : 0) + (T > 1 ? (int64_t)(T - 1) * r->row_stride : 0) + (int64_t)H * D;
  return overlap(r->data, (size_t)last * es, p, n);
}

template <typename T, int D>
static void launch_rows(RowsArgs& a, hipStream_t st) {
  constexpr int HPW = SQA_WAVE / (D / Piece<T>::E);
  a.q_groups = a.q_out ? (a.c.Hq + HPW - 1) / HPW : 0;
  a.kv_groups = (a.k_out || a.c.L.K) ? (a.c.Hkv + HPW - 1) / HPW : 0;
  const int64_t groups = (int64_t)a.c.B * (a.q_groups + a.kv_groups);
  constexpr int waves = kRowsThreads / SQA_WAVE;
  // two tokens per wave where that leaves every SIMD a wave, otherwise one.  (4 x 2048 tokens of 32 + 8 heads: 35.7 us with two, 39.1
  // with four, 42.3 with one; rows stored non-temporally 34.7, but what reads them next is slower by more.  From a quarter as many waves on or
  // only from four times as many on, in us against this rule: 64 tokens 4.8 and 4.1 against 4.9, 4 x 64 appended 6.7 and 6.1 against 6.7, 2 x 512
  // 8.1 either way.)
  const bool two = groups * ((a.c.T + 1) / 2) >= 1024;
  a.t_blocks = two ? (a.c.T + 1) / 2 : a.c.T;
  const int64_t blocks = (groups * a.t_blocks + waves - 1) / waves;
  if (two) chunk_rows_kernel<T, D, 2><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
  else chunk_rows_kernel<T, D, 1><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
}

static sqa_status rows_call(const sqa_token_rows* q, const sqa_token_rows* k, const sqa_token_rows* v, sqa_dtype dt, int B, int T, int Hq,
                            int Hkv, int D, const sqa_head_prep* prep, int32_t new_pos, void* q_out, void* k_out,
                            const sqa_layer_cache* layer, void* stream, const sqa_batch_opts* opts) {
  if ((q != nullptr) != (q_out != nullptr) || (q && !q->data) || (k && !k->data) || (v && !v->data)) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  const size_t es = dt == SQA_F32 ? 4 : 2;
  if ((q && bad_rows(*q, B, T, es)) || (k && bad_rows(*k, B, T, es)) || (v && bad_rows(*v, B, T, es))) return SQA_ERR_SHAPE;
  if (!aligned16(q_out) || !aligned16(k_out)) return SQA_ERR_SHAPE;
  RowsArgs a{};
  if (prep) {
    if (!aligned16(prep->q_weight) || !aligned16(prep->k_weight) || !aligned16(prep->rope)) return SQA_ERR_SHAPE;
    if ((prep->q_weight || prep->k_weight) && !(prep->eps >= 0.f)) return SQA_ERR_SHAPE;
    if (prep->rope && (prep->n_pos < 1 || prep->rot_dim < 16 || prep->rot_dim % 16 || prep->rot_dim > D ||
                       (prep->interleaved != 0 && prep->interleaved != 1) ||
                       (!(opts && opts->new_pos_seq) && !(opts && opts->prompt_len) && (int64_t)new_pos + T > prep->n_pos)))
      return SQA_ERR_SHAPE;
    a.prep = *prep;
  }
  // (where every sequence brings T tokens at new_pos, the host sees whether they fit)
  if (layer && !(opts && (opts->prompt_len || opts->new_pos_seq)) &&
      (int64_t)new_pos + T > (layer->budget < layer->capacity ? layer->budget : layer->capacity))
    return SQA_ERR_CAPACITY;
  const size_t q_bytes = (size_t)B * Hq * T * D * es, k_bytes = (size_t)B * Hkv * T * D * es;
  auto hits = [&](const void* p, size_t n) {
    return p && (rows_overlap(q, B, T, Hq, D, es, p, n) || rows_overlap(k, B, T, Hkv, D, es, p, n) || rows_overlap(v, B, T, Hkv, D, es, p, n));
  };
  if (hits(q_out, q_bytes) || hits(k_out, k_bytes) || (q_out && k_out && overlap(q_out, q_bytes, k_out, k_bytes))) return SQA_ERR_SHAPE;
  if (layer && !layer->unit_offset) {
    const size_t c_bytes = (layer->block_table ? (size_t)layer->n_blocks * SQA_BLOCK_SLOTS : (size_t)B * Hkv * layer->capacity) * D * es;
    if (hits(layer->K, c_bytes) || hits(layer->V, c_bytes)) return SQA_ERR_SHAPE;
  }
  a.c = chunk_args(layer, B, T, Hq, Hkv, new_pos, opts);
  if (q) a.q = *q;
  if (k) a.k = *k;
  if (v) a.v = *v;
  a.q_out = q_out; a.k_out = k_out;
  // (a launch of one wave per token and head group at most)
  if ((int64_t)B * T * ((Hq + 1) / 2 + (Hkv + 1) / 2) > (int64_t)INT32_MAX) return SQA_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) D == 64 ? launch_rows<float, 64>(a, st) : launch_rows<float, 128>(a, st);
  else D == 64 ? launch_rows<bf16_t, 64>(a, st) : launch_rows<bf16_t, 128>(a, st);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}

}  // namespace sqa

extern "C" sqa_status sqa_qk_norm_rope(const sqa_token_rows* q, const sqa_token_rows* k, sqa_dtype dt, int B, int T, int Hq, int Hkv,
                                       int D, const sqa_head_prep* prep, int32_t new_pos, void* q_out, void* k_out, void* stream,
                                       const sqa_batch_opts* opts) {
  if ((!q && !k) || (k != nullptr) != (k_out != nullptr)) return SQA_ERR_NULL;
  return sqa::rows_call(q, k, nullptr, dt, B, T, Hq, Hkv, D, prep, new_pos, q_out, k_out, nullptr, stream, opts);
}

extern "C" sqa_status sqa_chunk_append(const sqa_token_rows* q, const sqa_token_rows* k, const sqa_token_rows* v, sqa_dtype dt, int B,
                                       int T, int Hq, int Hkv, int D, const sqa_head_prep* prep, int32_t new_pos, void* q_out,
                                       const sqa_layer_cache* layer, void* stream, const sqa_batch_opts* opts) {
  if (!k || !v || !layer) return SQA_ERR_NULL;
  sqa_status why;
  if (sqa::bad_layer(*layer, &why)) return why;
  return sqa::rows_call(q, k, v, dt, B, T, Hq, Hkv, D, prep, new_pos, q_out, nullptr, layer, stream, opts);
}
