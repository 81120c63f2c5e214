// Rows into a cache in 4 bits (sqa_q4_append) and back (sqa_q4_read).
//   2^e = the smallest power of two with max |x| <= 7 * 2^e over 32 neighbours;  code = round(x / 2^e) on {0, 1/2, 1, 3/2, 2, 3, 4, 6}
// Bound by memory: 2 D bytes (bf16) read and D / 2 + D / 32 written for each of K and V.  A row is 16 bytes of input per lane, as in
// sqa_chunk_rows.hip; a group is 4 (bf16) or 8 (fp32) of those lanes, whose largest |x| meet by DPP; the rounding is the conversion
// instruction, which divides by the power and rounds ties to the even code.
#include "sqa_q4.h"
#include "sqa_rows.h"

namespace sqa {

struct Q4RowsArgs {
  Q4Args a;
  sqa_token_rows q, k, v;
  void* q_out;
  sqa_head_prep prep;
  AxesArgs axes;
  const int32_t* slot_map;
  int64_t rows;                                     // of the cache
  int q_groups, kv_groups;                          // groups of heads, as many as a wave's lanes hold rows
};

// E numbers of a lane, LPG lanes of which are a group: codes in the low 4 E bits, and the group's byte
template <int E> __device__ __forceinline__ uint32_t q4_round(const float (&y)[E], uint32_t& power) {
  constexpr int LPG = kGroup / E;
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
  auto of = [&](int x) { top = max(top, (uint32_t)x); };
  of(__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));                    // lanes 1, then 2 away
  of(__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
  if constexpr (LPG == 8) of(__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xF, 0xF, true));   // the other four of eight
  power = q4_power(top);
  const float scale = __uint_as_float(min(power, 252u) << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  if constexpr (E == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  }
  return w;
}

// A wave takes one token and U groups of heads: slots and angles are the same for all of them.
template <typename T, int D, int U, bool AXES>
__global__ __launch_bounds__(kRowsThreads) void q4_rows_kernel(const Q4RowsArgs a) {
  constexpr int E = Piece<T>::E, LPR = D / E, HPW = SQA_WAVE / LPR, LPG = kGroup / E;
  const int lane = threadIdx.x & (SQA_WAVE - 1), c = lane % LPR;
  const int64_t item = (int64_t)blockIdx.x * (kRowsThreads / SQA_WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / SQA_WAVE);
  const int groups = a.q_groups + a.kv_groups, runs = (groups + U - 1) / U, T_ = a.a.c.T;
  const int t = (int)(item % T_);
  const int64_t br = item / T_;
  const int b = (int)(br / runs), first = (int)(br % runs) * U;
  if (b >= a.a.c.B) return;
  const bool reports = first == 0 && lane == 0;
  const Q4Seq s = q4_seq(a.a, b, reports && t == 0);
  if (t >= s.n) return;
  const bool turn = a.prep.rope != nullptr;
  if (!AXES && turn && s.pos + s.n > a.prep.n_pos) {
    if (reports && t == 0 && a.a.c.status) *a.a.c.status = SQA_ERR_SHAPE;
    return;
  }
  const bool stores = a.slot_map || !s.why;         // (queries are written all the same)
  if (!stores && reports && t == 0 && a.a.c.status) *a.a.c.status = s.why;
  const int slot = stores && !a.slot_map ? s.slot(s.pos + t) : 0;

  auto head_of = [&](int group) { return (group < a.q_groups ? group : group - a.q_groups) * HPW + lane / LPR; };
  uint4 x[U], v[U];
  int64_t row[U];                                   // of the cache
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int group = min(first + i, groups - 1);
    const bool query = group < a.q_groups;
    const sqa_token_rows& src = query ? a.q : a.k;
    const int h = min(head_of(group), (query ? a.a.c.Hq : a.a.c.Hkv) - 1);
    const int64_t at = (int64_t)h * D + c * E;
    x[i] = ld16(static_cast<const T*>(src.data) + (int64_t)b * src.seq_stride + (int64_t)t * src.row_stride + at);
    if (!query) {
      v[i] = ld16(static_cast<const T*>(a.v.data) + (int64_t)b * a.v.seq_stride + (int64_t)t * a.v.row_stride + at);
      const int64_t u = (int64_t)b * a.a.c.Hkv + h;
      row[i] = a.slot_map ? a.slot_map[u * T_ + t]
             : a.a.L.block_table ? (int64_t)a.a.L.block_table[u * a.a.L.blocks_per_unit + slot / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS
                                 : u * a.a.L.capacity + slot;
    }
  }
  RowPrep<T, D> how(a.prep, lane);
  float cs[E], sn[E];
  if constexpr (AXES) {
    __shared__ float s_angles[kRowsThreads / SQA_WAVE][128];
    how.angles_of(a.axes, axes_of(a.axes, a.a.c, a.prep.n_pos, b, t, reports), s_angles[threadIdx.x / SQA_WAVE], cs, sn);
  } else if (turn) {
    how.angles_of(s.pos + t, cs, sn);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int group = first + i;
    if (group >= groups) break;
    const bool query = group < a.q_groups;
    const int h = head_of(group);
    const bool there = h < (query ? a.a.c.Hq : a.a.c.Hkv);
    float y[E];
    Piece<T>::open(x[i], y);
    how.normalise(y, query ? a.prep.q_weight : a.prep.k_weight);
    if (turn) how.turn(y, cs, sn);
    if (query) {
      const uint4 w = Piece<T>::close(y);
      if (there) st16(static_cast<T*>(a.q_out) + (((int64_t)b * a.a.c.Hq + h) * T_ + t) * D + c * E, w);
      continue;
    }
    if (!stores) continue;
    const bool inside = (uint64_t)row[i] < (uint64_t)a.rows;
    if (there && c == 0 && !inside && !(a.slot_map && row[i] == -1) && a.a.c.status) *a.a.c.status = SQA_ERR_SHAPE;
    const bool put = there && inside;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      if (kv) Piece<T>::open(v[i], y);
      uint32_t power;
      const uint32_t w = q4_round(y, power);
      if (!put) continue;
      char* const to = static_cast<char*>(kv ? a.a.L.V : a.a.L.K) + row[i] * (D / 2) + c * (E / 2);
      if constexpr (E == 8) *reinterpret_cast<uint32_t*>(to) = w;
      else *reinterpret_cast<uint16_t*>(to) = (uint16_t)w;
      if (c % LPG == 0) (kv ? a.a.L.V_scale : a.a.L.K_scale)[row[i] * (D / kGroup) + c / LPG] = (uint8_t)power;
    }
  }
}

// A lane takes 8 elements: 4 bytes of codes, 16 or 32 of numbers.
struct Q4ReadArgs { Q4Args a; void* k_out; void* v_out; };
template <typename T, int D> __global__ __launch_bounds__(kRowsThreads) void q4_read_kernel(const Q4ReadArgs a) {
  constexpr int LPR = D / 8;
  const int64_t i = (int64_t)blockIdx.x * kRowsThreads + threadIdx.x;
  const int64_t r = i / LPR;
  const int c = (int)(i % LPR);
  const int t = (int)(r % a.a.c.T);
  const int64_t u = r / a.a.c.T;
  if (u >= (int64_t)a.a.c.B * a.a.c.Hkv) return;
  const int b = (int)(u / a.a.c.Hkv);
  const bool reports = c == 0 && t == 0 && u % a.a.c.Hkv == 0;
  ChunkSeq s = chunk_seq(a.a.c, b, reports);
  int slots = a.a.L.capacity;
  if (a.a.c.budget_seq) {
    slots = a.a.c.budget_seq[b];
    if (slots <= a.a.L.n_sink || slots > a.a.L.capacity) {
      if (reports && s.n && a.a.c.status) *a.a.c.status = SQA_ERR_BUDGET;
      return;
    }
  }
  if (t >= s.n) return;
  const int64_t slot = s.pos + t;
  if (slot >= slots) {
    if (c == 0 && a.a.c.status) *a.a.c.status = SQA_ERR_CAPACITY;
    return;
  }
  int64_t row = u * a.a.L.capacity + slot;
  if (a.a.L.block_table) {
    const int block = a.a.L.block_table[u * a.a.L.blocks_per_unit + slot / SQA_BLOCK_SLOTS];
    if ((unsigned)block >= (unsigned)a.a.L.n_blocks) {
      if (c == 0 && a.a.c.status) *a.a.c.status = SQA_ERR_SHAPE;
      return;
    }
    row = (int64_t)block * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS;
  }
  auto read = [&](const void* codes, const uint8_t* powers, void* out) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const char*>(codes) + row * (D / 2) + 4 * c);
    const float scale = __uint_as_float((uint32_t)powers[row * (D / kGroup) + c / 4] << 23);
    const uint4 x = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
    T* const to = static_cast<T*>(out) + r * D + 8 * c;
    if constexpr (sizeof(T) == 2) st16(to, x);
    else {
      st16(to, make_uint4(x.x << 16, x.x & 0xffff0000u, x.y << 16, x.y & 0xffff0000u));
      st16(to + 4, make_uint4(x.z << 16, x.z & 0xffff0000u, x.w << 16, x.w & 0xffff0000u));
    }
  };
  if (a.k_out) read(a.a.L.K, a.a.L.K_scale, a.k_out);
  if (a.v_out) read(a.a.L.V, a.a.L.V_scale, a.v_out);
}

template <typename T, int D> static void launch_q4_rows(Q4RowsArgs& a, hipStream_t st) {
  constexpr int HPW = SQA_WAVE / (D / Piece<T>::E), waves = kRowsThreads / SQA_WAVE;
  a.q_groups = a.q_out ? (a.a.c.Hq + HPW - 1) / HPW : 0;
  a.kv_groups = (a.a.c.Hkv + HPW - 1) / HPW;
  const int groups = a.q_groups + a.kv_groups;
  const bool four = (int64_t)a.a.c.B * a.a.c.T * ((groups + 3) / 4) >= 2048;        // (two waves per SIMD)
  const int64_t items = (int64_t)a.a.c.B * a.a.c.T * (four ? (groups + 3) / 4 : groups);
  const unsigned blocks = (unsigned)((items + waves - 1) / waves);
  if (a.axes.n) four ? q4_rows_kernel<T, D, 4, true><<<blocks, kRowsThreads, 0, st>>>(a) : q4_rows_kernel<T, D, 1, true><<<blocks, kRowsThreads, 0, st>>>(a);
  else four ? q4_rows_kernel<T, D, 4, false><<<blocks, kRowsThreads, 0, st>>>(a) : q4_rows_kernel<T, D, 1, false><<<blocks, kRowsThreads, 0, st>>>(a);
}

}  // namespace sqa

extern "C" sqa_status sqa_q4_append(const sqa_token_rows* q, const sqa_token_rows* k, const sqa_token_rows* v, sqa_dtype dt, int B, int T,
                                    int Hq, int Hkv, int D, const sqa_head_prep* prep, int32_t new_pos, void* q_out, const sqa_q4_cache* layer,
                                    void* stream, const sqa_batch_opts* opts, const sqa_rope_axes* axes, const int32_t* slot_map) {
  using namespace sqa;
  if (!k || !v || !layer || !k->data || !v->data || (q != nullptr) != (q_out != nullptr) || (q && !q->data)) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  sqa_status why;
  if (bad_q4(*layer, D, &why)) return why;
  const size_t es = dt == SQA_F32 ? 4 : 2;
  if ((q && bad_rows(*q, B, T, es)) || bad_rows(*k, B, T, es) || bad_rows(*v, B, T, es) || !aligned16(q_out) || (reinterpret_cast<uintptr_t>(slot_map) & 3u)) return SQA_ERR_SHAPE;
  Q4RowsArgs a{};
  if (prep) {
    if ((why = check_prep(*prep, D, axes, new_pos, T, opts))) return why;
    a.prep = *prep;
  }
  if (axes && !axes_args(axes, prep, &a.axes, &why)) return why;
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  // (where every sequence brings T tokens at new_pos, the host sees whether they would overwrite their own)
  if (uniform && !slot_map && (int64_t)new_pos + T > layer->capacity && T > layer->capacity - layer->n_sink) return SQA_ERR_CAPACITY;
  a.rows = q4_rows(*layer, B, Hkv);
  const size_t q_bytes = (size_t)B * Hq * T * D * es, c_bytes = (size_t)a.rows * D / 2, p_bytes = (size_t)a.rows * D / kGroup;
  auto hits = [&](const void* p, size_t n) {
    return p && (rows_overlap(q, B, T, Hq, D, es, p, n) || rows_overlap(k, B, T, Hkv, D, es, p, n) || rows_overlap(v, B, T, Hkv, D, es, p, n));
  };
  if (hits(q_out, q_bytes) || hits(layer->K, c_bytes) || hits(layer->V, c_bytes) || hits(layer->K_scale, p_bytes) || hits(layer->V_scale, p_bytes))
    return SQA_ERR_SHAPE;
  if (in_q4(*layer, B, Hkv, D, q_out, q_bytes)) return SQA_ERR_SHAPE;
  // (keys and values are written at once; a call that only reads may be given one pool for both)
  if (overlap(layer->K, c_bytes, layer->V, c_bytes) || overlap(layer->K_scale, p_bytes, layer->V_scale, p_bytes)) return SQA_ERR_SHAPE;
  for (const void* codes : {layer->K, layer->V})
    if (overlap(codes, c_bytes, layer->K_scale, p_bytes) || overlap(codes, c_bytes, layer->V_scale, p_bytes)) return SQA_ERR_SHAPE;
  const size_t m_bytes = (size_t)B * Hkv * T * sizeof(int32_t);
  if (slot_map && (in_q4(*layer, B, Hkv, D, slot_map, m_bytes) || (q_out && overlap(slot_map, m_bytes, q_out, q_bytes)))) return SQA_ERR_SHAPE;
  if ((int64_t)B * T * ((Hq + 1) / 2 + (Hkv + 1) / 2) > (int64_t)INT32_MAX) return SQA_ERR_SHAPE;
  a.a = q4_args(layer, B, T, Hq, Hkv, new_pos, opts);
  if (q) a.q = *q;
  a.k = *k; a.v = *v; a.q_out = q_out; a.slot_map = slot_map;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) D == 64 ? launch_q4_rows<float, 64>(a, st) : launch_q4_rows<float, 128>(a, st);
  else D == 64 ? launch_q4_rows<bf16_t, 64>(a, st) : launch_q4_rows<bf16_t, 128>(a, st);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}

extern "C" sqa_status sqa_q4_read(const sqa_q4_cache* layer, sqa_dtype dt, int B, int T, int Hkv, int D, int32_t first_slot, void* k_out,
                                  void* v_out, void* stream, const sqa_batch_opts* opts) {
  using namespace sqa;
  if (!layer || (!k_out && !v_out)) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (bad_chunk_shape(B, T, Hkv, Hkv, D, first_slot, opts) || !aligned16(k_out) || !aligned16(v_out)) return SQA_ERR_SHAPE;
  sqa_status why;
  if (bad_q4(*layer, D, &why)) return why;
  if (!(opts && (opts->prompt_len || opts->new_pos_seq || opts->budget_seq)) && (int64_t)first_slot + T > layer->capacity) return SQA_ERR_CAPACITY;
  const size_t out_bytes = (size_t)B * Hkv * T * D * (dt == SQA_F32 ? 4 : 2);
  if (k_out && v_out && overlap(k_out, out_bytes, v_out, out_bytes)) return SQA_ERR_SHAPE;
  if (in_q4(*layer, B, Hkv, D, k_out, out_bytes) || in_q4(*layer, B, Hkv, D, v_out, out_bytes)) return SQA_ERR_SHAPE;
  const int64_t threads = (int64_t)B * Hkv * T * (D / 8), blocks = (threads + kRowsThreads - 1) / kRowsThreads;
  if (blocks > INT32_MAX) return SQA_ERR_SHAPE;
  Q4ReadArgs a{q4_args(layer, B, T, Hkv, Hkv, first_slot, opts), k_out, v_out};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) {
    if (D == 64) q4_read_kernel<float, 64><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
    else q4_read_kernel<float, 128><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
  } else {
    if (D == 64) q4_read_kernel<bf16_t, 64><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
    else q4_read_kernel<bf16_t, 128><<<(unsigned)blocks, kRowsThreads, 0, st>>>(a);
  }
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}
