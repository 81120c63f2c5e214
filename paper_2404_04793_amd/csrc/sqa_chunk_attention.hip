// Causal attention of a chunk of tokens over a layer cache that holds it (sqa_chunk_attention).
//   out_t = sum_j exp(s_tj - m_t) V_j / l_t,  s_tj = q_t.K_j / sqrt(D),  l_t = sum_j exp(s_tj - m_t),  j <= position of t
// One pass over the slots with a running maximum m and sum l per row.  The g query heads of a KV head and the chunk's tokens
// are one list of rows, row r = token r / g, head r % g: K and V are read once for all of them.  A workgroup of 4
// waves takes 32 RW of these rows, RW = 4, 2 or 1 by their number; with RW < 4 the 4 / RW waves of the same rows share
// out the slots of a tile and join at the end.  Few rows against many slots are shared out over workgroups too; their
// (m, l, sums) go through the workspace and the last one to arrive joins them, in order.
//   S^T = K.Q^T  a lane holds 16 of 32 slots of one row: maximum and sum need one exchange between the two lane halves, and
//                the probabilities are the next product's operand as they are
//   O^T = V^T.P^T  a row's sums lie in the two lanes of its column: rescaling is a multiplication by a lane's own number
// K and V tiles go from global memory straight to LDS, two buffers, in an order without bank conflicts (TileRows).
#include "sqa_chunk_mma.h"

namespace sqa {

constexpr int kAtThreads = 256;
constexpr float kFarLogit = 64.f;                   // in powers of two: below it the rounding is 2e-6 at most
constexpr int kAtItems = 512;                       // workgroups that few rows are shared out to: two per CU

struct AttentionArgs {
  ChunkArgs c;
  const void* q;
  void* out;
  float* lse;
  int32_t* count;                                   // [items]
  float2* part;                                     // [items][splits][32 RW][D / 2 + 1]: a row's sums, then (m, l)
  float scale;                                      // log2(e) / sqrt(D)
  int tiles, splits;
};

template <typename T, int D, int RW, int KT> struct AttentionTile {
  using R = TileRows<T, D>;
  static constexpr int KW = 4 / RW, KB = KT / KW / 32, M = 32 * RW, NB = D / 32;
  static constexpr int TILE = KT * R::RB;
  static constexpr int STAGE = 4 * TILE > 4 * 32 * D * 4 ? 4 * TILE : 4 * 32 * D * 4;
};

// Does a tile of BYTES bytes in LDS hold a number that is not finite?  This thread's share of it; CLEAR: such numbers become 0.
template <typename T, int BYTES, bool CLEAR> __device__ __forceinline__ bool odd_values(char* tile) {
  bool odd = false;
#pragma unroll 1
  for (int i = threadIdx.x * 16; i < BYTES; i += kAtThreads * 16) {
    const uint4 w = *reinterpret_cast<const uint4*>(tile + i);
    uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) {
        const bool lo = (v[k] & 0x7f80u) == 0x7f80u, hi = (v[k] & 0x7f800000u) == 0x7f800000u;
        odd |= lo || hi;
        if constexpr (CLEAR) v[k] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
      } else {
        const bool x = (v[k] & 0x7f800000u) == 0x7f800000u;
        odd |= x;
        if constexpr (CLEAR) v[k] = x ? 0u : v[k];
      }
    }
    if constexpr (CLEAR) *reinterpret_cast<uint4*>(tile + i) = make_uint4(v[0], v[1], v[2], v[3]);
  }
  return odd;
}

template <typename T, int D, int RW, int KT>
__global__ __launch_bounds__(kAtThreads, 2) void chunk_attention_kernel(const AttentionArgs a) {
  using C = AttentionTile<T, D, RW, KT>;
  using R = TileRows<T, D>;
  constexpr int KW = C::KW, KB = C::KB, M = C::M, NB = C::NB;
  extern __shared__ char s_stage[];
  __shared__ float s_m[KW][M], s_l[KW][M];
  __shared__ int s_word;
  int* const s_table = reinterpret_cast<int*>(s_stage + C::STAGE);

  const int64_t items = (int64_t)a.c.B * a.c.Hkv * a.tiles;
  const int64_t work = xcd_item(items * a.splits);
  if (work < 0) return;
  const int split = (int)(work % a.splits);
  const int64_t item = work / a.splits;
  const int u = (int)(item / a.tiles), tile = a.tiles - 1 - (int)(item % a.tiles);     // the longest first
  const int b = u / a.c.Hkv, h = u % a.c.Hkv, g = a.c.g;
  const ChunkSeq seq = chunk_seq(a.c, b, threadIdx.x == 0 && h == 0 && tile == 0 && split == 0);
  const int rows = seq.n * g, row0 = tile * M;
  if (row0 >= rows) return;
  const ChunkUnit unit = chunk_unit(a.c.L, u);
  const int last_row = min(row0 + M, rows) - 1;
  const int end = __builtin_amdgcn_readfirstlane((int)min(seq.pos + last_row / g + 1, (int64_t)INT32_MAX));   // slots that the tile's rows see

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, col = lane & 31, half = lane >> 5;

  // ---- does the unit hold the chunk, and do its blocks lie in the pools
  int why = chunk_held(a.c.L, unit, u, seq.pos + seq.n) ? 0 : SQA_ERR_STATE;
  if (!why && unit.table) {
    int outside = 0;
    for (int i = tid; i < (end + SQA_BLOCK_SLOTS - 1) / SQA_BLOCK_SLOTS; i += kAtThreads) {
      const int blk = unit.table[i];
      s_table[i] = blk;
      outside |= (unsigned)blk >= (unsigned)a.c.L.n_blocks;
    }
    if (__syncthreads_or(outside)) why = SQA_ERR_SHAPE;
  }
  auto place = [&](int r, int& t, int& head) { t = r / g; head = h * g + r % g; };
  T* const out = static_cast<T*>(a.out);
  if (why) {
    if (split) return;
    if (tid == 0 && a.c.status) *a.c.status = why;
    for (int i = tid; i < (last_row + 1 - row0) * R::PPR; i += kAtThreads) {
      int t, head;
      place(row0 + i / R::PPR, t, head);
      st16(out + (((int64_t)b * a.c.T + t) * a.c.Hq + head) * D + i % R::PPR * R::E, make_uint4(0, 0, 0, 0));
      if (a.lse && i % R::PPR == 0) a.lse[((int64_t)b * a.c.Hq + head) * a.c.T + t] = -INFINITY;
    }
    return;
  }

  // ---- the slots of this workgroup, in tiles of KT
  const int nt = (end + KT - 1) / KT, per = (nt + a.splits - 1) / a.splits;
  const int parts = (nt + per - 1) / per;
  if (split >= parts) return;
  const int tile0 = split * per, tile1 = min(tile0 + per, nt);

  // ---- this lane's query row
  const int r = row0 + 32 * rw + col;
  const bool mine = r < rows;
  int t, head;
  place(mine ? r : row0, t, head);
  const int see = (int)(seq.pos + t);                                                    // the last slot that the row sees
  const int see_all = (int)(seq.pos + min(row0 + 32 * rw, last_row) / g);                // ... that all of the wave's rows see
  const int see_all_tile = (int)(seq.pos + row0 / g);                                    // ... all of the workgroup's
  Frag<T, D> q;
  {
    const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (((int64_t)b * a.c.Hq + head) * a.c.T + t) * D);
#pragma unroll
    for (int s = 0; s < q.NS; ++s) q.p[s] = mine ? ld16(src + (2 * s + half) * 16) : make_uint4(0, 0, 0, 0);
  }

  // ---- copies of one tile: each wave the rows wave KT/4 .. of K and of V
  const char* const Kp = static_cast<const char*>(a.c.L.K);
  const char* const Vp = static_cast<const char*>(a.c.L.V);
  auto fetch = [&](int tl, int buf) {
    const uint32_t dst = lds_at(s_stage) + (uint32_t)(buf * 2 * C::TILE);
#pragma unroll
    for (int i = 0; i < KT / 4 / R::RPI; ++i) {
      const int rr = wave * (KT / 4) + i * R::RPI, row = rr + lane / R::PPR;
      const int slot = min(tl * KT + row, end - 1);
      const int64_t at = unit.table ? (int64_t)s_table[slot / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : unit.first + slot;
      fetch16(Kp + at * R::RB + (((lane % R::PPR) ^ R::k_swizzle(row)) << 4), dst + rr * R::RB);
      fetch16(Vp + at * R::RB + (((lane % R::PPR) ^ R::v_swizzle(row)) << 4), dst + C::TILE + rr * R::RB);
    }
  };

  f32x16_t o[NB];
#pragma unroll
  for (int e = 0; e < NB; ++e) o[e] = f32x16_t{};
  float m = -FLT_MAX, l = 0.f;                       // (finite: a row that sees nothing yet has no exp(inf - inf))

  fetch(tile0, 0);
  for (int tl = tile0; tl < tile1; ++tl) {
    const int buf = (tl - tile0) & 1;
    fetched();
    __syncthreads();
    if (tl + 1 < tile1) fetch(tl + 1, buf ^ 1);
    const char* const Kt = s_stage + buf * 2 * C::TILE;
    const char* const Vt = Kt + C::TILE;
    const int key0 = kw * (KT / KW);

    f32x16_t s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = f32x16_t{};
      const int row = key0 + 32 * kb + col;
#pragma unroll
      for (int x = 0; x < q.NS; ++x) {
        const uint4 k = *reinterpret_cast<const uint4*>(Kt + row * R::RB + (((2 * x + half) ^ R::k_swizzle(row)) << 4));
        mma_piece<T>(k, q.p[x], s[kb]);
      }
    }
    const int first = tl * KT + key0;
    if (first + 32 * KB - 1 > see_all) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (first + 32 * kb + c_row(i, half) > see) s[kb][i] = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    top = other_half_max(top);
    const float keep = exp2_fast((m - top) * a.scale);
    float off = top * a.scale;
    m = top;
    // s scale - off in one operation is off by the rounding of `off`: far from 0 the difference is taken first
    if (__any(fabsf(off) > kFarLogit)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] -= top;
      off = 0.f;
    }
    l *= keep;
#pragma unroll
    for (int e = 0; e < NB; ++e) o[e] *= keep;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[kb][i] = exp2_fast(fmaf(s[kb][i], a.scale, -off));
        l += s[kb][i];
      }

    // A slot that a row does not see has probability 0, but 0 x NaN is NaN: where some rows do not see all of the tile, its
    // values that are not finite are added to the sums of the rows that see them one by one, and are 0 for the product.
    if (tl * KT + KT - 1 > see_all_tile && __syncthreads_or(odd_values<T, C::TILE, false>(s_stage + buf * 2 * C::TILE + C::TILE))) {
#pragma unroll 1
      for (int k = 0; k < 32 * KB; ++k) {
        const int row = key0 + k;
        const bool seen = tl * KT + row <= see;
#pragma unroll
        for (int e = 0; e < NB; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int d = sizeof(T) == 2 ? 32 * e + c_row(i, half) : NB * c_row(i, half) + e;
            const int at = row * R::RB + (((d / R::E) ^ R::v_swizzle(row)) << 4) + d % R::E * (int)sizeof(T);
            float v;
            if constexpr (sizeof(T) == 2) v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(Vt + at) << 16);
            else v = *reinterpret_cast<const float*>(Vt + at);
            if (seen && !isfinite(v)) o[e][i] += v;
          }
      }
      __syncthreads();
      odd_values<T, C::TILE, true>(s_stage + buf * 2 * C::TILE + C::TILE);
      __syncthreads();
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int row = key0 + 32 * kb;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          bf16x8_t p;
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = (__bf16)s[kb][8 * ks + i];
          const int vr = row + 16 * ks + 4 * half + (lane & 15) / 4;
#pragma unroll
          for (int e = 0; e < NB; ++e) {
            const int piece = (4 * e + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ R::v_swizzle(vr);
            const char* at = Vt + vr * R::RB + piece * 16 + (lane & 1) * 8;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 8 * R::RB));
            const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o[e], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float* at = reinterpret_cast<const float*>(Vt + (row + c_row(i, half)) * R::RB) + NB * col;
          float v[NB];
#pragma unroll
          for (int e = 0; e < NB; ++e) v[e] = at[e];
#pragma unroll
          for (int e = 0; e < NB; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], s[kb][i], o[e], 0, 0, 0);
        }
      }
    }
  }
  l = other_half_sum(l);

  // ---- the waves of the same rows join: their sums as one list of 32 rows each in LDS, 16-byte pieces exchanged by the row
  __syncthreads();
  if (half == 0) { s_m[kw][32 * rw + col] = m; s_l[kw][32 * rw + col] = l; }
  if constexpr (KW > 1) {
    __syncthreads();
    float top = s_m[0][32 * rw + col];
#pragma unroll
    for (int k = 1; k < KW; ++k) top = fmaxf(top, s_m[k][32 * rw + col]);
    const float w = exp2_fast((m - top) * a.scale);
#pragma unroll
    for (int e = 0; e < NB; ++e) o[e] *= w;
  }
  constexpr int PP = D / 4;                          // pieces of a row of sums
  float4* const mine4 = reinterpret_cast<float4*>(s_stage) + (kw * M + 32 * rw + col) * PP;
#pragma unroll
  for (int i = 0; i < 16; i += 4)
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < NB; ++e) mine4[(8 * e + c_row(i, half) / 4) ^ (col & 15)] = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
    } else if constexpr (NB == 4) {
#pragma unroll
      for (int x = i; x < i + 4; ++x) mine4[c_row(x, half) ^ (col & 15)] = make_float4(o[0][x], o[1][x], o[2][x], o[3][x]);
    } else {
#pragma unroll
      for (int x = i; x < i + 4; x += 2) mine4[(c_row(x, half) / 2) ^ (col & 15)] = make_float4(o[0][x], o[1][x], o[0][x + 1], o[1][x + 1]);
    }
  __syncthreads();
  auto joined = [&](int row, float& mm, float& ll) {
    mm = s_m[0][row];
#pragma unroll
    for (int k = 1; k < KW; ++k) mm = fmaxf(mm, s_m[k][row]);
    ll = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) ll += s_l[k][row] * (KW > 1 ? exp2_fast((s_m[k][row] - mm) * a.scale) : 1.f);
  };
  auto piece4 = [&](int row, int p) {
    float4 v = reinterpret_cast<const float4*>(s_stage)[row * PP + (p ^ (row & 15))];
#pragma unroll
    for (int k = 1; k < KW; ++k) {
      const float4 x = reinterpret_cast<const float4*>(s_stage)[(k * M + row) * PP + (p ^ (row & 15))];
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    return v;
  };
  auto store4 = [&](int row, int p, float4 v, float mm, float ll) {
    int tt, hh;
    place(row0 + row, tt, hh);
    const float inv = 1.f / ll;
    T* dst = out + (((int64_t)b * a.c.T + tt) * a.c.Hq + hh) * D + 4 * p;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(dst) = make_uint2(f32_to_bf16_bits(v.x * inv) | (f32_to_bf16_bits(v.y * inv) << 16),
                                                  f32_to_bf16_bits(v.z * inv) | (f32_to_bf16_bits(v.w * inv) << 16));
    else
      *reinterpret_cast<float4*>(dst) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    if (p == 0 && a.lse) a.lse[((int64_t)b * a.c.Hq + hh) * a.c.T + tt] = 0.6931471805599453f * fmaf(mm, a.scale, log2f(ll));
  };
  const int live = (last_row + 1 - row0) * PP;
  if (parts == 1) {
    for (int i = tid; i < live; i += kAtThreads) {
      float mm, ll;
      joined(i / PP, mm, ll);
      store4(i / PP, i % PP, piece4(i / PP, i % PP), mm, ll);
    }
    return;
  }

  // ---- ... and the workgroups of the same rows
  constexpr int REC = D / 2 + 1;
  float2* const rec = a.part + (item * a.splits) * M * REC;
  for (int i = tid; i < live; i += kAtThreads) {
    const int row = i / PP, p = i % PP;
    float2* dst = rec + ((int64_t)split * M + row) * REC;
    const float4 v = piece4(row, p);
    hand_over(dst + 2 * p, make_float2(v.x, v.y));
    hand_over(dst + 2 * p + 1, make_float2(v.z, v.w));
    if (p == 0) {
      float mm, ll;
      joined(row, mm, ll);
      hand_over(dst + D / 2, make_float2(mm, ll));
    }
  }
  if (!last_to_arrive(a.count + item, parts, &s_word)) return;
  for (int i = tid; i < live; i += kAtThreads) {
    const int row = i / PP, p = i % PP;
    float mm = -FLT_MAX, ll = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < parts; ++k) mm = fmaxf(mm, handed_over(rec + ((int64_t)k * M + row) * REC + D / 2).x);
    for (int k = 0; k < parts; ++k) {
      const float2* src = rec + ((int64_t)k * M + row) * REC;
      const float2 ml = handed_over(src + D / 2), x = handed_over(src + 2 * p), y = handed_over(src + 2 * p + 1);
      const float w = exp2_fast((ml.x - mm) * a.scale);
      ll = fmaf(ml.y, w, ll);
      v.x = fmaf(x.x, w, v.x); v.y = fmaf(x.y, w, v.y); v.z = fmaf(y.x, w, v.z); v.w = fmaf(y.y, w, v.w);
    }
    store4(row, p, v, mm, ll);
  }
}

struct AttentionPlan { int rw, tiles, splits; };
// (rows of 512 bytes have no form for 32 rows: its tiles would not fit the LDS)
static int attention_rw(int rows, bool rows_of_512) { return rows <= 32 && !rows_of_512 ? 1 : (rows <= 64 ? 2 : 4); }
static AttentionPlan attention_plan(sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t slots) {
  AttentionPlan p;
  const int rows = T * (Hq / Hkv);
  p.rw = attention_rw(rows, dt == SQA_F32 && D == 128);
  p.tiles = (rows + 32 * p.rw - 1) / (32 * p.rw);
  const int64_t items = (int64_t)B * Hkv * p.tiles;
  int64_t s = kAtItems / items;
  s = s > slots / 256 ? slots / 256 : s;             // (a workgroup's start and the join cost what some hundred slots do)
  p.splits = s < 1 ? 1 : (int)s;
  return p;
}
// (any T' <= T, any length: items x splits <= kAtItems where there are splits)
size_t chunk_attention_scratch(int B, int T, int Hq, int Hkv, int D, int64_t slots) {
  (void)B; (void)slots;
  return (size_t)kAtItems * 32 * attention_rw(T * (Hq / Hkv), D == 128) * (D / 2 + 1) * sizeof(float2);
}

template <typename T, int D, int RW, int KT>
static sqa_status launch_attention(const AttentionArgs& a, hipStream_t st) {
  using C = AttentionTile<T, D, RW, KT>;
  const auto fn = chunk_attention_kernel<T, D, RW, KT>;
  size_t lds = C::STAGE;
  if (a.c.L.block_table) lds += (size_t)(a.c.L.blocks_per_unit + 3) / 4 * 16;
  SQA_HIP_CHECK(allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds));
  const int64_t work = (int64_t)a.c.B * a.c.Hkv * a.tiles * a.splits;
  fn<<<(unsigned)xcd_grid(work), kAtThreads, lds, st>>>(a);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}
template <typename T, int D>
static sqa_status launch_attention(int rw, const AttentionArgs& a, hipStream_t st) {
  constexpr bool wide = D * sizeof(T) == 512;        // rows of 512 bytes: half the slots
  if (rw == 4) return launch_attention<T, D, 4, wide ? 32 : 64>(a, st);
  if constexpr (wide) return launch_attention<T, D, 2, 64>(a, st);
  else return rw == 2 ? launch_attention<T, D, 2, 64>(a, st) : launch_attention<T, D, 1, 128>(a, st);
}

}  // namespace sqa

extern "C" size_t sqa_chunk_workspace_bytes(const sqa_layer_cache* layer, int B, int T, int Hq, int Hkv, int D) {
  sqa_status why;
  if (!layer || sqa::bad_layer(*layer, &why) || sqa::bad_chunk_shape(B, T, Hq, Hkv, D, 0, nullptr)) return 0;
  const size_t x = sqa::chunk_attention_scratch(B, T, Hq, Hkv, D, layer->capacity);
  const size_t y = sqa::chunk_scores_scratch(B, T, Hq, Hkv, D, layer->capacity);
  return (sqa::kChunkCounterBytes + (x > y ? x : y) + 255) / 256 * 256;
}

extern "C" sqa_status sqa_chunk_attention(const void* q, sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos,
                                          const sqa_layer_cache* layer, void* out, float* lse, void* workspace, size_t ws_bytes,
                                          void* stream, const sqa_batch_opts* opts) {
  if (!q || !layer || !out || !workspace) return SQA_ERR_NULL;
  sqa_status why;
  if (sqa::bad_layer(*layer, &why)) return why;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (sqa::bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  if (!sqa::aligned16(q) || !sqa::aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return SQA_ERR_SHAPE;
  if (ws_bytes < sqa_chunk_workspace_bytes(layer, B, T, Hq, Hkv, D)) return SQA_ERR_CAPACITY;
  if (!(opts && (opts->prompt_len || opts->new_pos_seq)) && (int64_t)new_pos + T > layer->capacity) return SQA_ERR_CAPACITY;
  const size_t es = dt == SQA_F32 ? 4 : 2, qb = (size_t)B * Hq * T * D * es, lb = (size_t)B * Hq * T * sizeof(float);
  if (sqa::overlap(q, qb, out, qb) || (lse && (sqa::overlap(lse, lb, q, qb) || sqa::overlap(lse, lb, out, qb)))) return SQA_ERR_SHAPE;
  sqa::AttentionArgs a{};
  a.c = sqa::chunk_args(layer, B, T, Hq, Hkv, new_pos, opts);
  a.q = q; a.out = out; a.lse = lse;
  a.count = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float2*>(static_cast<char*>(workspace) + sqa::kChunkCounterBytes);
  a.scale = (float)(1.4426950408889634 / sqrt((double)D));
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  const sqa::AttentionPlan p = sqa::attention_plan(dt, B, T, Hq, Hkv, D, uniform ? (int64_t)new_pos + T : layer->capacity);
  a.tiles = p.tiles; a.splits = p.splits;
  if ((int64_t)B * Hkv * p.tiles * p.splits > INT32_MAX - 8) return SQA_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? sqa::launch_attention<float, 64>(p.rw, a, st) : sqa::launch_attention<float, 128>(p.rw, a, st);
  return D == 64 ? sqa::launch_attention<sqa::bf16_t, 64>(p.rw, a, st) : sqa::launch_attention<sqa::bf16_t, 128>(p.rw, a, st);
}
