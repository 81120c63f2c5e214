// Causal attention of a chunk of tokens over a layer cache that holds it (sqa_chunk_attention).
//   out_t = sum_j exp(s_tj - m_t) V_j / l_t,  s_tj = q_t.K_j / sqrt(D),  l_t = sum_j exp(s_tj - m_t),  j <= position of t
// One pass over the slots with a running maximum m and sum l per row.  The g query heads of a KV head and the chunk's tokens
// are one list of rows, row r = token r / g, head r % g: K and V are read once for all of them.  A workgroup of 4
// waves takes 32 RW of these rows, RW = 4, 2 or 1: by their number, and fewer while that leaves workgroups short and each would have less
// than 512 slots (attention_plan).  With RW < 4 the 4 / RW waves of the same rows share
// out the slots of a tile and join at the end.  Few rows against many slots are shared out over workgroups too; their
// (m, l, sums) go through the workspace and the last one to arrive joins them, in order.
//   S^T = K.Q^T  a lane holds 16 of 32 slots of one row: maximum and sum need one exchange between the two lane halves, and
//                the probabilities are the next product's operand as they are
//   O^T = V^T.P^T  a row's sums lie in the two lanes of its column: rescaling is a multiplication by a lane's own number
// K and V tiles go from global memory straight to LDS, two buffers, in an order without bank conflicts (TileRows).
// Few rows are bound by how tiles of K and V arrive: two stages of 64 KB, one workgroup per CU, a barrier a tile.  16 x 1-5 tokens of 32 heads over 8, up
// to 4095 slots, bf16, 202 MB: 58 us with caches from HBM, as a model of many layers finds them (3.5 TB/s; a read reaches 6.3 to 7.1), 47 us where the
// last-level cache holds them (4.3 TB/s).  Many rows are bound by how far products and vector instructions of a SIMD's two waves overlap (8 x 2048
// tokens of 32 heads 350 us, 785 TFLOP/s, busy 0.39 and 0.46; 512 of 64 heads over 8 after 7680 141 us, 945, 0.46 and 0.43) and, where
// those run long enough, by power (2048 of 32 heads over 8 after 30000 930 to 1010 us from card to card, 1120 to 1030 TFLOP/s).
#include "sqa_chunk_mma.h"
#include <type_traits>

namespace sqa {

constexpr int kAtThreads = 256;
constexpr float kFarLogit = 64.f;                   // in powers of two: below it the rounding is 2e-6 at most
constexpr int kAtJoin = 512;                        // slots of a workgroup, see attention_plan()
constexpr int kAtItems = 512;                       // workgroups that few rows are shared out to: two per CU

struct AttentionArgs {
  ChunkArgs c;
  const void* q;
  void* out;
  float* lse;
  int32_t* count;                                   // [items]
  float4* part;                                     // [items]: [splits][32 RW][D / 4] rows of sums, [splits][32 RW] (m, l)
  float scale;                                      // log2(e) / sqrt(D)
  float near;                                       // 8 / scale: logits that close to a row's reference do not move it
  uint32_t group_m;                                 // 2^32 / g, for divisions by g
  int tiles, splits;
  int group;                                        // units whose rows are taken in turn (below)
};

// Two probabilities as two bf16 each, high + low = p to 2^-15 of it: few rows leave the matrix cores idle, so that V is multiplied by both and the
// caller's bf16 values meet probabilities as good as in fp32 (rms error of 16 x 1-5 tokens of 32 heads over 8 against 64 bits 1.66e-3, all of it
// the output's rounding; with p rounded to one bf16 2.10e-3; 46.3 -> 47.9 us; one token after 30000 29.3 either way, 512 tokens of 32 heads 14.9 -> 16.9, 4 x 64
// of 32 heads of 64 over 8 after 3000 25 -> 29).  The high part is cut off, the low part is what is left, but not below
// the smallest normal number or p itself: neither is 0 unless p is, since 0 x inf would spoil a sum that is infinite.
struct Halves { uint32_t high, low; };
__device__ __forceinline__ Halves halves(float x, float y) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  auto low = [](float p, uint32_t w) { return __builtin_amdgcn_fmed3f(p - __uint_as_float(w & 0xffff0000u), p, FLT_MIN); };
  return {__builtin_amdgcn_perm(b, a, 0x07060302u), pair(low(x, a), low(y, b))};
}

// the halves of a pair of bf16 that are not finite, as a mask
__device__ __forceinline__ uint32_t odd_mask(uint32_t v) {
  return ((v & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Does a tile of BYTES bytes in LDS hold a number that is not finite?  This thread's share of it; CLEAR: such numbers become 0.
template <typename T, int BYTES, int NT, bool CLEAR> __device__ __forceinline__ bool odd_values(char* tile) {
  bool odd = false;
#pragma unroll 1
  for (int i = threadIdx.x * 16; i < BYTES; i += NT * 16) {
    const uint4 w = *reinterpret_cast<const uint4*>(tile + i);
    uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t x = odd_mask(v[k]);
        odd |= x != 0;
        if constexpr (CLEAR) v[k] &= ~x;
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

// Adds the values of slots from .. from + n - 1 of a tile in LDS that are not finite to the sums of the rows that see them.
template <typename T, int D>
__device__ __forceinline__ void add_odd_values(const char* Vt, int from, int n, int tile_slot, int see, int half, f32x16_t (&o)[D / 32]) {
  using R = TileRows<T, D>;
  constexpr int NB = D / 32;
#pragma unroll 1
  for (int k = from; k < from + n; ++k) {
    const bool sees = tile_slot + k <= see;
    const char* const row = Vt + k * R::RB;
    if constexpr (sizeof(T) == 2) {
      const int swz = R::v_swizzle(k) << 4;
#pragma unroll
      for (int e = 0; e < NB; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const uint2 v = *reinterpret_cast<const uint2*>(row + ((64 * e + 4 * i) ^ swz) + 8 * half);
          o[e][i] += sees && odd_mask(v.x << 16) ? bf16_lo(v.x) : 0.f;
          o[e][i + 1] += sees && odd_mask(v.x & 0xffff0000u) ? bf16_hi(v.x) : 0.f;
          o[e][i + 2] += sees && odd_mask(v.y << 16) ? bf16_lo(v.y) : 0.f;
          o[e][i + 3] += sees && odd_mask(v.y & 0xffff0000u) ? bf16_hi(v.y) : 0.f;
        }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < NB; ++e) {
          const float v = reinterpret_cast<const float*>(row + 4 * NB * c_row(0, half))[NB * c_row(i, 0) + e];
          o[e][i] += sees && !isfinite(v) ? v : 0.f;
        }
    }
  }
}

// What a workgroup of NT threads works on: M rows of one unit and a run of its slots, in tiles of KT.
template <typename T, int D, int NT, int M, int KT> struct AttentionWork {
  using R = TileRows<T, D>;
  static constexpr int PP = D / 4;                  // 16-byte pieces of a row of sums
  static constexpr int REC = PP + 1;                // a row of sums and its (m, l)
  int64_t item;
  int u, b, h, g, n, row0, rows, last_row;          // n tokens, rows of the whole unit
  int split, parts, tile0, tile1, end;              // end: the slots that the rows see
  int64_t pos;
  ChunkUnit unit;
  bool held_slots;

  uint32_t group_m;                                 // (division by g: for rows below 2^31 the quotient is one too large at most, and place() puts it right)

  // Where the work is; false: there is none.  Nothing is known yet of what the unit holds, but its first `end` slots can be read where
  // held_slots is true.
  __device__ __forceinline__ bool locate(const AttentionArgs& a) {
    const uint32_t count = (uint32_t)(a.c.B * a.c.Hkv) * (uint32_t)(a.tiles * a.splits);
    const uint32_t per8 = (count + 7) / 8, work = (blockIdx.x & 7) * per8 + (blockIdx.x >> 3);     // (one run of items per XCD, see xcd_item)
    if (blockIdx.x >> 3 >= per8 || work >= count) return false;
    split = (int)(work % (uint32_t)a.splits);
    const uint32_t it = work / (uint32_t)a.splits;
    item = it;
    u = (int)(it / (uint32_t)a.tiles);
    int tile = (int)(it - (uint32_t)u * (uint32_t)a.tiles);
    if (a.group > 1) {                               // ... of `group` units, not of one
      const uint32_t of = (uint32_t)(a.group * a.tiles), first = it / of, rest = it - first * of;
      tile = (int)(rest / (uint32_t)a.group);
      u = (int)(first * (uint32_t)a.group + rest % (uint32_t)a.group);
    }
    tile = a.tiles - 1 - tile;                       // the longest first
    b = u / a.c.Hkv; h = u - b * a.c.Hkv; g = a.c.g;
    group_m = a.group_m;
    const ChunkSeq seq = chunk_seq(a.c, b, threadIdx.x == 0 && h == 0 && tile == 0 && split == 0);
    n = __builtin_amdgcn_readfirstlane(seq.n);
    rows = n * g;
    row0 = tile * M;
    if (row0 >= rows) return false;
    pos = seq.pos;
    unit = chunk_unit(a.c.L, u);
    last_row = min(row0 + M, rows) - 1;
    int t, head;
    place(last_row, t, head);
    held_slots = pos + n <= unit.slots;
    end = __builtin_amdgcn_readfirstlane(held_slots ? (int)pos + t + 1 : 1);          // (positions may be any up to 2^31: 1 for a unit that is refused)
    const int nt = (end + KT - 1) / KT, per = (nt + a.splits - 1) / a.splits;
    parts = (nt + per - 1) / per;
    tile0 = split * per;
    tile1 = min(tile0 + per, nt);
    return split < parts;
  }
  // Does the unit hold the chunk, and do its blocks (to s_table) lie in the pools?  Otherwise its rows become zeros.
  __device__ __forceinline__ bool check(const AttentionArgs& a, int* s_table) const {
    const int tid = threadIdx.x;
    int why = held_slots && chunk_held(a.c.L, unit, u, pos + n) ? 0 : SQA_ERR_STATE;
    if (held_slots && unit.table) {
      int outside = 0;
      for (int i = tid; i < (int)((pos + n + SQA_BLOCK_SLOTS - 1) / SQA_BLOCK_SLOTS); i += NT) {
        const int blk = unit.table[i];
        s_table[i] = blk;
        outside |= (unsigned)blk >= (unsigned)a.c.L.n_blocks;
      }
      if (__syncthreads_or(outside) && !why) why = SQA_ERR_SHAPE;
    }
    if (!why) return true;
    if (split) return false;
    if (tid == 0 && a.c.status) *a.c.status = why;
    for (int i = tid; i < (last_row + 1 - row0) * R::PPR; i += NT) {
      int t, head;
      place(row0 + i / R::PPR, t, head);
      st16(static_cast<T*>(a.out) + (((int64_t)b * a.c.T + t) * a.c.Hq + head) * D + i % R::PPR * R::E, make_uint4(0, 0, 0, 0));
      if (a.lse && i % R::PPR == 0) a.lse[((int64_t)b * a.c.Hq + head) * a.c.T + t] = -INFINITY;
    }
    return false;
  }
  __device__ __forceinline__ void place(int r, int& t, int& head) const {
    t = g > 1 ? (int)__umulhi((uint32_t)r, group_m) : r;
    int i = r - t * g;
    if (i < 0) { --t; i += g; }
    head = h * g + i;
  }

  // 32 bytes of a row of sums as the output's 8 (bf16) or 2 x 4 (fp32) elements
  __device__ __forceinline__ void store8(const AttentionArgs& a, int row, int p, const float4 (&v)[2], float mm, float ll) const {
    int t, head;
    place(row0 + row, t, head);
    const float inv = 1.f / ll;
    T* dst = static_cast<T*>(a.out) + (((int64_t)b * a.c.T + t) * a.c.Hq + head) * D + 8 * p;
    if constexpr (sizeof(T) == 2)
      st16(dst, make_uint4(pair(v[0].x * inv, v[0].y * inv), pair(v[0].z * inv, v[0].w * inv), pair(v[1].x * inv, v[1].y * inv), pair(v[1].z * inv, v[1].w * inv)));
    else
#pragma unroll
      for (int k = 0; k < 2; ++k) reinterpret_cast<float4*>(dst)[k] = make_float4(v[k].x * inv, v[k].y * inv, v[k].z * inv, v[k].w * inv);
    if (p == 0 && a.lse) a.lse[((int64_t)b * a.c.Hq + head) * a.c.T + t] = 0.6931471805599453f * fmaf(mm, a.scale, log2f(ll));
  }

  // The waves' sums (this one's: the rows 32 rw .. in o, their references m and sums l) joined over the KW waves of the same rows and
  // the workgroups of the same rows, and stored.  Each wave's go through LDS as 32 rows, 16-byte pieces exchanged by the row.
  template <int KW>
  __device__ __forceinline__ void finish(const AttentionArgs& a, char* s_stage, float (*s_m)[M], float (*s_l)[M], int* s_word, int rw, int kw,
                                         f32x16_t (&o)[D / 32], float m, float l) const {
    constexpr int NB = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    l = other_half_sum(l);
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
    const int live = (last_row + 1 - row0) * (PP / 2);
    if (parts == 1) {
      for (int i = tid; i < live; i += NT) {
        const int row = i / (PP / 2), p = i % (PP / 2);
        float mm, ll;
        joined(row, mm, ll);
        const float4 v[2] = {piece4(row, 2 * p), piece4(row, 2 * p + 1)};
        store8(a, row, p, v, mm, ll);
      }
      return;
    }
    const char* const base = uniform(reinterpret_cast<const char*>(a.part + item * a.splits * (M * REC)));
    const HandOver rec(reinterpret_cast<float4*>(const_cast<char*>(base)), (uint32_t)(a.splits * (M * REC * 16)));
    const uint32_t refs = (uint32_t)(a.splits * M * PP);                                     // all rows' sums, then all rows' (m, l)
    for (int i = tid; i < 2 * live; i += NT) rec.put((uint32_t)(split * M * PP + i), piece4(i / PP, i % PP));
    for (int row = tid; row <= last_row - row0; row += NT) {
      float mm, ll;
      joined(row, mm, ll);
      rec.put(refs + split * M + row, make_float4(mm, ll, 0.f, 0.f));
    }
    if (!last_to_arrive(a.count + item, parts, s_word)) return;
    // eight records' loads in flight: of one piece where every thread has one at most, otherwise of several.  (With four: 512 tokens of
    // 64 heads over 8 after 7680 150 us, now 145; one token after 30000 30.7, now 29.5.)
    if (live <= NT) join<1, 8>(a, rec, refs, live);
    else if (parts == 2) join<(M * PP / 2 < 4 * NT ? 2 : 4), 2>(a, rec, refs, live);
    else join<2, 4>(a, rec, refs, live);
  }

  // the records of all workgroups of these rows added up in order and stored: NI pieces of 32 bytes, K records of each in flight
  template <int NI, int K> __device__ __forceinline__ void join(const AttentionArgs& a, const HandOver& rec, uint32_t refs, int live) const {
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < live; i0 += NI * NT) {
      float mm[NI], ll[NI];
      float4 v[NI][2];
#pragma unroll
      for (int x = 0; x < NI; ++x) { mm[x] = -FLT_MAX; ll[x] = 0.f; v[x][0] = v[x][1] = make_float4(0.f, 0.f, 0.f, 0.f); }
#pragma unroll 1
      for (int k0 = 0; k0 < parts; k0 += K) {
        float4 ml[NI][K], lo[NI][K], hi[NI][K];
#pragma unroll
        for (int x = 0; x < NI; ++x)
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const int i = min(i0 + x * NT, live - 1), row = i / (PP / 2), p = i % (PP / 2);
            const uint32_t from = (uint32_t)(min(k0 + k, parts - 1) * M + row);
            ml[x][k] = rec.get(refs + from); lo[x][k] = rec.get(from * PP + 2 * p); hi[x][k] = rec.get(from * PP + 2 * p + 1);
          }
#pragma unroll
        for (int x = 0; x < NI; ++x)
#pragma unroll
          for (int k = 0; k < K; ++k)
            if (k0 + k < parts) {
              const float top = fmaxf(mm[x], ml[x][k].x), w0 = exp2_fast((mm[x] - top) * a.scale), w1 = exp2_fast((ml[x][k].x - top) * a.scale);
              mm[x] = top;
              ll[x] = fmaf(ll[x], w0, ml[x][k].y * w1);
              const float4 l4 = lo[x][k], h4 = hi[x][k];
              v[x][0] = make_float4(fmaf(v[x][0].x, w0, l4.x * w1), fmaf(v[x][0].y, w0, l4.y * w1), fmaf(v[x][0].z, w0, l4.z * w1), fmaf(v[x][0].w, w0, l4.w * w1));
              v[x][1] = make_float4(fmaf(v[x][1].x, w0, h4.x * w1), fmaf(v[x][1].y, w0, h4.y * w1), fmaf(v[x][1].z, w0, h4.z * w1), fmaf(v[x][1].w, w0, h4.w * w1));
            }
      }
#pragma unroll
      for (int x = 0; x < NI; ++x) {
        const int i = i0 + x * NT;
        if (i < live) store8(a, i / (PP / 2), i % (PP / 2), v[x], mm[x], ll[x]);
      }
    }
  }
};

template <typename T, int D, int RW, int KT> struct AttentionTile {
  using R = TileRows<T, D>;
  static constexpr int KW = 4 / RW, KB = KT / KW / 32, M = 32 * RW, NB = D / 32;
  static constexpr int TILE = KT * R::RB;
  static constexpr int STAGE = 4 * TILE > 4 * 32 * D * 4 ? 4 * TILE : 4 * 32 * D * 4;
};

// (Rows of 512 bytes and tiles of 64 slots fill a CU's LDS: one wave per SIMD, and registers for it.)
template <typename T, int D, int RW, int KT>
__global__ __launch_bounds__(kAtThreads, KT * D * sizeof(T) == 64 * 512 && RW == 2 ? 1 : 2) void chunk_attention_kernel(const AttentionArgs a) {
  using C = AttentionTile<T, D, RW, KT>;
  using R = TileRows<T, D>;
  constexpr int KW = C::KW, KB = C::KB, M = C::M, NB = C::NB;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // (16-byte reads of 8-byte places take 8 times as long)
  __shared__ float s_m[KW][M], s_l[KW][M];
  __shared__ int s_word;
  int* const s_table = reinterpret_cast<int*>(s_stage + C::STAGE);
  AttentionWork<T, D, kAtThreads, M, KT> w;
  if (!w.locate(a)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, col = lane & 31, half = lane >> 5;

  // ---- this lane's query row
  const int r = w.row0 + 32 * rw + col;
  const bool mine = r < w.rows;
  int t, head;
  w.place(min(r, w.last_row), t, head);
  const int see = (int)(w.pos + t);                                                    // the last slot that the row sees
  int t_first, t_tile, any;
  w.place(min(w.row0 + 32 * rw, w.last_row), t_first, any);
  w.place(w.row0, t_tile, any);
  const int see_all = (int)w.pos + t_first, see_all_tile = (int)w.pos + t_tile;          // ... that all of the wave's, of the workgroup's rows see
  Frag<T, D> q;
  {
    const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (((int64_t)w.b * a.c.Hq + head) * a.c.T + t) * D);
#pragma unroll
    for (int s = 0; s < q.NS; ++s) q.p[s] = mine ? ld16(src + (2 * s + half) * 16) : make_uint4(0, 0, 0, 0);
  }
  if (!w.check(a, s_table)) return;
  arrived(q);

  // ---- copies of one tile: each wave the rows wave KT/4 .. of K and of V
  const char* const Kp = static_cast<const char*>(a.c.L.K);
  const char* const Vp = static_cast<const char*>(a.c.L.V);
  auto fetch = [&](int tl, int buf) {
    const uint32_t dst = lds_at(s_stage) + (uint32_t)(buf * 2 * C::TILE);
#pragma unroll
    for (int i = 0; i < KT / 4 / R::RPI; ++i) {
      const int rr = wave * (KT / 4) + i * R::RPI, row = rr + lane / R::PPR;
      const int slot = min(tl * KT + row, w.end - 1);
      const int64_t at = w.unit.table ? (int64_t)s_table[slot / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : w.unit.first + slot;
      fetch16(Kp + at * R::RB + (((lane % R::PPR) ^ R::k_swizzle(row)) << 4), dst + rr * R::RB);
      fetch16(Vp + at * R::RB + (((lane % R::PPR) ^ R::v_swizzle(row)) << 4), dst + C::TILE + rr * R::RB);
    }
  };

  f32x16_t o[NB];
#pragma unroll
  for (int e = 0; e < NB; ++e) o[e] = f32x16_t{};
  float m = -FLT_MAX, l = 0.f;                       // (finite: a row that sees nothing yet has no exp(inf - inf))

  fetch(w.tile0, 0);
  for (int tl = w.tile0; tl < w.tile1; ++tl) {
    const int buf = (tl - w.tile0) & 1;
    fetched();
    __syncthreads();
    if (tl + 1 < w.tile1) fetch(tl + 1, buf ^ 1);
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
    // s scale - off in one operation is off by the rounding of `off`: far from 0 the difference is taken first.  (Each row for itself, so that
    // no row's bits depend on slots that only others see.)
    if (const bool far = fabsf(off) > kFarLogit; __any(far)) {
      const float from = far ? top : 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] -= from;
      off = far ? 0.f : off;
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
    if (tl * KT + KT - 1 > see_all_tile && __syncthreads_or(odd_values<T, C::TILE, kAtThreads, false>(s_stage + buf * 2 * C::TILE + C::TILE))) {
      add_odd_values<T, D>(Vt, key0, 32 * KB, tl * KT, see, half, o);
      __syncthreads();
      odd_values<T, C::TILE, kAtThreads, true>(s_stage + buf * 2 * C::TILE + C::TILE);
      __syncthreads();
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int row = key0 + 32 * kb;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          uint32_t p[2][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Halves x = halves(s[kb][8 * ks + 2 * i], s[kb][8 * ks + 2 * i + 1]);
            p[0][i] = x.high; p[1][i] = x.low;
          }
          const int vr = row + 16 * ks + 4 * half + (lane & 15) / 4;
#pragma unroll
          for (int e = 0; e < NB; ++e) {
            const int piece = (4 * e + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ R::v_swizzle(vr);
            const char* at = Vt + vr * R::RB + piece * 16 + (lane & 1) * 8;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 8 * R::RB));
            const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int x = 0; x < 2; ++x)
              o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8_t, make_uint4(p[x][0], p[x][1], p[x][2], p[x][3])), o[e], 0, 0, 0);
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
  w.template finish<KW>(a, s_stage, s_m, s_l, &s_word, rw, kw, o, m, l);
}

// The same for many rows in bf16: 128 rows and tiles of 64 slots, two workgroups per CU.  Probabilities are rounded to one bf16 for the product
// with V, which is what bounds long calls: with a low part too (as above) 8 x 2048 tokens of 32 heads take 450 us in place of 350, 512 of 64 heads over
// 8 after 7680 192 in place of 141, 2048 of 32 over 8 after 30000 1360 in place of 958; it would take the rms error against 64 bits from 2.1e-3 (2.35e-3
// after 7680) to the output's own rounding, 1.66e-3.  Nothing orders the two waves of a SIMD, which
// drift apart until one's products run beside the other's softmax.  V^T.P^T of a tile follows K.Q^T of the next one, K of tile j + 1
// and V of tile j are asked for when tile j begins; the reference m moves only when a logit is 2^8 times beyond it, so that the sums
// are seldom multiplied.  Tiles that not all rows see are worked off afterwards, one after the other.
constexpr int kWideSlots = 64;

// (Copies stay in flight; what was read from LDS has arrived, so that the buffers may be overwritten.)
__device__ __forceinline__ void part_done() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D> __global__ __launch_bounds__(kAtThreads, 2) void chunk_attention_wide_kernel(const AttentionArgs a) {
  constexpr int NW = kAtThreads / 64, kWideRows = 32 * NW;
  using T = bf16_t;
  using R = TileRows<T, D>;
  constexpr int NB = D / 32, NS = Frag<T, D>::NS, TILE = kWideSlots * R::RB;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // K, K', V, V'; at the end all rows' sums
  __shared__ float s_m[1][kWideRows], s_l[1][kWideRows];
  __shared__ int s_word;
  int* const s_table = reinterpret_cast<int*>(s_stage + kWideRows * D * 4);
  AttentionWork<T, D, kAtThreads, kWideRows, kWideSlots> w;
  if (!w.locate(a)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;

  // ---- this lane's query row
  const int r = w.row0 + 32 * wave + col;
  const bool mine = r < w.rows;
  int t, head;
  w.place(min(r, w.last_row), t, head);
  const int see = (int)(w.pos + t);                                                                                            // the last slot that the row sees
  int t_first, t_last, t_tile, any;
  w.place(min(w.row0 + 32 * wave, w.last_row), t_first, any);
  w.place(min(w.row0 + 32 * wave + 31, w.last_row), t_last, any);
  w.place(w.row0, t_tile, any);
  const int see_all = __builtin_amdgcn_readfirstlane((int)w.pos + t_first);              // ... that all of the wave's rows see
  const int see_any = __builtin_amdgcn_readfirstlane((int)w.pos + t_last);               // ... that any of them sees
  const int see_all_tile = __builtin_amdgcn_readfirstlane((int)w.pos + t_tile);          // ... that all of the workgroup's see
  Frag<T, D> q;
  {
    const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (((int64_t)w.b * a.c.Hq + head) * a.c.T + t) * D);
#pragma unroll
    for (int x = 0; x < NS; ++x) q.p[x] = mine ? ld16(src + (2 * x + half) * 16) : make_uint4(0, 0, 0, 0);
  }
  if (!w.check(a, s_table)) return;
  arrived(q);

  // ---- copies: each wave 64 / NW rows of K and of V of a tile (they lie in one block)
  constexpr int WR = kWideSlots / NW, NI = WR / R::RPI;
  const uint32_t lds0 = lds_at(s_stage) + wave * WR * R::RB;
  uint32_t k_from[NI], v_from[NI];                   // the lane's row and piece among the wave's
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r0 = i * R::RPI + lane / R::PPR, row = wave * WR + r0;
    k_from[i] = (uint32_t)(r0 * R::RB + (((lane % R::PPR) ^ R::k_swizzle(row)) << 4));
    v_from[i] = (uint32_t)(r0 * R::RB + (((lane % R::PPR) ^ R::v_swizzle(row)) << 4));
  }
  auto wave_slot = [&](int j) { return (w.tile0 + j) * kWideSlots + wave * WR; };
  auto block_of = [&](int j) { return w.unit.table ? s_table[min(wave_slot(j), w.end - 1) / SQA_BLOCK_SLOTS] : 0; };
  auto row_of = [&](int j, int block) {              // where the wave's first row lies
    return w.unit.table ? (int64_t)__builtin_amdgcn_readfirstlane(block) * SQA_BLOCK_SLOTS + wave_slot(j) % SQA_BLOCK_SLOTS : w.unit.first + wave_slot(j);
  };
  auto copy = [&](const void* from, int j, int64_t row, uint32_t dst, const uint32_t (&at)[NI]) {
    const int last = w.end - 1 - wave_slot(j);       // (rows behind the last: that one again)
    const char* const base = uniform(static_cast<const char*>(from) + row * R::RB);
    if (last >= WR - 1) {
#pragma unroll
      for (int i = 0; i < NI; ++i) fetch16(base, at[i], dst + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int r0 = i * R::RPI + lane / R::PPR, back = r0 - min(r0, last);
        if (last >= 0) fetch16(base + (int64_t)at[i] - back * R::RB, dst + i * 1024);
        else {                                       // (they lie elsewhere)
          const int slot = w.end - 1;
          const int64_t to = w.unit.table ? (int64_t)s_table[slot / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : w.unit.first + slot;
          fetch16(static_cast<const char*>(from) + to * R::RB + at[i] - r0 * R::RB, dst + i * 1024);
        }
      }
    }
  };

  // ---- the lane's places in a tile of K and of V
  int k_at[NS], v_at[NB];
#pragma unroll
  for (int x = 0; x < NS; ++x) k_at[x] = col * R::RB + (((2 * x + half) ^ R::k_swizzle(col)) << 4);
  {
    const int row = 4 * half + (lane & 15) / 4;
#pragma unroll
    for (int e = 0; e < NB; ++e)
      v_at[e] = row * R::RB + (((4 * e + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ R::v_swizzle(row)) << 4) + (lane & 1) * 8;
  }

  f32x16_t o[NB], s[2];
  bf16x8_t p[4];
#pragma unroll
  for (int e = 0; e < NB; ++e) o[e] = f32x16_t{};
  float m = -FLT_MAX, l = 0.f;                       // m: a reference that a row's largest logit is near, not always that logit

  auto keys = [&](int j) {                           // s = K.Q^T of tile j
    const char* const Kt = s_stage + (j & 1) * TILE;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      uint4 k[NS];
#pragma unroll
      for (int x = 0; x < NS; ++x) k[x] = *reinterpret_cast<const uint4*>(Kt + k_at[x] + 32 * kb * R::RB);
      s[kb] = f32x16_t{};
#pragma unroll
      for (int x = 0; x < NS; ++x) mma_piece<T>(k[x], q.p[x], s[kb]);
    }
  };
  auto values = [&](int j) {                         // o += V^T.P^T of tile j
    const char* const Vt = s_stage + (2 + (j & 1)) * TILE;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int e = 0; e < NB; ++e) {
        const char* at = Vt + v_at[e] + 16 * ks * R::RB;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 8 * R::RB));
        const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[ks], o[e], 0, 0, 0);
      }
  };
  // edge: not all rows of the workgroup see all slots of the tile
  auto softmax = [&](int j, auto edge) {
    if constexpr (decltype(edge)::value) {
      const int first = (w.tile0 + j) * kWideSlots;
      if (first + kWideSlots - 1 > see_all) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (first + 32 * kb + c_row(i, half) > see) s[kb][i] = -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    top = other_half_max(top);
    // the reference of a row moves when one of its logits is 2^8 times beyond it: seldom after the first tiles
    if (const bool beyond = top > m + a.near; __any(beyond)) {
      const float to = beyond ? top : m, keep = exp2_fast((m - to) * a.scale);
      m = to;
      l *= keep;
#pragma unroll
      for (int e = 0; e < NB; ++e) o[e] *= keep;
    }
    float off = m * a.scale;
    // (see the kernel above)
    if (const bool far = fabsf(off) > kFarLogit; __any(far)) {
      const float from = far ? m : 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] -= from;
      off = far ? 0.f : off;
    }
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float x = exp2_fast(fmaf(s[kb][i], a.scale, -off)), y = exp2_fast(fmaf(s[kb][i + 1], a.scale, -off));
        l0 += x; l1 += y;
        p[2 * kb + i / 8][i % 8] = (__bf16)x; p[2 * kb + i / 8][i % 8 + 1] = (__bf16)y;
      }
    l += l0 + l1;
  };
  // a slot that a row does not see has probability 0, but 0 x NaN is NaN (see the kernel above)
  auto take_odd_values = [&](int j) {
    char* const Vt = s_stage + (2 + (j & 1)) * TILE;
    if (!__syncthreads_or(odd_values<T, TILE, kAtThreads, false>(Vt))) return;
    add_odd_values<T, D>(Vt, 0, kWideSlots, (w.tile0 + j) * kWideSlots, see, half, o);
    __syncthreads();
    odd_values<T, TILE, kAtThreads, true>(Vt);
    __syncthreads();
  };

  const int n = w.tile1 - w.tile0;
  const int whole = min(max((see_all_tile + 1) / kWideSlots - w.tile0, 0), n);        // the first tiles, that every row sees all of
  int64_t row_k = row_of(0, block_of(0)), row_v = row_k;           // of the tile whose keys were asked for last, and of the one before
  int block = 0;                                                   // of the tile after that
  auto copy_k = [&](int j) {
    if (j >= n) return;
    row_v = row_k;
    row_k = row_of(j, block);
    copy(a.c.L.K, j, row_k, lds0 + (j & 1) * TILE, k_from);
    block = block_of(j + 1);
  };
  auto copy_v = [&](int j, int64_t row) { if (j < n) copy(a.c.L.V, j, row, lds0 + (2 + (j & 1)) * TILE, v_from); };
  copy(a.c.L.K, 0, row_k, lds0, k_from);
  block = block_of(1);
  fetched();
  part_done();
  // ---- the tiles that all rows see: K of tile j + 1 and V of tile j are asked for when tile j begins
  if (whole > 0) {
    for (int j = 0; j < whole; ++j) {
      copy_k(j + 1); copy_v(j, j + 1 < n ? row_v : row_k);
      __builtin_amdgcn_s_setprio(1);                 // the wave that has products to give goes first: 954 -> 929 us (30000 slots), 143 -> 140
      keys(j);
      if (j > 0) values(j - 1);
      __builtin_amdgcn_s_setprio(0);
      softmax(j, std::false_type{});
      fetched();
      part_done();
    }
    values(whole - 1);
    part_done();
  }
  // ---- the others, in step: K and V of tile j + 1 are asked for when tile j begins
  copy_v(whole, row_k);                              // (row_k: tile `whole`, the last that was asked for)
  for (int j = whole; j < n; ++j) {
    fetched();
    part_done();
    copy_k(j + 1);
    copy_v(j + 1, row_k);
    const bool seen = (w.tile0 + j) * kWideSlots <= see_any;
    if (seen) {
      keys(j);
      softmax(j, std::true_type{});
    }
    take_odd_values(j);
    if (seen) values(j);
  }
  w.template finish<1>(a, s_stage, s_m, s_l, &s_word, wave, 0, o, m, l);
}

struct AttentionPlan { int rw, tiles, splits, group; };          // rw: 32-row blocks of a workgroup
// (rows of 512 bytes have no form for 32 rows: its tiles would not fit the LDS)
static int attention_rw(int rows, bool bf16, int D) {
  return rows <= 32 && (bf16 || D == 64) ? 1 : (rows <= 64 ? 2 : 4);
}
// uniform: every sequence brings T tokens at new_pos; otherwise nothing is known on the host of what the units hold but their room
static AttentionPlan attention_plan(sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos, int32_t capacity, bool uniform) {
  AttentionPlan p;
  const bool ragged = !uniform;
  const int64_t slots = uniform ? (int64_t)new_pos + T : capacity;
  const int rows = T * (Hq / Hkv), least = attention_rw(1, dt == SQA_BF16, D);
  int64_t items, s;
  for (p.rw = attention_rw(rows, dt == SQA_BF16, D);; p.rw /= 2) {
    p.tiles = (rows + 32 * p.rw - 1) / (32 * p.rw);
    items = (int64_t)B * Hkv * p.tiles;
    // as many as run at a time (tiles of few rows fill half a CU's LDS or all of it); twice that where sequences differ in length: five
    // tokens of 16 sequences over 4095 slots 48 us (57 with twice as many), over 2048 to 4095 slots 51 (46 with twice as many)
    s = (p.rw == 4 || ragged ? kAtItems : kAtItems / 2) / items;
    // a join costs what some hundred slots do: short units are shared out by rows first.  With 256, 512 and 1024 slots in place of kAtJoin: 128 tokens
    // of 32 heads over 8 after 1000 20.3, 15.1, 15.1 us, 64 after 4000 25.1, 21.3, 21.3, 256 after 1500 26.4, 26.7, 27.4
    if (p.rw == least || s <= 1 || slots / s >= kAtJoin) break;
  }
  // The least slots of a workgroup, so that a join is worth its time (fp32 products take 8 times as long).  With twice as many 1 token of 32 heads
  // over 8 after 2000 takes 17.2 in place of 12.9 us, 5 of 8 heads of 128 after 1000 in fp32 34 in place of 21; with half as many 10.9 and 18.3.  From
  // 4000 slots on, or 16 sequences of 4000, it makes no difference (46 us).
  const int few = dt == SQA_BF16 ? 384 : 128;
  s = s > slots / few ? slots / few : s;
  p.splits = s < 1 ? 1 : (int)s;
  // Row tiles of a unit see from new_pos to new_pos + T slots.  Where that is not much the same for all, an XCD (an eighth of the units)
  // takes the longest of several units first, so that the launch ends in short ones.  (An eighth of the units has to be a whole number of such groups;
  // other numbers of units are taken one after the other.)
  p.group = 1;
  // (8 x 32 heads x 2048 tokens 383 -> 363 us, one sequence of them 66 -> 59; 16 or 32 units at a time 378, 396.)
  if (p.splits == 1 && p.tiles >= 8 && uniform && new_pos < T)
    for (int k = 8; k > 1; k /= 2)
      if ((int64_t)B * Hkv % (8 * k) == 0) { p.group = k; break; }
  return p;
}
// (any T' <= T, any length, either type: items x splits <= kAtItems where there are splits)
size_t chunk_attention_scratch(int T, int Hq, int Hkv, int D) {
  const int rw = attention_rw(T * (Hq / Hkv), false, D);
  return (size_t)kAtItems * 32 * rw * (D / 4 + 1) * sizeof(float4);
}

static sqa_status start_attention(void (*fn)(AttentionArgs), int threads, size_t lds, const AttentionArgs& a, hipStream_t st) {
  if (a.c.L.block_table) lds += (size_t)(a.c.L.blocks_per_unit + 3) / 4 * 16;
  SQA_HIP_CHECK(allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds));
  const int64_t work = (int64_t)a.c.B * a.c.Hkv * a.tiles * a.splits;
  fn<<<(unsigned)xcd_grid(work), threads, lds, st>>>(a);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}
template <typename T, int D, int RW, int KT>
static sqa_status launch_attention(const AttentionArgs& a, hipStream_t st) {
  return start_attention(chunk_attention_kernel<T, D, RW, KT>, kAtThreads, AttentionTile<T, D, RW, KT>::STAGE, a, st);
}
template <typename T, int D>
static sqa_status launch_attention(int rw, const AttentionArgs& a, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (rw == 4) return start_attention(chunk_attention_wide_kernel<D>, kAtThreads, 128 * D * 4, a, st);
  }
  constexpr bool wide = D * sizeof(T) == 512;        // rows of 512 bytes: half the slots
  if constexpr (sizeof(T) == 4)
    if (rw == 4) return launch_attention<T, D, 4, wide ? 32 : 64>(a, st);
  if constexpr (wide) return launch_attention<T, D, 2, 64>(a, st);
  else return rw == 2 ? launch_attention<T, D, 2, 64>(a, st) : launch_attention<T, D, 1, 128>(a, st);
}

}  // namespace sqa

extern "C" size_t sqa_chunk_workspace_bytes(const sqa_layer_cache* layer, int B, int T, int Hq, int Hkv, int D) {
  sqa_status why;
  if (!layer || sqa::bad_layer(*layer, &why) || sqa::bad_chunk_shape(B, T, Hq, Hkv, D, 0, nullptr)) return 0;
  const size_t x = sqa::chunk_attention_scratch(T, Hq, Hkv, D);
  const size_t y = sqa::chunk_scores_scratch();
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
  const size_t need = sqa_chunk_workspace_bytes(layer, B, T, Hq, Hkv, D);
  if (ws_bytes < need) return SQA_ERR_CAPACITY;
  if (!(opts && (opts->prompt_len || opts->new_pos_seq)) && (int64_t)new_pos + T > layer->capacity) return SQA_ERR_CAPACITY;
  const size_t es = dt == SQA_F32 ? 4 : 2, qb = (size_t)B * Hq * T * D * es, lb = (size_t)B * Hq * T * sizeof(float);
  if (sqa::overlap(q, qb, out, qb) || (lse && (sqa::overlap(lse, lb, q, qb) || sqa::overlap(lse, lb, out, qb)))) return SQA_ERR_SHAPE;
  // (workgroups that still read these would see what others have stored)
  if (sqa::overlap(workspace, need, q, qb) || sqa::overlap(workspace, need, out, qb) || (lse && sqa::overlap(workspace, need, lse, lb)) ||
      sqa::in_layer(*layer, B, Hkv, D, es, out, qb) || sqa::in_layer(*layer, B, Hkv, D, es, lse, lb) || sqa::in_layer(*layer, B, Hkv, D, es, workspace, need))
    return SQA_ERR_SHAPE;
  sqa::AttentionArgs a{};
  a.c = sqa::chunk_args(layer, B, T, Hq, Hkv, new_pos, opts);
  a.q = q; a.out = out; a.lse = lse;
  a.count = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float4*>(static_cast<char*>(workspace) + sqa::kChunkCounterBytes);
  a.scale = (float)(1.4426950408889634 / sqrt((double)D));
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  const sqa::AttentionPlan p = sqa::attention_plan(dt, B, T, Hq, Hkv, D, new_pos, layer->capacity, uniform);
  a.near = 8.f / a.scale;
  a.group_m = 0xffffffffu / (uint32_t)a.c.g + 1;
  a.tiles = p.tiles; a.splits = p.splits; a.group = p.group;
  if ((int64_t)B * Hkv * p.tiles * p.splits > INT32_MAX - 8) return SQA_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? sqa::launch_attention<float, 64>(p.rw, a, st) : sqa::launch_attention<float, 128>(p.rw, a, st);
  return D == 64 ? sqa::launch_attention<sqa::bf16_t, 64>(p.rw, a, st) : sqa::launch_attention<sqa::bf16_t, 128>(p.rw, a, st);
}

extern "C" sqa_status sqa_chunk_plan(const sqa_layer_cache* layer, sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos,
                                     const sqa_batch_opts* opts, sqa_chunk_plan_info* info) {
  if (!layer || !info) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (sqa::bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  if (layer->capacity < 1 || (uniform && (int64_t)new_pos + T > layer->capacity)) return SQA_ERR_CAPACITY;
  const sqa::AttentionPlan p = sqa::attention_plan(dt, B, T, Hq, Hkv, D, new_pos, layer->capacity, uniform);
  info->rows = 32 * p.rw; info->row_tiles = p.tiles; info->slot_splits = p.splits; info->units_in_turn = p.group;
  info->rounded_probs = dt == SQA_BF16 && p.rw == 4;
  const sqa::ScoresPlan q = sqa::scores_plan(dt, B, T, Hq, Hkv, D, new_pos, layer->capacity, uniform);
  info->score_slots = q.slots; info->score_slot_tiles = q.tiles; info->score_row_splits = q.splits;
  return SQA_OK;
}
