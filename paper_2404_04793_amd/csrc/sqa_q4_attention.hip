// Causal attention of a chunk of tokens over a cache in 4 bits (sqa_q4_attention).
//   out_t = sum_j exp(s_tj - m_t) V_j / l_t,  s_tj = q_t.K_j / sqrt(D),  l_t = sum_j exp(s_tj - m_t),  over the slots j that token t sees
// One pass over the slots with a running reference m and sum l per row; the g query heads of a KV head and the chunk's tokens are one list
// of rows, row r = token r / g, head r % g.
//   S^T = K.Q^T  K becomes bf16 in registers (exactly, one conversion for two numbers), as the row's pieces lie: a lane's 32 numbers
//                are the operand of four products.  Q is bf16 as it comes, fp32 the sum of three parts of bf16.  (The matrix cores take
//                codes and powers as they are, v_mfma_scale_f32_16x16x128_f8f6f4, but keep no more than about 13 bits below the largest of a
//                product's 128 terms: logits off by 1e-5 to 1e-4.)
//   O^T = V^T.P^T  V becomes bf16 on its way through LDS, where the transposing reads make it the operand; P is the sum of 2 (bf16) or
//                3 (fp32) parts of bf16
// Each wave takes tiles of 32 slots for itself: no barrier before the end, where the waves' sums are joined, and those of several
// workgroups that share out a unit's slots through the workspace, by the last one to arrive, in order.
#include "sqa_chunk_mma.h"
#include "sqa_q4.h"
#include <algorithm>

namespace sqa {

constexpr int kQ4Slots = 32;                        // slots of a tile
constexpr float kQ4FarLogit = 64.f;                 // in powers of two: below it the rounding is 2e-6 at most
typedef __attribute__((address_space(1))) const uint8_t g_u8_t;
typedef __attribute__((address_space(3))) v4u_t lds_v4u_t;

constexpr int kQ4Splits = 64;                       // workgroups that share out a unit's slots: a lane each when they are joined
constexpr int kQ4WideRows = 65;                     // rows of a unit from which on a workgroup may take 128 of them (bf16)

struct Q4AttentionArgs {
  Q4Args a;
  const void* q;
  void* out;
  float* lse;
  int32_t* count;                                   // [items]
  float4* part;                                     // [items][splits][rows][D / 4 + 1]: sums, then (m, l, bad)
  float scale;                                      // log2(e) / sqrt(D)
  float near;                                       // 8 / scale: logits that close to a row's reference do not move it
  uint32_t group_m, heads_m, tiles_m, splits_m;     // 2^32 / g, / Hkv, / tiles, / splits: for divisions by them (tiles_m: / B Hkv where tile_major)
  int tiles, splits;
  int tile_major;                                   // all units' longest row tiles first, in place of one run of units per XCD
};

// q = x / d and what is left, for 0 <= x < 2^31 and m = 2^32 / d rounded up: the high product is one too large at most
__device__ __forceinline__ void divide(int x, int d, uint32_t m, int& q, int& r) {
  q = d > 1 ? (int)__umulhi((uint32_t)x, m) : x;
  r = x - q * d;
  if (r < 0) { --q; r += d; }
}
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }           // (the same in all lanes)
__device__ __forceinline__ float lanes16_max(float v) { v = fmaxf(v, __shfl_xor(v, 16, SQA_WAVE)); return fmaxf(v, __shfl_xor(v, 32, SQA_WAVE)); }
__device__ __forceinline__ float lanes16_sum(float v) { v += __shfl_xor(v, 16, SQA_WAVE); return v + __shfl_xor(v, 32, SQA_WAVE); }

// 8 codes and their group's power as bf16
__device__ __forceinline__ uint4 q4_open(uint32_t w, float power) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 3)));
}

// Two numbers as NV pairs of bf16, the first ones cut off, the last one rounded: their sum is the number to 8 NV bits.
template <int NV> __device__ __forceinline__ void split16(float x, float y, uint32_t (&w)[NV]) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (k == NV - 1) { w[k] = pair(x, y); break; }
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    w[k] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    x -= __uint_as_float(a & 0xffff0000u); y -= __uint_as_float(b & 0xffff0000u);
  }
}

template <typename T, int D> struct Q4Tile {
  static constexpr int NP = sizeof(T) == 2 ? 1 : 3, NV = sizeof(T) == 2 ? 2 : 3;
  static constexpr int RB = D / 2;                  // bytes of a row of codes
  static constexpr int NL = D / 64;                 // 16-byte loads of a lane for 32 rows of V
  static constexpr int KD = D / 32;                 // dwords of a row of K in a lane: 8 KD numbers
  static constexpr int NE = D / 16;                 // blocks of 16 elements
  static constexpr int GPR = D / kGroup;            // groups of a row
  static constexpr int VB = kQ4Slots * D * 2;       // a wave's tile of V in LDS
  // piece p (16 bytes) of row r of V in bf16 lies at place p ^ swizzle(r): the transposing reads (32 bytes of each of 16 rows) meet all banks; of the
  // writes 8 lanes (2 or 4 rows) take two turns.  (A lane per row writes without conflicts, 35 % fewer LDS cycles, but asks for V in another order: 16 x
  // 16 tokens after 4000 40.0 -> 39.3 us, 64 x 32 units of 571 slots 30.5 -> 30.9.)
  static __device__ __forceinline__ int swizzle(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
};

// threadIdx.x anew: what is derived from it takes no registers from here back to its first use
__device__ __forceinline__ int late_tid() {
  int x = threadIdx.x;
  asm volatile("" : "+v"(x));
  return x;
}

// A barrier, and whether x is true in any thread (__syncthreads_or keeps the packed thread numbers in a register until its last use)
template <int NT> __device__ __forceinline__ bool any_thread(bool x, int* s_flags /*[NT / 64]*/) {
  s_flags[threadIdx.x >> 6] = __any(x);
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int k = 0; k < NT / 64; ++k) all |= s_flags[k];
  return scalar(all) != 0;
}

// What a workgroup of NT threads works on: M rows of one unit and a run of its slots, in tiles of KT.
template <typename T, int D, int NT, int M, int KT> struct Q4Work {
  static constexpr int PP = D / 4, REC = PP + 1;    // 16-byte pieces of a row of sums; and its (m, l, bad)
  Q4Seq s;
  int item, split, u, b, h, g, row0, last_row, parts, tile0, tile1;
  int len, end, whole;                              // slots that hold tokens, that the workgroup's rows see, that all of its rows see lie before them
  int newest, fixed, ring, back_most;               // back_most: tokens of the chunk behind the first row's
  int gap0, gap;                                    // tiles gap0 .. gap0 + gap - 1 no row of the workgroup sees: left out of the count
  bool turned;
  uint32_t group_m;

  // false: there is nothing to do.  (All of it the same in all lanes.)
  __device__ __forceinline__ bool locate(const Q4AttentionArgs& a) {
    const uint32_t total = (uint32_t)(a.a.c.B * a.a.c.Hkv) * (uint32_t)(a.tiles * a.splits);
    const uint32_t per8 = (total + 7) / 8, work = a.tile_major ? blockIdx.x : (blockIdx.x & 7) * per8 + (blockIdx.x >> 3);    // (one run of items per XCD, see xcd_item)
    if (blockIdx.x >> 3 >= per8 || work >= total) return false;
    int tile;
    divide((int)work, a.splits, a.splits_m, item, split);
    if (a.tile_major) divide(item, a.a.c.B * a.a.c.Hkv, a.tiles_m, tile, u);
    else divide(item, a.tiles, a.tiles_m, u, tile);
    tile = a.tiles - 1 - tile;                      // (the longest first)
    divide(u, a.a.c.Hkv, a.heads_m, b, h);
    g = a.a.c.g; group_m = a.group_m;
    s = q4_seq(a.a, b, threadIdx.x == 0 && h == 0 && tile == 0 && split == 0);
    s.n = scalar(s.n); s.slots = scalar(s.slots); s.why = scalar(s.why);
    s.pos = (int64_t)scalar((int)s.pos);            // (positions are 32-bit numbers)
    const int rows = s.n * g;
    row0 = tile * M;
    if (row0 >= rows) return false;
    last_row = min(row0 + M, rows) - 1;
    int t_first, t_last, any;
    place(row0, t_first, any);
    place(last_row, t_last, any);
    t_first = scalar(t_first); t_last = scalar(t_last);
    turned = s.end() > s.slots;
    len = s.why ? 1 : s.len();
    end = turned ? len : min((int)s.pos + t_last + 1, len);
    whole = min((int)s.pos + t_first + 1, len);
    back_most = scalar(s.n - 1 - t_first);
    newest = s.why ? 0 : scalar(s.slot(s.end() - 1));
    fixed = turned ? s.sink : 0; ring = turned ? s.slots - s.sink : 0;
    int nt = (int)((uint32_t)(end + KT - 1) / KT);
    gap0 = gap = 0;
    if (turned && !s.why) {
      // the tokens behind the last row's, `hidden` of them: slots up to the newest, and where these begin at the ring's start its end too.  One run of
      // whole tiles among them, the longer one.
      const int hidden = scalar(s.n - 1 - t_last), low = min(hidden, newest + 1 - fixed), high = hidden - low;
      auto leave = [&](int from, int to) {
        const int x = (from + KT - 1) / KT, y = to == len ? nt : to / KT;
        if (y - x > gap) { gap0 = x; gap = y - x; }
      };
      leave(newest + 1 - low, newest + 1);
      if (high > 0) leave(len - high, len);
      nt -= gap;
    }
    gap0 = scalar(gap0); gap = scalar(gap);
    int per = nt, rest;
    parts = 1;
    if (a.splits > 1) {
      divide(nt + a.splits - 1, a.splits, a.splits_m, per, rest);
      per = scalar(per);
      parts = scalar((int)((uint32_t)(nt + per - 1) / (uint32_t)per));
    }
    tile0 = scalar(split * per); tile1 = scalar(min(tile0 + per, nt));
    len = scalar(len); end = scalar(end); whole = scalar(whole); fixed = scalar(fixed); ring = scalar(ring);
    if (split >= parts) return false;
    if (s.why) {
      if (split == 0) refuse(a, s.why);
      return false;
    }
    return true;
  }
  // the i-th tile of those that some row sees
  __device__ __forceinline__ int tile_of(int i) const { return i + (i >= gap0 ? gap : 0); }
  __device__ __forceinline__ void place(int r, int& t, int& head) const {
    int x;
    divide(r, g, group_m, t, x);
    head = h * g + x;
  }
  // Does a row whose token is `back` tokens before the newest see a slot?  The newest lies at `newest`, the others of the ring before it.
  // (Without branches.  `if (!(a && (b || c))) s[0] = -INFINITY` for the first register of a product's result was compiled to -inf where !a and to an
  // empty region for the lanes where only b || c is false: these kept their logit.  tests/test_no_empty_branches.py finds such regions; no kernel has one.)
  __device__ __forceinline__ bool sees(int slot, int back) const {
    int behind = newest - slot;
    behind += behind < 0 ? ring : 0;
    return (bool)((int)(slot < len) & ((int)(slot < fixed) | (int)(behind >= back)));
  }
  // Does some row not see some slot of tile tl?  (The same in all lanes.)  In a ring that has turned: by how far its newest slot lies behind the newest.
  __device__ __forceinline__ bool is_edge(int tl) const {
    const int from = tl * KT, to = from + KT;
    if (!turned) return to > whole;
    const int hi = min(to, len) - 1, lo = max(from, fixed);
    int behind = newest - hi;
    behind += behind < 0 ? ring : 0;
    behind = (int)(lo <= newest) & (int)(newest <= hi) ? 0 : behind;
    return (bool)((int)(to > len) | ((int)(lo <= hi) & (int)(behind < back_most)));
  }
  // block numbers of this workgroup's slots to LDS; does one of them lie outside the pools?
  __device__ __forceinline__ bool stage_blocks(const sqa_q4_cache& L, int* s_table, int* s_flags) const {
    if (!L.block_table) return false;
    constexpr int BPT = KT / SQA_BLOCK_SLOTS;
    const int32_t* table = L.block_table + (int64_t)u * L.blocks_per_unit;
    bool bad = false;
    for (int x = threadIdx.x; x < BPT * (tile1 - tile0); x += NT) {
      const int e = BPT * tile_of(tile0 + x / BPT) + x % BPT;
      int blk = e * SQA_BLOCK_SLOTS < end ? table[e] : 0;
      if ((unsigned)blk >= (unsigned)L.n_blocks) { bad = true; blk = 0; }
      s_table[x] = blk;
    }
    return any_thread<NT>(bad, s_flags);
  }
  __device__ __forceinline__ void refuse(const Q4AttentionArgs& a, int why) const {
    const int tid = threadIdx.x;
    if (tid == 0 && a.a.c.status) *a.a.c.status = why;
    constexpr int E = 16 / (int)sizeof(T), PPR = D / E;
    for (int x = tid; x < (last_row + 1 - row0) * PPR; x += NT) {
      int t, head;
      place(row0 + x / PPR, t, head);
      st16(static_cast<T*>(a.out) + (((int64_t)b * a.a.c.T + t) * a.a.c.Hq + head) * D + x % PPR * E, make_uint4(0, 0, 0, 0));
      if (a.lse && x % PPR == 0) a.lse[((int64_t)b * a.a.c.Hq + head) * a.a.c.T + t] = -INFINITY;
    }
  }
  // pieces 2 p and 2 p + 1 of a row of sums
  __device__ __forceinline__ void store8(const Q4AttentionArgs& a, int row, int p, const float4 (&v)[2], float mm, float ll) const {
    int t, head;
    place(row0 + row, t, head);
    const float inv = 1.f / ll;
    T* dst = static_cast<T*>(a.out) + (((int64_t)b * a.a.c.T + t) * a.a.c.Hq + head) * D + 8 * p;
    if constexpr (sizeof(T) == 2)
      st16(dst, make_uint4(pair(v[0].x * inv, v[0].y * inv), pair(v[0].z * inv, v[0].w * inv), pair(v[1].x * inv, v[1].y * inv), pair(v[1].z * inv, v[1].w * inv)));
    else
#pragma unroll
      for (int k = 0; k < 2; ++k) reinterpret_cast<float4*>(dst)[k] = make_float4(v[k].x * inv, v[k].y * inv, v[k].z * inv, v[k].w * inv);
    if (p == 0 && a.lse) a.lse[((int64_t)b * a.a.c.Hq + head) * a.a.c.T + t] = 0.6931471805599453f * fmaf(mm, a.scale, log2f(ll));
  }

  // The sums of KW waves for each row (in s_stage, [KW][M] rows of pieces, piece p of row r at place p ^ (r & 15); references and sums in s_m and
  // s_l) joined, those of the workgroups of the same rows too, and stored.
  template <int KW>
  __device__ __forceinline__ void finish(const Q4AttentionArgs& a, char* s_stage, float (*s_m)[M], float (*s_l)[M], int* s_word, int* s_flags, bool bad) const {
    const int tid = late_tid(), lane = tid & 63, wave = tid >> 6;
    auto joined = [&](int row, float& mm, float& ll) {
      mm = s_m[0][row];
#pragma unroll 2
      for (int w = 1; w < KW; ++w) mm = fmaxf(mm, s_m[w][row]);
      ll = 0.f;
#pragma unroll 2
      for (int w = 0; w < KW; ++w) ll += s_l[w][row] * exp2_fast((s_m[w][row] - mm) * a.scale);
    };
    auto piece4 = [&](int row, int p) {
      float4 v = reinterpret_cast<const float4*>(s_stage)[row * PP + (p ^ (row & 15))];
#pragma unroll 2
      for (int w = 1; w < KW; ++w) {
        const float4 x = reinterpret_cast<const float4*>(s_stage)[(w * M + row) * PP + (p ^ (row & 15))];
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
      return v;
    };
    const int live = (last_row + 1 - row0) * (PP / 2);
    if (parts == 1) {
      if (bad) { refuse(a, SQA_ERR_SHAPE); return; }
      for (int x = tid; x < live; x += NT) {
        const int row = x / (PP / 2), p = x % (PP / 2);
        float mm, ll;
        joined(row, mm, ll);
        const float4 v[2] = {piece4(row, 2 * p), piece4(row, 2 * p + 1)};
        store8(a, row, p, v, mm, ll);
      }
      return;
    }
    const char* const base = uniform(reinterpret_cast<const char*>(a.part + (int64_t)item * a.splits * (M * REC)));
    const HandOver rec(reinterpret_cast<float4*>(const_cast<char*>(base)), (uint32_t)(a.splits * (M * REC * 16)));
    const uint32_t refs = (uint32_t)(a.splits * M * PP);                                   // all rows' sums, then all rows' (m, l, bad)
    for (int x = tid; x < 2 * live; x += NT) rec.put((uint32_t)(split * M * PP + x), piece4(x / PP, x % PP));
    for (int row = tid; row <= last_row - row0; row += NT) {
      float mm, ll;
      joined(row, mm, ll);
      rec.put(refs + split * M + row, make_float4(mm, ll, bad ? 1.f : 0.f, 0.f));
    }
    if (!last_to_arrive(a.count + item, parts, s_word)) return;
    // ---- all workgroups' sums.  Few records: a thread asks for all that it needs at once.
    if (parts <= 4) {
      bad = false;
      for (int x = tid; x < live; x += NT) {
        const int row = x / (PP / 2), p = x % (PP / 2);
        float4 ml[4], w4[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t from = (uint32_t)(min(k, parts - 1) * M + row);
          ml[k] = rec.get(refs + from); w4[k][0] = rec.get(from * PP + 2 * p); w4[k][1] = rec.get(from * PP + 2 * p + 1);
        }
        float mm = ml[0].x, ll = 0.f;
#pragma unroll
        for (int k = 1; k < 4; ++k) mm = fmaxf(mm, ml[k].x);
        float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k >= parts) break;
          const float w = exp2_fast((ml[k].x - mm) * a.scale);
          ll = fmaf(w, ml[k].y, ll);
          bad |= ml[k].z != 0.f;
#pragma unroll
          for (int y = 0; y < 2; ++y)
            v[y] = make_float4(fmaf(w4[k][y].x, w, v[y].x), fmaf(w4[k][y].y, w, v[y].y), fmaf(w4[k][y].z, w, v[y].z), fmaf(w4[k][y].w, w, v[y].w));
        }
        if (bad) break;
        store8(a, row, p, v, mm, ll);
      }
      if (any_thread<NT>(bad, s_flags)) refuse(a, SQA_ERR_SHAPE);
      return;
    }
    // Many: each one's weight per row first, then the weighted pieces, the records shared out among groups of threads.
    float* const s_weight = reinterpret_cast<float*>(s_stage);                             // [parts][M], then the groups' sums
    const int live_rows = last_row + 1 - row0;
    bad = false;
    for (int row = wave; row < live_rows; row += NT / 64) {                                     // a lane per record (there are 64 at most)
      const float4 ml = rec.get(refs + (uint32_t)(min(lane, parts - 1) * M + row));
      const bool there = lane < parts;
      bad |= there && ml.z != 0.f;
      float mm = there ? ml.x : -FLT_MAX;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o, SQA_WAVE));
      const float w = exp2_fast((ml.x - mm) * a.scale);
      const float ll = wave_sum(there ? w * ml.y : 0.f);
      if (there) s_weight[lane * M + row] = w;
      if (lane == 0) { s_m[0][row] = mm; s_l[0][row] = ll; }
    }
    if (any_thread<NT>(bad, s_flags)) { refuse(a, SQA_ERR_SHAPE); return; }
    int groups = 1;
    while (groups * 2 * live <= NT && groups < parts) groups *= 2;
    float4* const s_sum = reinterpret_cast<float4*>(s_stage + kQ4Splits * M * 4);
    const int per_group = groups * live;
    for (int x0 = 0; x0 < live; x0 += NT) {            // (once, but for more pieces than threads: one group then)
      const int x = x0 + tid % (groups > 1 ? live : NT), grp = groups > 1 ? tid / live : 0;
      if (x >= live || (groups > 1 && tid >= per_group)) { if (groups == 1) continue; else break; }
      const int row = x / (PP / 2), p = x % (PP / 2);
      float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
      for (int k0 = grp; k0 < parts; k0 += 8 * groups) {
        float4 w4[8][2];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t from = (uint32_t)(min(k0 + k * groups, parts - 1) * M + row) * PP + 2 * p;
          w4[k][0] = rec.get(from); w4[k][1] = rec.get(from + 1);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k0 + k * groups < parts) {
            const float w = s_weight[(k0 + k * groups) * M + row];
#pragma unroll
            for (int y = 0; y < 2; ++y)
              v[y] = make_float4(fmaf(w4[k][y].x, w, v[y].x), fmaf(w4[k][y].y, w, v[y].y), fmaf(w4[k][y].z, w, v[y].z), fmaf(w4[k][y].w, w, v[y].w));
          }
      }
      if (groups == 1) store8(a, row, p, v, s_m[0][row], s_l[0][row]);
      else { s_sum[2 * (grp * live + x)] = v[0]; s_sum[2 * (grp * live + x) + 1] = v[1]; }
    }
    if (groups == 1) return;
    __syncthreads();
    if (tid < live) {
      const int row = tid / (PP / 2), p = tid % (PP / 2);
      float4 v[2] = {s_sum[2 * tid], s_sum[2 * tid + 1]};
      for (int k = 1; k < groups; ++k)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float4 x = s_sum[2 * (k * live + tid) + y];
          v[y].x += x.x; v[y].y += x.y; v[y].z += x.z; v[y].w += x.w;
        }
      store8(a, row, p, v, s_m[0][row], s_l[0][row]);
    }
  }
};

template <typename T, int D, int NW, int R>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 && R == 1 ? 4 : 2) void q4_attention_kernel(const Q4AttentionArgs a) {
  using C = Q4Tile<T, D>;
  constexpr int M = 16 * R, NE = C::NE, NL = C::NL, NP = C::NP, NV = C::NV, KD = C::KD, PP = D / 4, NT = 64 * NW;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // V tiles of the waves, at the end their sums; then the table
  __shared__ float s_m[NW][M], s_l[NW][M];
  __shared__ int s_word, s_flags[NW];
  int* const s_table = reinterpret_cast<int*>(s_stage + R * NW * C::VB);
  const sqa_q4_cache& L = a.a.L;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, j = lane >> 4;

  Q4Work<T, D, NT, M, kQ4Slots> w;
  if (!w.locate(a)) return;
  const int tile0 = w.tile0, tile1 = w.tile1, end = w.end;
  // ---- this lane's query rows: i of each 16
  int back[R];                                      // tokens of the chunk behind its token
  // its elements 8 KD j .. of step x: 8 (KD j + x) ..
  uint4 qp[R][NP][KD];
#pragma unroll
  for (int n = 0; n < R; ++n) {
    int t, head;
    w.place(min(w.row0 + 16 * n + i, w.last_row), t, head);
    back[n] = w.s.n - 1 - t;
    const T* src = static_cast<const T*>(a.q) + (((int64_t)w.b * a.a.c.Hq + head) * a.a.c.T + t) * D + 8 * KD * j;
#pragma unroll
    for (int x = 0; x < KD; ++x) {
      if constexpr (sizeof(T) == 2) qp[n][0][x] = ld16(src + 8 * x);
      else {
        const uint4 lo = ld16(src + 8 * x), hi = ld16(src + 8 * x + 4);
        const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        uint32_t w[4][NP];
#pragma unroll
        for (int y = 0; y < 4; ++y) split16<NP>(__uint_as_float(v[2 * y]), __uint_as_float(v[2 * y + 1]), w[y]);
#pragma unroll
        for (int p = 0; p < NP; ++p) qp[n][p][x] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
      }
    }
  }

  const bool bad = w.stage_blocks(L, s_table, s_flags);
  // ---- rows of 16 neighbouring slots lie one after the other; slots behind the last one are read as that one again
  const int64_t unit_row = (int64_t)w.u * L.capacity;
  auto row_of = [&](int tl, int slot, int k) {      // (the same in all lanes)
    return L.block_table ? (int64_t)__builtin_amdgcn_readfirstlane(s_table[2 * (tl - tile0) + k]) * SQA_BLOCK_SLOTS : unit_row + slot + 16 * k;
  };
  struct At { int64_t row[2]; int last[2]; };       // of a tile's halves: the first row, and the last that there is behind it
  auto locate = [&](int tl) {
    const int slot = w.tile_of(tl) * kQ4Slots;
    At x;
    x.row[0] = row_of(tl, slot, 0); x.last[0] = min(end - 1 - slot, 15);
    const bool two = end - slot > 16;               // (a half without a slot: the first half again)
    x.row[1] = two ? row_of(tl, slot, 1) : x.row[0]; x.last[1] = two ? min(end - 17 - slot, 15) : x.last[0];
    return x;
  };
  struct Codes { uint32_t k[2][KD], kp[2], vp[NL]; uint4 v[NL]; } now;
  auto fetch_keys = [&](const At& x, Codes& to) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint32_t r = (uint32_t)min(i, x.last[kb]);
      const char* at = uniform(static_cast<const char*>(L.K) + x.row[kb] * C::RB) + (r * C::RB + 4 * KD * j);
      if constexpr (KD == 4) { const uint4 w = ld16(at); to.k[kb][0] = w.x; to.k[kb][1] = w.y; to.k[kb][2] = w.z; to.k[kb][3] = w.w; }
      else { const v2u_t w = *(const g_v2u_t*)at; to.k[kb][0] = w.x; to.k[kb][1] = w.y; }
      to.kp[kb] = *(const g_u8_t*)(uniform(reinterpret_cast<const char*>(L.K_scale) + x.row[kb] * C::GPR) + (r * C::GPR + KD * j / 4));
    }
  };
  auto fetch_values = [&](const At& x, Codes& to) {
#pragma unroll
    for (int y = 0; y < NL; ++y) {
      const int half = D == 128 ? y : lane >> 5;    // (rows of 64: 32 of them in one load)
      const uint32_t r = D == 128 ? (uint32_t)min(lane >> 2, x.last[y]) : (uint32_t)min((lane >> 1) & 15, half ? x.last[1] : x.last[0]);
      const uint32_t c = D == 128 ? lane & 3 : lane & 1;
      const char* codes = uniform(static_cast<const char*>(L.V) + x.row[D == 128 ? y : 0] * C::RB);
      const char* powers = uniform(reinterpret_cast<const char*>(L.V_scale) + x.row[D == 128 ? y : 0] * C::GPR);
      if constexpr (D == 64) {
        const char* const c1 = uniform(static_cast<const char*>(L.V) + x.row[1] * C::RB);
        const char* const p1 = uniform(reinterpret_cast<const char*>(L.V_scale) + x.row[1] * C::GPR);
        codes = half ? c1 : codes; powers = half ? p1 : powers;
      }
      to.v[y] = ld16_nt(codes + (r * C::RB + 16 * c));
      to.vp[y] = *(const g_u8_t*)(powers + (r * C::GPR + c));
    }
  };

  f32x4_t o[R][NE];
  float m[R], l[R];
#pragma unroll
  for (int n = 0; n < R; ++n) {
#pragma unroll
    for (int e = 0; e < NE; ++e) o[n][e] = f32x4_t{};
    m[n] = -FLT_MAX; l[n] = 0.f;
  }
  // the lane's places in the wave's tile of V: of its first row's pieces (the others by exclusive or), of its column's rows
  const int put_row = D == 128 ? lane >> 2 : lane >> 1, put_piece = D == 128 ? 4 * (lane & 3) : 4 * (lane & 1), get_row = 4 * j + i / 4;
  const uint32_t tile_at = lds_at(s_stage) + wave * C::VB;
  uint32_t put = tile_at + put_row * (2 * D) + ((put_piece ^ C::swizzle(put_row)) << 4);
  uint32_t get = tile_at + get_row * (2 * D) + ((((i & 3) >> 1) ^ C::swizzle(get_row)) << 4) + (i & 1) * 8;

  if (tile0 + wave < tile1) {
    const At x = locate(tile0 + wave);
    fetch_keys(x, now);
    fetch_values(x, now);
  }
#pragma unroll 1
  for (int tl = tile0 + wave; tl < tile1; tl += NW) {
    asm volatile("" : "+v"(put), "+v"(get));        // (their exclusive ors take an instruction each, not registers of their own)
    // (the last one again where there are no more: a load under a condition would have the compiler wait for all loads before the next use)
    const At ahead = locate(tl + NW < tile1 ? tl + NW : tl);
    // ---- sc[n][kb][r]: slot first + 16 kb + 4 j + r of row 16 n + i
    f32x4_t sc[R][2];
#pragma unroll
    for (int n = 0; n < R; ++n) sc[n][0] = sc[n][1] = f32x4_t{};
#pragma unroll
    for (int x = 0; x < KD; ++x) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8_t k = __builtin_bit_cast(bf16x8_t, q4_open(now.k[kb][x], __uint_as_float(now.kp[kb] << 23)));
#pragma unroll
        for (int n = 0; n < R; ++n)
#pragma unroll
          for (int p = 0; p < NP; ++p) sc[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(bf16x8_t, qp[n][p][x]), sc[n][kb], 0, 0, 0);
      }
    }
    fetch_keys(ahead, now);               // (into registers that have just been used)
    // ---- V to LDS as bf16
    const int first = w.tile_of(tl) * kQ4Slots;
    const bool edge = w.is_edge(w.tile_of(tl));
    uint64_t odd[NL] = {};                          // (lanes whose group is not finite, where not every row sees it)
#pragma unroll
    for (int y = 0; y < NL; ++y) {
      uint4 w = now.v[y];
      uint32_t power = now.vp[y];
      if (edge) {
        const bool left_out = power > 252u;
        odd[y] = __ballot(left_out);
        w.x = left_out ? 0u : w.x; w.y = left_out ? 0u : w.y; w.z = left_out ? 0u : w.z; w.w = left_out ? 0u : w.w;
        power = left_out ? 127u : power;
      }
      const float vs = __uint_as_float(power << 23);
      const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int p = 0; p < 4; ++p)
        *(lds_v4u_t*)(uintptr_t)((put ^ (p << 4)) + y * (32 * D)) = __builtin_bit_cast(v4u_t, q4_open(c[p], vs));
    }
    fetch_values(ahead, now);
    asm volatile("" ::: "memory");                  // (a wave's LDS accesses are done in order)
    // ---- softmax
    uint32_t pw[R][NV][4];
#pragma unroll
    for (int n = 0; n < R; ++n) {
      f32x4_t (&s)[2] = sc[n];
      if (edge) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[kb][r] = w.sees(first + 16 * kb + 4 * j + r, back[n]) ? s[kb][r] : -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      if (__any(top > m[n] + a.near)) {             // the reference of a row moves when one of its logits is 2^8 times beyond it
        top = lanes16_max(top);
        const float to = top > m[n] + a.near ? top : m[n], keep = exp2_fast((m[n] - to) * a.scale);
        m[n] = to;
        l[n] *= keep;
#pragma unroll
        for (int e = 0; e < NE; ++e) o[n][e] *= keep;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const float x = exp2_fast((s[kb][r] - m[n]) * a.scale), y = exp2_fast((s[kb][r + 1] - m[n]) * a.scale);
          l[n] += x + y;
          uint32_t w[NV];
          split16<NV>(x, y, w);
#pragma unroll
          for (int k = 0; k < NV; ++k) pw[n][k][2 * kb + r / 2] = w[k];
        }
    }
    // ---- O^T += V^T.P^T, four blocks of 16 elements at a time
#pragma unroll
    for (int e0 = 0; e0 < NE; e0 += 4) {
      bf16x8_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t at = get ^ ((e0 + e) << 5);
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)at);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)(at + 32 * D));
        v[e] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int n = 0; n < R; ++n)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const bf16x8_t pk = __builtin_bit_cast(bf16x8_t, make_uint4(pw[n][k][0], pw[n][k][1], pw[n][k][2], pw[n][k][3]));
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][e0 + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[e], pk, o[n][e0 + e], 0, 0, 0);
        }
    }
    // the groups that are not finite, to the rows that see them
#pragma unroll
    for (int y = 0; y < NL; ++y)
      while (odd[y]) {
        const int from = __builtin_ctzll(odd[y]);
        odd[y] &= odd[y] - 1;
        const int slot = first + (D == 128 ? 16 * y + (from >> 2) : from >> 1), group = D == 128 ? from & 3 : from & 1;
#pragma unroll
        for (int n = 0; n < R; ++n) {
          const float add = w.sees(slot, back[n]) ? NAN : 0.f;
#pragma unroll
          for (int e = 0; e < NE; ++e) o[n][e] += e / 2 == group ? add : 0.f;
        }
      }
    asm volatile("" ::: "memory");
  }

  // ---- the waves' sums joined, each row's pieces of 16 bytes in an order without bank conflicts
#pragma unroll
  for (int n = 0; n < R; ++n) {
    l[n] = lanes16_sum(l[n]);
    if (j == 0) { s_m[wave][16 * n + i] = m[n]; s_l[wave][16 * n + i] = l[n]; }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < R; ++n) {
    float top = s_m[0][16 * n + i];
#pragma unroll 2
    for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][16 * n + i]);
    const float keep = exp2_fast((m[n] - top) * a.scale);
    float4* const mine = reinterpret_cast<float4*>(s_stage) + (wave * M + 16 * n + i) * PP;
#pragma unroll
    for (int e = 0; e < NE; ++e) mine[(4 * e + j) ^ i] = make_float4(o[n][e][0] * keep, o[n][e][1] * keep, o[n][e][2] * keep, o[n][e][3] * keep);
  }
  __syncthreads();
  w.template finish<NW>(a, s_stage, s_m, s_l, &s_word, s_flags, bad);
}

// The same for many more rows in bf16: 128 rows and tiles of 64 slots, two workgroups per CU.  A tile is opened once for all four waves: K and V of the
// next ones are on their way in 4 bits in registers (16 bytes of each a thread) and are opened into LDS as bf16 between the products K.Q^T of a
// tile; the exponentials of a tile stand between the products V^T.P^T of the one before.  (Step by step, as the order is written: left to itself, or told by
// groups, the compiler gathers products and vector instructions.  2048 tokens of 64 heads over 8 after 6144 482 -> 463 us, 4 x up to 1067 of 12 over 3 44 ->
// 40; with priority for either part 461 and 40, but 8 x 233 of 256 over 32 104 -> 108.)  Probabilities are rounded to one bf16, as in
// sqa_chunk_attention's form for many rows: the products bound these calls, and a second part would make it half as many again.  (rms error against 64 bits
// 2.3e-3 of the output, of which 1.7e-3 are its own rounding to bf16; sums and statistics are fp32's, from probabilities that are not rounded.)
template <int D> struct Q4Wide {
  using R = TileRows<bf16_t, D>;
  static constexpr int Slots = 64, Rows = 128, TILE = Slots * R::RB;
  static constexpr int STAGE = 4 * TILE > Rows * D * 4 + 8192 ? 4 * TILE : Rows * D * 4 + 8192;            // K, K', V, V'; at the end all rows' sums
  // piece p of row r of V lies at place p ^ v_swizzle(r): 64 bytes of each of 4 rows are read at a time, 8 lanes write one piece of 8 rows (heads of 128: no
  // conflicts; four lanes a row took a quarter more LDS cycles and 0.4 % more time)
  static __device__ __forceinline__ int v_swizzle(int r) { return R::PPR == 8 ? 4 * ((r >> 1) & 1) : 5 * (r & 3) ^ ((r >> 2) & 1); }
};

template <int D> __global__ __launch_bounds__(256, 2) void q4_attention_wide_kernel(const Q4AttentionArgs a) {
  using T = bf16_t;
  using C = Q4Wide<D>;
  using R = TileRows<T, D>;
  constexpr int NB = D / 32, NS = Frag<T, D>::NS, TILE = C::TILE, KT = C::Slots, GPR = D / kGroup, KD = D / 32;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];
  __shared__ float s_m[1][C::Rows], s_l[1][C::Rows];
  __shared__ __attribute__((aligned(16))) uint8_t s_odd[2][256];                         // of a tile of V: is a thread's part not finite, and left out?
  __shared__ int s_word, s_flags[4];
  int* const s_table = reinterpret_cast<int*>(s_stage + C::STAGE);
  Q4Work<T, D, 256, C::Rows, KT> w;
  if (!w.locate(a)) return;
  const sqa_q4_cache& L = a.a.L;
  const int tid = threadIdx.x, lane = tid & 63, wave = scalar(tid >> 6), col = lane & 31, half = lane >> 5;

  // ---- this lane's query row
  int t, head;
  w.place(min(w.row0 + 32 * wave + col, w.last_row), t, head);
  const int back = w.s.n - 1 - t;
  Frag<T, D> q;
  {
    const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (((int64_t)w.b * a.a.c.Hq + head) * a.a.c.T + t) * D);
#pragma unroll
    for (int x = 0; x < NS; ++x) q.p[x] = ld16(src + (2 * x + half) * 16);
  }
  const bool bad = w.stage_blocks(L, s_table, s_flags);

  // ---- a thread's part of a tile: 8 KD numbers of a row, a wave the same part of all 64
  const int row = lane, part = wave;
  const int64_t unit_row = (int64_t)w.u * L.capacity;
  auto row_of = [&](int j) {                        // (slots behind the last one: that one again)
    const int from = w.tile_of(w.tile0 + j) * KT, at = min(row, w.end - 1 - from), slot = from + at;
    return L.block_table ? (int64_t)s_table[KT / SQA_BLOCK_SLOTS * j + at / SQA_BLOCK_SLOTS] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : unit_row + slot;
  };
  struct Codes { uint32_t c[KD], power; };
  auto fetch = [&](const void* codes, const uint8_t* powers, int64_t at) {
    Codes x;
    const char* from = static_cast<const char*>(codes) + at * (D / 2) + 4 * KD * part;
    if constexpr (KD == 4) { const uint4 v = ld16(from); x.c[0] = v.x; x.c[1] = v.y; x.c[2] = v.z; x.c[3] = v.w; }
    else { const v2u_t v = *(const g_v2u_t*)from; x.c[0] = v.x; x.c[1] = v.y; }
    x.power = *(const g_u8_t*)(powers + at * GPR + KD * part / 4);
    return x;
  };
  const uint32_t lds0 = lds_at(s_stage);
  auto put_piece = [&](const Codes& x, int p, uint32_t tile, int swizzle) {
    *(lds_v4u_t*)(uintptr_t)(lds0 + tile + row * R::RB + (((KD * part + p) ^ swizzle) << 4)) = __builtin_bit_cast(v4u_t, q4_open(x.c[p], __uint_as_float(x.power << 23)));
  };
  auto is_edge = [&](int j) { return w.is_edge(w.tile_of(w.tile0 + j)); };
  auto leave_out = [&](Codes& x, int j) {           // a slot that a row does not see has probability 0, but 0 x NaN is NaN: see odd_values()
    const bool odd = x.power > 252u;
    s_odd[j & 1][4 * row + part] = odd;
#pragma unroll
    for (int p = 0; p < KD; ++p) x.c[p] = odd ? 0u : x.c[p];
    x.power = odd ? 127u : x.power;
  };

  // ---- the lane's places in a tile of K and of V
  int k_at[NS], v_at[NB];
#pragma unroll
  for (int x = 0; x < NS; ++x) k_at[x] = col * R::RB + (((2 * x + half) ^ R::k_swizzle(col)) << 4);
  {
    const int r = 4 * half + (lane & 15) / 4;
#pragma unroll
    for (int e = 0; e < NB; ++e) v_at[e] = r * R::RB + (((4 * e + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ C::v_swizzle(r)) << 4) + (lane & 1) * 8;
  }

  f32x16_t o[NB], sc[2];
  bf16x8_t p[4];
#pragma unroll
  for (int e = 0; e < NB; ++e) o[e] = f32x16_t{};
  float m = -FLT_MAX, l = 0.f;                       // m: a reference that a row's largest logit is near, not always that logit

  Codes kc, vc;
  // sc = K.Q^T of tile j, and between the products V of tile j and K of the next one opened into LDS
  auto keys = [&](int j) {
    if (is_edge(j)) leave_out(vc, j);
    const char* const Kt = s_stage + (j & 1) * TILE;
    constexpr int N = 2 * NS, AHEAD = 3;
    uint4 k[AHEAD + 1];
    auto fetch_k = [&](int n) { k[n % (AHEAD + 1)] = *reinterpret_cast<const uint4*>(Kt + k_at[n / 2] + 32 * (n % 2) * R::RB); };
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) fetch_k(n);
    sc[0] = sc[1] = f32x16_t{};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (n + AHEAD < N) fetch_k(n + AHEAD);
      mma_piece<T>(k[n % (AHEAD + 1)], q.p[n / 2], sc[n % 2]);
      if (n % 2) {
        const int p = n / 2;
        if (p < KD) put_piece(vc, p, (2 + (j & 1)) * TILE, C::v_swizzle(row));
        else put_piece(kc, p - KD, ((j + 1) & 1) * TILE, R::k_swizzle(row));
      }
      __builtin_amdgcn_sched_barrier(0);
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
  auto odd_values = [&](int j) {
    if (is_edge(j)) {                               // the groups that are not finite, to the rows that see them
      uint64_t odd = __ballot(reinterpret_cast<const uint32_t*>(s_odd[j & 1])[lane] != 0);            // (a lane per slot)
      while (odd) {
        const int r = __builtin_ctzll(odd);
        odd &= odd - 1;
        const float add = w.sees(w.tile_of(w.tile0 + j) * KT + r, back) ? NAN : 0.f;
#pragma unroll
        for (int e = 0; e < NB; ++e)
          if (s_odd[j & 1][4 * r + 4 / KD * e]) o[e] += add;
      }
    }
  };
  auto softmax = [&](int j, bool before) {           // p of tile j; before: and o += V^T.P^T of the tile before it
    if (is_edge(j)) {
      const int first = w.tile_of(w.tile0 + j) * KT;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] = w.sees(first + 32 * kb + c_row(i, half), back) ? sc[kb][i] : -INFINITY;
    }
    float top = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kb][i]);
    top = other_half_max(top);
    // the reference of a row moves when one of its logits is 2^8 times beyond it: seldom after the first tiles
    if (const bool beyond = top > m + a.near; __any(beyond)) {
      if (before) { values(j - 1); odd_values(j - 1); }
      before = false;
      const float to = beyond ? top : m, keep = exp2_fast((m - to) * a.scale);
      m = to;
      l *= keep;
#pragma unroll
      for (int e = 0; e < NB; ++e) o[e] *= keep;
    }
    float off = m * a.scale;
    // s scale - off in one operation is off by the rounding of `off`: far from 0 the difference is taken first, each row for itself
    if (const bool far = fabsf(off) > kQ4FarLogit; __any(far)) {
      const float from = far ? m : 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) sc[kb] -= from;
      off = far ? 0.f : off;
    }
    float l0 = 0.f, l1 = 0.f;
    if (!before) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float x = exp2_fast(fmaf(sc[kb][i], a.scale, -off)), y = exp2_fast(fmaf(sc[kb][i + 1], a.scale, -off));
          l0 += x; l1 += y;
          p[2 * kb + i / 8][i % 8] = (__bf16)x; p[2 * kb + i / 8][i % 8 + 1] = (__bf16)y;
        }
    } else {
      bf16x8_t pn[4];
      const char* const Vt = s_stage + (2 + ((j - 1) & 1)) * TILE;
      constexpr int N = 4 * NB, AHEAD = 3;           // products; fragments of V on their way
      s16x4_t vlo[AHEAD + 1], vhi[AHEAD + 1];
      auto fetch_v = [&](int n) {
        const char* at = Vt + v_at[n % NB] + 16 * (n / NB) * R::RB;
        vlo[n % (AHEAD + 1)] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at));
        vhi[n % (AHEAD + 1)] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 8 * R::RB));
      };
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) fetch_v(n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        if (n < N) {
          if (n + AHEAD < N) fetch_v(n + AHEAD);
          const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(vlo[n % (AHEAD + 1)], vhi[n % (AHEAD + 1)], 0, 1, 2, 3, 4, 5, 6, 7));
          o[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[n / NB], o[n % NB], 0, 0, 0);
        }
        const int kb = n / 8, i = 2 * n % 16;
        const float x = exp2_fast(fmaf(sc[kb][i], a.scale, -off)), y = exp2_fast(fmaf(sc[kb][i + 1], a.scale, -off));
        l0 += x; l1 += y;
        pn[2 * kb + i / 8][i % 8] = (__bf16)x; pn[2 * kb + i / 8][i % 8 + 1] = (__bf16)y;
        __builtin_amdgcn_sched_barrier(0);
      }
      // (without it the compiler takes these exponentials out again, to be one with those of the other branch)
      asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(pn[2]), "+v"(pn[3]), "+v"(l0), "+v"(l1));
#pragma unroll
      for (int x = 0; x < 4; ++x) p[x] = pn[x];
      odd_values(j - 1);
    }
    l += l0 + l1;
  };

  const int n = w.tile1 - w.tile0;
  {
    const int64_t at = row_of(0);
    kc = fetch(L.K, L.K_scale, at);
#pragma unroll
    for (int p = 0; p < KD; ++p) put_piece(kc, p, 0, R::k_swizzle(row));
    vc = fetch(L.V, L.V_scale, at);
    kc = fetch(L.K, L.K_scale, row_of(min(1, n - 1)));
  }
  __syncthreads();
  for (int j = 0; j < n; ++j) {
    keys(j);
    kc = fetch(L.K, L.K_scale, row_of(min(j + 2, n - 1)));           // (the last one again where there are no more)
    vc = fetch(L.V, L.V_scale, row_of(min(j + 1, n - 1)));
    softmax(j, j > 0);
    __syncthreads();
  }
  values(n - 1);
  odd_values(n - 1);
  __syncthreads();

  // ---- sums to LDS as rows
  l = other_half_sum(l);
  if (half == 0) { s_m[0][32 * wave + col] = m; s_l[0][32 * wave + col] = l; }
  float4* const mine = reinterpret_cast<float4*>(s_stage) + (32 * wave + col) * (D / 4);
#pragma unroll
  for (int e = 0; e < NB; ++e)
#pragma unroll
    for (int i = 0; i < 16; i += 4) mine[(8 * e + c_row(i, half) / 4) ^ (col & 15)] = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
  __syncthreads();
  w.template finish<1>(a, s_stage, s_m, s_l, &s_word, s_flags, bad);
}

struct Q4Plan { int waves, rows, tiles, splits; bool tile_major; };   // waves and rows (16, 32, 128) of a workgroup, row tiles of a unit, workgroups that share out the slots of the same rows
static Q4Plan q4_plan(sqa_dtype dt, int B, int T, int Hq, int Hkv, int32_t new_pos, int32_t capacity, bool uniform) {
  Q4Plan p;
  const int64_t slots = uniform ? std::min<int64_t>((int64_t)new_pos + T, capacity) : capacity, rows = (int64_t)T * (Hq / Hkv);
  const int64_t units = (int64_t)B * Hkv, wide = units * ((rows + 127) / 128);
  int64_t s;
  // 128 rows a workgroup where they fill the chip, or nearly do over many slots (a join of 128 rows costs what some hundred slots do), and half of them or more
  // are there.  32 heads over 8, us with 16, 32 and 128 rows: 16 x 24 tokens after 4000 65, 75 and 60, 64 x 24 after 1000 75, 73 and 51 (64 x 33 with 32 rows
  // 105, 64 x 48 with 128 94), 16 x 64 after 500 29, 26 and 23, 8 x 64 after 2000 48, 40 and 38, 1 x 256 after 30000 288, 214 and 172; 64 x 16 after 1000 47, 41 and 45, 16 x 32 after 500 17, 17 and 20, 1 x 256 after
  // 4000 48, 38 and 41, 1 x 128 after 30000 150, 116 and 126.
  if (dt == SQA_BF16 && rows >= kQ4WideRows && (wide >= 256 || (wide >= 64 && wide * slots >= 300000))) {
    p.rows = 128; p.waves = 4;
    p.tiles = (int)((rows + 127) / 128);
    s = std::min(512 / wide, slots / 1024);         // (two workgroups per CU; 64 of them over 4256 slots: 4 a unit 42 us, 8 67)
    // The longest row tiles of all units first, where a chunk's rows differ much in what they see: an XCD's units in turn leave some XCDs with the long ones.
    // (us, units in turn and the longest first: 8 x 2048 tokens of 32 heads 371 and 338, 34 x up to 936 of 16 over 4 156 and 139, 13 x up to 1019 of 6 over 2 45
    // and 36, 4 x up to 1067 after 254 49 and 43; 2048 after 6144 482 and 481; 40 x up to 417 of 5 over 1 after 9155 384 and 400, units' tiles meeting in L2.)
    p.tile_major = (int64_t)T * 4 >= slots;
  } else {
    // 32 rows a workgroup (codes are opened once for both 16s, and half as many waves fit) where there is work enough for it: 32 heads over 8, us with
    // 16 and with 32 rows: 16 x 5 tokens after 4000 29.1 and 27.1, 16 x 16 49.4 and 40.2, 64 x 5 after 1000 28.2 and 25.3, 64 x 16 47.3 and 40.6, 1 x 128
    // after 4000 26.6 and 24.9; 16 x 5 after 500 9.7 and 12.2, 4 x 16 after 2000 14.4 and 15.7, 1 x 5 after 30000 23.5 and 27.4.
    p.tile_major = false;
    p.rows = dt == SQA_BF16 && rows > 16 && units * ((rows + 31) / 32) * slots >= 400000 ? 32 : 16;
    p.tiles = (int)((rows + p.rows - 1) / p.rows);
    const int64_t items = units * p.tiles;
    // A join through the workspace costs 5 us, one inside a workgroup 1: units are shared out among waves before workgroups, and among these
    // only until every CU has one.  (256 units of 1000 slots: 8 waves 12.2 us, 4 with 3 workgroups a unit 14.0; 8 units of 30000: 32
    // workgroups of 8 waves each 19.2, 64 22.8, 64 of 4 waves 24.6; 512 units of 1000: 4 waves 18.7, 8 20.0; 2048 of 571: 2 waves 31.2, 4 36.5, 8 44.)
    p.waves = items >= 1024 ? 2 : (items >= 512 ? 4 : 8);
    // (8 tiles at least, a wave each, of units as long as `slots`.  In a ragged batch that is the capacity, and shorter units are cut into as many shares.
    // One token of 32 heads over 8 with no slot to spare and with room for 32768, us: 1 sequence of 500 tokens 9.1 and 12.1, of 2000 12.0 and 13.9, 8 of 500
    // 8.5 and 9.8, 8 of 2000 12.3 and 12.0.)
    s = std::min(256 / items, slots / 256);
  }
  s = std::min<int64_t>(s, kQ4Splits);
  p.splits = s < 1 ? 1 : (int)s;
  return p;
}
// rows of sums that may be joined: no more workgroups than the plan shares out slots to
static size_t q4_records(int T, int Hq, int Hkv) {
  const int64_t rows = (int64_t)T * (Hq / Hkv);
  return rows >= kQ4WideRows ? 512 * 128 : rows > 16 ? 256 * 32 : 256 * 16;
}

static sqa_status start_q4(void (*fn)(Q4AttentionArgs), int threads, size_t lds, const Q4AttentionArgs& a, hipStream_t st) {
  if (a.a.L.block_table) lds += (size_t)(a.a.L.blocks_per_unit + 3) / 4 * 16 + 16;       // (whole tiles of block numbers)
  SQA_HIP_CHECK(allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds));
  const int64_t work = (int64_t)a.a.c.B * a.a.c.Hkv * a.tiles * a.splits;
  fn<<<(unsigned)xcd_grid(work), threads, lds, st>>>(a);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}
template <typename T, int D> static sqa_status launch_q4(const Q4Plan& p, const Q4AttentionArgs& a, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (p.rows == 128) return start_q4(q4_attention_wide_kernel<D>, 256, Q4Wide<D>::STAGE, a, st);
  const size_t lds = (size_t)p.waves * (p.rows / 16) * Q4Tile<T, D>::VB;
  if constexpr (sizeof(T) == 2)
    if (p.rows == 32) {
      if (p.waves == 2) return start_q4(q4_attention_kernel<T, D, 2, 2>, 128, lds, a, st);
      return p.waves == 8 ? start_q4(q4_attention_kernel<T, D, 8, 2>, 512, lds, a, st) : start_q4(q4_attention_kernel<T, D, 4, 2>, 256, lds, a, st);
    }
  if (p.waves == 2) return start_q4(q4_attention_kernel<T, D, 2, 1>, 128, lds, a, st);
  return p.waves == 8 ? start_q4(q4_attention_kernel<T, D, 8, 1>, 512, lds, a, st) : start_q4(q4_attention_kernel<T, D, 4, 1>, 256, lds, a, st);
}

}  // namespace sqa

extern "C" size_t sqa_q4_workspace_bytes(const sqa_q4_cache* layer, int B, int T, int Hq, int Hkv, int D) {
  sqa_status why;
  if (!layer || sqa::bad_q4(*layer, D, &why) || sqa::bad_chunk_shape(B, T, Hq, Hkv, D, 0, nullptr)) return 0;
  return sqa::kChunkCounterBytes + sqa::q4_records(T, Hq, Hkv) * (D / 4 + 1) * 16;
}

extern "C" sqa_status sqa_q4_attention(const void* q, sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos,
                                       const sqa_q4_cache* layer, void* out, float* lse, void* workspace, size_t ws_bytes, void* stream,
                                       const sqa_batch_opts* opts) {
  using namespace sqa;
  if (!q || !layer || !out || !workspace) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  sqa_status why;
  if (bad_q4(*layer, D, &why)) return why;
  if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return SQA_ERR_SHAPE;
  const size_t need = sqa_q4_workspace_bytes(layer, B, T, Hq, Hkv, D);
  if (ws_bytes < need) return SQA_ERR_CAPACITY;
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  if (uniform && (int64_t)new_pos + T > layer->capacity && T > layer->capacity - layer->n_sink) return SQA_ERR_CAPACITY;
  const size_t es = dt == SQA_F32 ? 4 : 2, qb = (size_t)B * Hq * T * D * es, lb = (size_t)B * Hq * T * sizeof(float);
  if (overlap(q, qb, out, qb) || (lse && (overlap(lse, lb, q, qb) || overlap(lse, lb, out, qb)))) return SQA_ERR_SHAPE;
  // (workgroups that still read these would see what others have stored)
  if (overlap(workspace, need, q, qb) || overlap(workspace, need, out, qb) || (lse && overlap(workspace, need, lse, lb)) || in_q4(*layer, B, Hkv, D, out, qb) ||
      in_q4(*layer, B, Hkv, D, lse, lb) || in_q4(*layer, B, Hkv, D, workspace, need)) return SQA_ERR_SHAPE;
  const Q4Plan p = q4_plan(dt, B, T, Hq, Hkv, new_pos, layer->capacity, uniform);
  if ((int64_t)B * Hkv * p.tiles * p.splits > INT32_MAX - 8) return SQA_ERR_SHAPE;
  Q4AttentionArgs a{};
  a.a = q4_args(layer, B, T, Hq, Hkv, new_pos, opts);
  a.q = q; a.out = out; a.lse = lse;
  a.count = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float4*>(static_cast<char*>(workspace) + kChunkCounterBytes);
  a.scale = (float)(1.4426950408889634 / sqrt((double)D));
  a.near = 8.f / a.scale;
  auto reciprocal = [](int d) { return 0xffffffffu / (uint32_t)d + 1; };
  a.group_m = reciprocal(a.a.c.g); a.heads_m = reciprocal(Hkv); a.tiles_m = reciprocal(p.tile_major ? B * Hkv : p.tiles); a.splits_m = reciprocal(p.splits);
  a.tiles = p.tiles; a.splits = p.splits; a.tile_major = p.tile_major;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? launch_q4<float, 64>(p, a, st) : launch_q4<float, 128>(p, a, st);
  return D == 64 ? launch_q4<bf16_t, 64>(p, a, st) : launch_q4<bf16_t, 128>(p, a, st);
}

extern "C" sqa_status sqa_q4_plan(const sqa_q4_cache* layer, sqa_dtype dt, int B, int T, int Hq, int Hkv, int D, int32_t new_pos,
                                  const sqa_batch_opts* opts, sqa_q4_plan_info* info) {
  if (!layer || !info) return SQA_ERR_NULL;
  if (dt != SQA_F32 && dt != SQA_BF16) return SQA_ERR_DTYPE;
  if (sqa::bad_chunk_shape(B, T, Hq, Hkv, D, new_pos, opts)) return SQA_ERR_SHAPE;
  if (layer->capacity < 1 || layer->capacity > sqa::kQ4MostSlots) return SQA_ERR_CAPACITY;
  const sqa::Q4Plan p = sqa::q4_plan(dt, B, T, Hq, Hkv, new_pos, layer->capacity, !(opts && (opts->prompt_len || opts->new_pos_seq)));
  info->rows = p.rows; info->waves = p.waves; info->row_tiles = p.tiles; info->slot_splits = p.splits; info->rounded_probs = p.rows == 128;
  return SQA_OK;
}
