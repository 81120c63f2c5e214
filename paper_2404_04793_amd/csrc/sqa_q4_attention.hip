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
constexpr int kQ4Records = 16384;                   // rows of sums that the workspace has room for

struct Q4AttentionArgs {
  Q4Args a;
  const void* q;
  void* out;
  float* lse;
  int32_t* count;                                   // [items]
  float4* part;                                     // [items][splits][rows][D / 4 + 1]: sums, then (m, l, bad)
  float scale;                                      // log2(e) / sqrt(D)
  float near;                                       // 8 / scale: logits that close to a row's reference do not move it
  uint32_t group_m;                                 // 2^32 / g, for divisions by g
  int tiles, splits;
};

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
  // piece p (16 bytes) of row r of V in bf16 lies at place p ^ swizzle(r): both the writes (8 lanes: 2 or 4 rows) and the transposing
  // reads (32 bytes of each of 16 rows) meet all banks
  static __device__ __forceinline__ int swizzle(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
};

template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW) void q4_attention_kernel(const Q4AttentionArgs a) {
  using C = Q4Tile<T, D>;
  constexpr int M = 16, NE = C::NE, NL = C::NL, NP = C::NP, NV = C::NV, KD = C::KD, PP = D / 4, REC = PP + 1, NT = 64 * NW;
  extern __shared__ __attribute__((aligned(1024))) char s_stage[];   // V tiles of the waves, at the end their sums; then the table
  __shared__ float s_m[NW][M], s_l[NW][M];
  __shared__ int s_word;
  int* const s_table = reinterpret_cast<int*>(s_stage + NW * C::VB);
  const sqa_q4_cache& L = a.a.L;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, j = lane >> 4;

  // ---- where the work is
  const uint32_t total = (uint32_t)(a.a.c.B * a.a.c.Hkv) * (uint32_t)(a.tiles * a.splits);
  const uint32_t per8 = (total + 7) / 8, work = (blockIdx.x & 7) * per8 + (blockIdx.x >> 3);
  if (blockIdx.x >> 3 >= per8 || work >= total) return;
  const int split = (int)(work % (uint32_t)a.splits);
  const uint32_t item = work / (uint32_t)a.splits;
  const int u = (int)(item / (uint32_t)a.tiles), tile = a.tiles - 1 - (int)(item % (uint32_t)a.tiles);      // (the longest first)
  const int b = u / a.a.c.Hkv, h = u - b * a.a.c.Hkv, g = a.a.c.g;
  const Q4Seq s = q4_seq(a.a, b, tid == 0 && h == 0 && tile == 0 && split == 0);
  const int rows = s.n * g, row0 = tile * M;
  if (row0 >= rows) return;
  const int last_row = min(row0 + M, rows) - 1;
  auto place = [&](int r, int& t, int& head) {
    t = g > 1 ? (int)__umulhi((uint32_t)r, a.group_m) : r;
    int x = r - t * g;
    if (x < 0) { --t; x += g; }
    head = h * g + x;
  };
  int t_first, t_last, any;
  place(row0, t_first, any);
  place(last_row, t_last, any);
  const bool turned = s.end() > s.slots;
  const int len = s.why ? 1 : s.len();
  const int end = turned ? len : min((int)s.pos + t_last + 1, len);                      // slots that the rows see lie before it
  const int whole = turned ? (s.n == 1 ? len : 0) : min((int)s.pos + t_first + 1, len);   // ... that all rows see
  const int nt = (end + kQ4Slots - 1) / kQ4Slots, per = (nt + a.splits - 1) / a.splits, parts = (nt + per - 1) / per;
  const int tile0 = split * per, tile1 = min(tile0 + per, nt);
  if (split >= parts) return;

  auto refuse = [&](int why) {
    if (tid == 0 && a.a.c.status) *a.a.c.status = why;
    constexpr int E = 16 / (int)sizeof(T), PPR = D / E;
    for (int x = tid; x < (last_row + 1 - row0) * PPR; x += NT) {
      int t, head;
      place(row0 + x / PPR, t, head);
      st16(static_cast<T*>(a.out) + (((int64_t)b * a.a.c.T + t) * a.a.c.Hq + head) * D + x % PPR * E, make_uint4(0, 0, 0, 0));
      if (a.lse && x % PPR == 0) a.lse[((int64_t)b * a.a.c.Hq + head) * a.a.c.T + t] = -INFINITY;
    }
  };
  if (s.why) {
    if (split == 0) refuse(s.why);
    return;
  }

  // ---- this lane's query row
  int t, head;
  place(min(row0 + i, last_row), t, head);
  const int back = s.n - 1 - t;                     // a slot of the ring is seen when its token is at least so far behind the newest
  const int newest = s.slot(s.end() - 1);           // ... and it lies here
  const int fixed = turned ? s.sink : 0, ring = s.slots - s.sink;
  auto sees = [&](int slot) {
    int behind = newest - slot;
    if (turned && behind < 0) behind += ring;
    return slot < len && (slot < fixed || behind >= back);
  };
  // its elements 8 KD j .. of step x: 8 (KD j + x) ..
  uint4 qp[NP][KD];
  {
    const T* src = static_cast<const T*>(a.q) + (((int64_t)b * a.a.c.Hq + head) * a.a.c.T + t) * D + 8 * KD * j;
#pragma unroll
    for (int x = 0; x < KD; ++x) {
      if constexpr (sizeof(T) == 2) qp[0][x] = ld16(src + 8 * x);
      else {
        const uint4 lo = ld16(src + 8 * x), hi = ld16(src + 8 * x + 4);
        const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        uint32_t w[4][NP];
#pragma unroll
        for (int y = 0; y < 4; ++y) split16<NP>(__uint_as_float(v[2 * y]), __uint_as_float(v[2 * y + 1]), w[y]);
#pragma unroll
        for (int p = 0; p < NP; ++p) qp[p][x] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
      }
    }
  }

  // ---- block numbers of this workgroup's slots
  int bad = 0;
  if (L.block_table) {
    const int32_t* table = L.block_table + (int64_t)u * L.blocks_per_unit;
    for (int x = tid; x < 2 * (tile1 - tile0); x += NT) {
      const int e = 2 * tile0 + x;
      int blk = e * SQA_BLOCK_SLOTS < end ? table[e] : 0;
      if ((unsigned)blk >= (unsigned)L.n_blocks) { bad = 1; blk = 0; }
      s_table[x] = blk;
    }
    bad = __syncthreads_or(bad);
  }
  const int64_t unit_row = (int64_t)u * L.capacity;
  auto row_of = [&](int slot) {                     // (slots behind the last: that one again)
    slot = min(slot, end - 1);
    return L.block_table ? (int64_t)s_table[slot / SQA_BLOCK_SLOTS - 2 * tile0] * SQA_BLOCK_SLOTS + slot % SQA_BLOCK_SLOTS : unit_row + slot;
  };

  struct Loaded { uint32_t k[2][KD]; uint4 v[NL]; uint32_t kp[2], vp[NL]; };
  auto fetch = [&](int tl, Loaded& x) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int64_t row = row_of(tl * kQ4Slots + 16 * kb + i);
      const char* at = static_cast<const char*>(L.K) + row * C::RB + 4 * KD * j;
      if constexpr (KD == 4) { const uint4 w = ld16(at); x.k[kb][0] = w.x; x.k[kb][1] = w.y; x.k[kb][2] = w.z; x.k[kb][3] = w.w; }
      else { const uint2 w = *reinterpret_cast<const uint2*>(at); x.k[kb][0] = w.x; x.k[kb][1] = w.y; }
      x.kp[kb] = L.K_scale[row * C::GPR + KD * j / 4];
    }
#pragma unroll
    for (int y = 0; y < NL; ++y) {
      const int vr = D == 128 ? 16 * y + (lane >> 2) : lane >> 1, vc = D == 128 ? lane & 3 : lane & 1;
      const int64_t row = row_of(tl * kQ4Slots + vr);
      x.v[y] = ld16(static_cast<const char*>(L.V) + row * C::RB + 16 * vc);
      x.vp[y] = L.V_scale[row * C::GPR + vc];
    }
  };

  f32x4_t o[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e) o[e] = f32x4_t{};
  float m = -FLT_MAX, l = 0.f;
  char* const Vt = s_stage + wave * C::VB;

  Loaded now{}, next{};
  if (tile0 + wave < tile1) fetch(tile0 + wave, now);
#pragma unroll 1
  for (int tl = tile0 + wave; tl < tile1; tl += NW) {
    if (tl + NW < tile1) fetch(tl + NW, next);
    // ---- s[kb][r]: slot 32 tl + 16 kb + 4 j + r of row i
    f32x4_t sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      sc[kb] = f32x4_t{};
      const float power = __uint_as_float(now.kp[kb] << 23);
#pragma unroll
      for (int x = 0; x < KD; ++x) {
        const bf16x8_t k = __builtin_bit_cast(bf16x8_t, q4_open(now.k[kb][x], power));
#pragma unroll
        for (int p = 0; p < NP; ++p) sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(bf16x8_t, qp[p][x]), sc[kb], 0, 0, 0);
      }
    }
    // ---- V to LDS as bf16
    const bool edge = (tl + 1) * kQ4Slots > whole;
    uint64_t odd[NL] = {};                          // (lanes whose group is not finite, where not every row sees it)
#pragma unroll
    for (int y = 0; y < NL; ++y) {
      const int row = D == 128 ? 16 * y + (lane >> 2) : lane >> 1, first = D == 128 ? 4 * (lane & 3) : 4 * (lane & 1);
      uint4 w = now.v[y];
      uint32_t power = now.vp[y];
      if (edge) {
        odd[y] = __ballot(power > 252u);
        if (power > 252u) { w = make_uint4(0, 0, 0, 0); power = 127; }
      }
      const float vs = __uint_as_float(power << 23);
      const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int p = 0; p < 4; ++p)
        *reinterpret_cast<uint4*>(Vt + row * (2 * D) + (((first + p) ^ C::swizzle(row)) << 4)) = q4_open(c[p], vs);
    }
    asm volatile("" ::: "memory");                  // (a wave's LDS accesses are done in order)
    // ---- softmax
    if (edge) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!sees(tl * kQ4Slots + 16 * kb + 4 * j + r)) sc[kb][r] = -INFINITY;
    }
    float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
    if (__any(top > m + a.near)) {                  // the reference of a row moves when one of its logits is 2^8 times beyond it
      top = lanes16_max(top);
      const float to = top > m + a.near ? top : m, keep = exp2_fast((m - to) * a.scale);
      m = to;
      l *= keep;
#pragma unroll
      for (int e = 0; e < NE; ++e) o[e] *= keep;
    }
    uint32_t pw[NV][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float x = exp2_fast((sc[kb][r] - m) * a.scale), y = exp2_fast((sc[kb][r + 1] - m) * a.scale);
        l += x + y;
        uint32_t w[NV];
        split16<NV>(x, y, w);
#pragma unroll
        for (int k = 0; k < NV; ++k) pw[k][2 * kb + r / 2] = w[k];
      }
    // ---- O^T += V^T.P^T
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      s16x4_t half[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int row = 16 * kb + 4 * j + i / 4, piece = (2 * e + ((i & 3) >> 1)) ^ C::swizzle(row);
        half[kb] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(Vt + row * (2 * D) + piece * 16 + (i & 1) * 8));
      }
      const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int k = 0; k < NV; ++k)
        o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, make_uint4(pw[k][0], pw[k][1], pw[k][2], pw[k][3])), o[e], 0, 0, 0);
    }
    // the groups that are not finite, to the rows that see them
#pragma unroll
    for (int y = 0; y < NL; ++y)
      while (odd[y]) {
        const int from = __builtin_ctzll(odd[y]);
        odd[y] &= odd[y] - 1;
        const int slot = tl * kQ4Slots + (D == 128 ? 16 * y + (from >> 2) : from >> 1), group = D == 128 ? from & 3 : from & 1;
        const float add = sees(slot) ? NAN : 0.f;
#pragma unroll
        for (int e = 0; e < NE; ++e) o[e] += e / 2 == group ? add : 0.f;
      }
    asm volatile("" ::: "memory");
    now = next;
  }

  // ---- the waves' sums joined, each row's pieces of 16 bytes in an order without bank conflicts
  l = lanes16_sum(l);
  if (j == 0) { s_m[wave][i] = m; s_l[wave][i] = l; }
  __syncthreads();
  float top = s_m[0][i];
#pragma unroll
  for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][i]);
  const float keep = exp2_fast((m - top) * a.scale);
  float4* const mine = reinterpret_cast<float4*>(s_stage) + (wave * M + i) * PP;
#pragma unroll
  for (int e = 0; e < NE; ++e) mine[(4 * e + j) ^ i] = make_float4(o[e][0] * keep, o[e][1] * keep, o[e][2] * keep, o[e][3] * keep);
  __syncthreads();
  auto joined = [&](int row, float& mm, float& ll) {
    mm = s_m[0][row];
#pragma unroll
    for (int w = 1; w < NW; ++w) mm = fmaxf(mm, s_m[w][row]);
    ll = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) ll += s_l[w][row] * exp2_fast((s_m[w][row] - mm) * a.scale);
  };
  auto piece4 = [&](int row, int p) {
    float4 v = reinterpret_cast<const float4*>(s_stage)[row * PP + (p ^ row)];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      const float4 x = reinterpret_cast<const float4*>(s_stage)[(w * M + row) * PP + (p ^ row)];
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    return v;
  };
  auto store8 = [&](int row, int p, const float4 (&v)[2], float mm, float ll) {          // pieces 2 p and 2 p + 1
    int tt, hh;
    place(row0 + row, tt, hh);
    const float inv = 1.f / ll;
    T* dst = static_cast<T*>(a.out) + (((int64_t)b * a.a.c.T + tt) * a.a.c.Hq + hh) * D + 8 * p;
    if constexpr (sizeof(T) == 2)
      st16(dst, make_uint4(pair(v[0].x * inv, v[0].y * inv), pair(v[0].z * inv, v[0].w * inv), pair(v[1].x * inv, v[1].y * inv), pair(v[1].z * inv, v[1].w * inv)));
    else
#pragma unroll
      for (int k = 0; k < 2; ++k) reinterpret_cast<float4*>(dst)[k] = make_float4(v[k].x * inv, v[k].y * inv, v[k].z * inv, v[k].w * inv);
    if (p == 0 && a.lse) a.lse[((int64_t)b * a.a.c.Hq + hh) * a.a.c.T + tt] = 0.6931471805599453f * fmaf(mm, a.scale, log2f(ll));
  };
  const int live = (last_row + 1 - row0) * (PP / 2);
  if (parts == 1) {
    if (bad) { refuse(SQA_ERR_SHAPE); return; }
    for (int x = tid; x < live; x += NT) {
      const int row = x / (PP / 2), p = x % (PP / 2);
      float mm, ll;
      joined(row, mm, ll);
      const float4 v[2] = {piece4(row, 2 * p), piece4(row, 2 * p + 1)};
      store8(row, p, v, mm, ll);
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
    rec.put(refs + split * M + row, make_float4(mm, ll, (float)bad, 0.f));
  }
  if (!last_to_arrive(a.count + item, parts, &s_word)) return;
  bad = 0;
  for (int x = tid; x < parts; x += NT) bad |= rec.get(refs + x * M).z != 0.f;
  if (__syncthreads_or(bad)) { refuse(SQA_ERR_SHAPE); return; }
  for (int x = tid; x < live; x += NT) {
    const int row = x / (PP / 2), p = x % (PP / 2);
    float mm = -FLT_MAX, ll = 0.f;
    float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int k0 = 0; k0 < parts; k0 += 4) {
      float4 ml[4], w4[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t from = (uint32_t)(min(k0 + k, parts - 1) * M + row);
        ml[k] = rec.get(refs + from); w4[k][0] = rec.get(from * PP + 2 * p); w4[k][1] = rec.get(from * PP + 2 * p + 1);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k0 + k < parts) {
          const float to = fmaxf(mm, ml[k].x), w0 = exp2_fast((mm - to) * a.scale), w1 = exp2_fast((ml[k].x - to) * a.scale);
          mm = to;
          ll = fmaf(ll, w0, ml[k].y * w1);
#pragma unroll
          for (int y = 0; y < 2; ++y)
            v[y] = make_float4(fmaf(v[y].x, w0, w4[k][y].x * w1), fmaf(v[y].y, w0, w4[k][y].y * w1), fmaf(v[y].z, w0, w4[k][y].z * w1), fmaf(v[y].w, w0, w4[k][y].w * w1));
        }
    }
    store8(row, p, v, mm, ll);
  }
}

struct Q4Plan { int tiles, splits; };
static Q4Plan q4_plan(int B, int T, int Hq, int Hkv, int D, int32_t new_pos, int32_t capacity, bool uniform) {
  Q4Plan p;
  const int64_t slots = uniform ? std::min<int64_t>((int64_t)new_pos + T, capacity) : capacity;
  p.tiles = (T * (Hq / Hkv) + 15) / 16;
  const int64_t items = (int64_t)B * Hkv * p.tiles;
  int64_t s = items > kChunkCounters ? 1 : 1024 / items;
  s = std::min(s, slots / 256);
  s = std::min<int64_t>(s, kQ4Records / 16 / items);
  p.splits = s < 1 ? 1 : (int)s;
  return p;
}

template <typename T, int D> static sqa_status launch_q4(const Q4AttentionArgs& a, hipStream_t st) {
  constexpr int NW = 4;
  auto fn = q4_attention_kernel<T, D, NW>;
  size_t lds = NW * Q4Tile<T, D>::VB;
  if (a.a.L.block_table) lds += (size_t)(a.a.L.blocks_per_unit + 3) / 4 * 16 + 16;
  SQA_HIP_CHECK(allow_dynamic_lds(reinterpret_cast<const void*>(fn), lds));
  const int64_t work = (int64_t)a.a.c.B * a.a.c.Hkv * a.tiles * a.splits;
  fn<<<(unsigned)xcd_grid(work), 64 * NW, lds, st>>>(a);
  SQA_HIP_CHECK(hipGetLastError());
  return SQA_OK;
}

}  // namespace sqa

extern "C" size_t sqa_q4_workspace_bytes(const sqa_q4_cache* layer, int B, int T, int Hq, int Hkv, int D) {
  sqa_status why;
  if (!layer || sqa::bad_q4(*layer, D, &why) || sqa::bad_chunk_shape(B, T, Hq, Hkv, D, 0, nullptr)) return 0;
  return sqa::kChunkCounterBytes + (size_t)sqa::kQ4Records * (D / 4 + 1) * 16;
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
  if (ws_bytes < sqa_q4_workspace_bytes(layer, B, T, Hq, Hkv, D)) return SQA_ERR_CAPACITY;
  const bool uniform = !(opts && (opts->prompt_len || opts->new_pos_seq));
  if (uniform && (int64_t)new_pos + T > layer->capacity && T > layer->capacity - layer->n_sink) return SQA_ERR_CAPACITY;
  const size_t es = dt == SQA_F32 ? 4 : 2, qb = (size_t)B * Hq * T * D * es, lb = (size_t)B * Hq * T * sizeof(float);
  if (overlap(q, qb, out, qb) || (lse && (overlap(lse, lb, q, qb) || overlap(lse, lb, out, qb)))) return SQA_ERR_SHAPE;
  const Q4Plan p = q4_plan(B, T, Hq, Hkv, D, new_pos, layer->capacity, uniform);
  if ((int64_t)B * Hkv * p.tiles * p.splits > INT32_MAX - 8) return SQA_ERR_SHAPE;
  Q4AttentionArgs a{};
  a.a = q4_args(layer, B, T, Hq, Hkv, new_pos, opts);
  a.q = q; a.out = out; a.lse = lse;
  a.count = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float4*>(static_cast<char*>(workspace) + kChunkCounterBytes);
  a.scale = (float)(1.4426950408889634 / sqrt((double)D));
  a.near = 8.f / a.scale;
  a.group_m = 0xffffffffu / (uint32_t)a.a.c.g + 1;
  a.tiles = p.tiles; a.splits = p.splits;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dt == SQA_F32) return D == 64 ? launch_q4<float, 64>(a, st) : launch_q4<float, 128>(a, st);
  return D == 64 ? launch_q4<bf16_t, 64>(a, st) : launch_q4<bf16_t, 128>(a, st);
}
