// 32 x 32 blocks of products on the matrix cores, and rows of D elements staged in LDS for them.
//   bf16  v_mfma_f32_32x32x16_bf16: A row / B column = lane % 32, a lane of half j = lane / 32 holds 8 contraction slots
//   fp32  v_mfma_f32_32x32x2_f32: one slot per lane half
//   C     column = lane % 32, rows 8 (i / 4) + 4 j + i % 4 for i = 0..15
// Which elements are a lane's contraction slots is free as long as both operands agree: q.k takes the row's 16-byte pieces
// 2 s + j; p.V takes the rows of C as they come out, so probabilities go from one product to the next without leaving the lane.
#pragma once
#include <cfloat>
#include "sqa_chunk.h"

namespace sqa {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

typedef __attribute__((address_space(3))) const char lds_char_t;
__device__ __forceinline__ uint32_t lds_at(const char* p) { return (uint32_t)(uintptr_t)(lds_char_t*)p; }

// Direct global -> LDS copy, lds + 16 x lane <- *g of each lane; as an instruction, because the compiler would wait for
// all copies in flight before the first read of a buffer.  Whoever reads it waits: vmcnt, then the workgroup's barrier.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void fetch16(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(g), "s"(__builtin_amdgcn_readfirstlane(lds)) : "m0", "memory");
}
__device__ __forceinline__ void fetch16(const void* base /*the same in all lanes*/, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);        // (the builtin's result is signed)
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  return reinterpret_cast<const char*>((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ void fetched() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float other_half_max(float v) {
  typedef unsigned u2_t __attribute__((ext_vector_type(2)));
  const u2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float other_half_sum(float v) {
  typedef unsigned u2_t __attribute__((ext_vector_type(2)));
  const u2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}
// row of C that a lane half j holds in register i
__device__ __forceinline__ constexpr int c_row(int i, int j) { return 8 * (i / 4) + 4 * j + i % 4; }

// A row's 16-byte pieces as they lie in LDS, no padding: piece p of row r at place p ^ swizzle(r).
template <typename T, int D> struct TileRows {
  static constexpr int E = 16 / (int)sizeof(T);
  static constexpr int RB = D * (int)sizeof(T);     // bytes of a row: 128, 256 or 512
  static constexpr int PPR = RB / 16;
  static constexpr int RPI = SQA_WAVE / PPR;        // rows of a wave's 1 KB copy
  // read as q.k's operand: one piece of each of 16 rows at a time, in 16 different columns of the banks
  static __device__ __forceinline__ int k_swizzle(int r) { return PPR == 8 ? (r >> 1) & 7 : r & 15; }
  // read as p.V's: bf16 by transposed reads of 64 bytes of each of 4 rows; fp32 rows r and r + 4 beside each other
  static __device__ __forceinline__ int v_swizzle(int r) {
    if constexpr (sizeof(T) == 2) return PPR == 8 ? 4 * ((r >> 1) & 1) : 4 * (r & 3);
    return 0;
  }
};

// the pieces of one row of Q or K as a lane holds them: NS steps of 16 bytes
template <typename T, int D> struct Frag {
  static constexpr int NS = D * (int)sizeof(T) / 32;
  uint4 p[NS];
};

// The compiler waits for the row's loads here, not at their first use: inside a loop that wait would be for all copies in flight.
template <typename T, int D> __device__ __forceinline__ void arrived(Frag<T, D>& f) {
#pragma unroll
  for (int i = 0; i < Frag<T, D>::NS; ++i) asm volatile("" : "+v"(f.p[i].x), "+v"(f.p[i].y), "+v"(f.p[i].z), "+v"(f.p[i].w));
}

// c += a.b over the contraction slots of one piece of each lane
template <typename T> __device__ __forceinline__ void mma_piece(const uint4& a, const uint4& b, f32x16_t& c);
template <> __device__ __forceinline__ void mma_piece<bf16_t>(const uint4& a, const uint4& b, f32x16_t& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma_piece<float>(const uint4& a, const uint4& b, f32x16_t& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

// Consecutive workgroups go to the 8 XCDs of the chip in turn, each with an L2 of its own: an XCD takes one run of the
// work items, so that items that read the same rows read them through the same L2.  `count` items, a grid of xcd_grid(count).
__device__ __forceinline__ int64_t xcd_item(int64_t count) {
  const int64_t per = (count + 7) / 8;
  const int64_t slot = blockIdx.x >> 3;
  const int64_t i = (int64_t)(blockIdx.x & 7) * per + slot;
  return slot < per && i < count ? i : -1;
}
inline int64_t xcd_grid(int64_t count) { return (count + 7) / 8 * 8; }

}  // namespace sqa
