// Rows of heads as projections leave them, a lane holding 16 bytes of one: norm and rotation for waves that take one token and several groups of
// heads (axis_rows_kernel in sqa_chunk_rows.hip, q4_rows_kernel), and the checks of all such calls' arguments.  chunk_rows_kernel, whose waves take
// several tokens of one group, has the same two steps in an order of its own.
#pragma once
#include "sqa_chunk.h"

namespace sqa {

constexpr int kRowsThreads = 256;

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

// Positions on several axes (sqa_rope_axes): which axis a pair goes by, two bits each, as the host works it out.
struct AxesArgs {
  const int32_t* pos;                               // [n][B][T]
  uint32_t axis[4];                                 // pair i: bits 2 (i % 16) of word i / 16
  int n;
};

struct AxisPos { int x, y, z, w; };

// What is done to each row of a head (sqa_head_prep), for lane `lane` of a wave whose rows are LPR lanes each.
template <typename T, int D> struct RowPrep {
  static constexpr int E = Piece<T>::E, LPR = D / E;
  const sqa_head_prep& prep;
  bool mine, first;
  int half, e0, step, partner;
  __device__ __forceinline__ RowPrep(const sqa_head_prep& p, int lane) : prep(p) {
    half = p.rot_dim / 2; e0 = lane % LPR * E; step = p.interleaved ? 0 : half / E;
    mine = p.rope != nullptr && e0 < p.rot_dim; first = e0 < half;
    partner = mine ? (first ? lane + step : lane - step) : lane;
  }
  __device__ __forceinline__ int first_pair() const { return mine ? (prep.interleaved ? e0 / 2 : (first ? e0 : e0 - half)) : 0; }
  // n cosines and sines of neighbouring pairs of one row of the table
  template <int N> __device__ __forceinline__ void neighbours(const float* from, float (&cs)[E], float (&sn)[E]) const {
    if constexpr (N >= 4) {
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        *reinterpret_cast<float4*>(cs + e) = *reinterpret_cast<const float4*>(from + e);
        *reinterpret_cast<float4*>(sn + e) = *reinterpret_cast<const float4*>(from + half + e);
      }
    } else {
      *reinterpret_cast<float2*>(cs) = *reinterpret_cast<const float2*>(from);
      *reinterpret_cast<float2*>(sn) = *reinterpret_cast<const float2*>(from + half);
    }
  }
  // What the lane's pairs turn by (E of them where pairs lie half a head apart, E / 2 where they are neighbours): from the table's row of the
  // token's position,
  __device__ __forceinline__ void angles_of(int64_t pos, float (&cs)[E], float (&sn)[E]) const {
    const float* from = prep.rope + pos * prep.rot_dim + first_pair();
    if (prep.interleaved) neighbours<E / 2>(from, cs, sn);
    else neighbours<E>(from, cs, sn);
  }
  // or of its positions on the axes: a lane of the wave fetches one pair's, and they are handed out through LDS (s_wave: 128 numbers of this wave).
  // (Fetched by each lane that needs them, one pair at a time: 58 us where this takes 50, 2 x 4500 tokens of 40 heads.)
  __device__ __forceinline__ void angles_of(const AxesArgs& a, AxisPos at, float* s_wave, float (&cs)[E], float (&sn)[E]) const {
    const int lane = threadIdx.x & (SQA_WAVE - 1), word = lane / 16;
    uint32_t axis = a.axis[0];
    if (word == 1) axis = a.axis[1];
    if (word == 2) axis = a.axis[2];
    if (word == 3) axis = a.axis[3];
    axis = axis >> 2 * (lane % 16) & 3;
    int p = at.x;
    if (axis == 1) p = at.y;
    if (axis == 2) p = at.z;
    if (axis == 3) p = at.w;
    if (lane < half) {
      const float* from = prep.rope + (int64_t)p * prep.rot_dim + lane;
      s_wave[lane] = from[0];
      s_wave[64 + lane] = from[half];
    }
    asm volatile("" ::: "memory");                  // (a wave's LDS accesses are done in order)
    const int p0 = first_pair();
    const int n = prep.interleaved ? E / 2 : E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
      if (e < n) {
        *reinterpret_cast<float2*>(cs + e) = *reinterpret_cast<const float2*>(s_wave + p0 + e);
        *reinterpret_cast<float2*>(sn + e) = *reinterpret_cast<const float2*>(s_wave + 64 + p0 + e);
      }
  }

  __device__ __forceinline__ void normalise(float (&y)[E], const void* weight) const {
    if (!weight) return;
    float w[E], ss = 0.f;
    Piece<T>::open(ld16(static_cast<const T*>(weight) + e0), w);
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, LPR);
    const float r = 1.f / sqrtf(ss * (1.f / D) + prep.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = y[e] * r * w[e];
  }
  __device__ __forceinline__ void turn(float (&y)[E], const float (&cs)[E], const float (&sn)[E]) const {
    if (prep.interleaved) {
      if (mine) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float p = y[e], q = y[e + 1];
          y[e] = p * cs[e / 2] - q * sn[e / 2];
          y[e + 1] = q * cs[e / 2] + p * sn[e / 2];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float other = step == LPR / 2 ? half_row_away<LPR>(y[e]) : __shfl(y[e], partner);
        const float z = fmaf(y[e], cs[e], first ? -other * sn[e] : other * sn[e]);
        y[e] = mine ? z : y[e];
      }
    }
  }
};

// The positions of token t of sequence b on the axes; those outside the table as the nearest in it, and reported.
__device__ __forceinline__ AxisPos axes_of(const AxesArgs& x, const ChunkArgs& a, int n_pos, int b, int t, bool report) {
  const int32_t* from = x.pos + (int64_t)b * a.T + t;
  const int64_t step = (int64_t)a.B * a.T;
  AxisPos p{from[0], 0, 0, 0};
  if (x.n > 1) p.y = from[step];
  if (x.n > 2) p.z = from[2 * step];
  if (x.n > 3) p.w = from[3 * step];
  const uint32_t most = (uint32_t)n_pos - 1, far = max(max((uint32_t)p.x, (uint32_t)p.y), max((uint32_t)p.z, (uint32_t)p.w));
  if (far > most) {
    if (report && a.status) *a.status = SQA_ERR_SHAPE;
    p.x = min(max(p.x, 0), (int)most); p.y = min(max(p.y, 0), (int)most);
    p.z = min(max(p.z, 0), (int)most); p.w = min(max(p.w, 0), (int)most);
  }
  return p;
}

inline bool bad_rows(const sqa_token_rows& r, int B, int T, size_t es) {
  const int64_t per16 = (int64_t)(16 / es);
  return !aligned16(r.data) || (B > 1 && (r.seq_stride < 0 || r.seq_stride % per16)) || (T > 1 && (r.row_stride < 0 || r.row_stride % per16));
}

inline bool rows_overlap(const sqa_token_rows* r, int B, int T, int H, int D, size_t es, const void* p, size_t n) {
  if (!r) return false;
  const int64_t last = (B > 1 ? (int64_t)(B - 1) * r->seq_stride : 0) + (T > 1 ? (int64_t)(T - 1) * r->row_stride : 0) + (int64_t)H * D;
  return overlap(r->data, (size_t)last * es, p, n);
}

// the library's view of a caller's axes; false: refused
inline bool axes_args(const sqa_rope_axes* axes, const sqa_head_prep* prep, AxesArgs* out, sqa_status* why) {
  *why = SQA_ERR_NULL;
  if (!prep || !prep->rope || !axes->pos) return false;
  *why = SQA_ERR_SHAPE;
  if (axes->n_axes < 1 || axes->n_axes > SQA_MAX_ROPE_AXES || (axes->turns != 0 && axes->turns != 1) || (reinterpret_cast<uintptr_t>(axes->pos) & 3u))
    return false;
  int left[4] = {0, 0, 0, 0}, sum = 0;
  for (int i = 0; i < axes->n_axes; ++i) {
    if (axes->pairs[i] < 0 || axes->pairs[i] > 64) return false;
    left[i] = axes->pairs[i];
    sum += left[i];
  }
  if (sum != prep->rot_dim / 2) return false;
  out->pos = axes->pos; out->n = axes->n_axes;
  for (uint32_t& w : out->axis) w = 0;
  int at = 0;
  for (int i = 0; i < sum; ++i) {
    while (!left[at]) at = (at + 1) % axes->n_axes;
    out->axis[i / 16] |= (uint32_t)at << 2 * (i % 16);
    --left[at];
    if (axes->turns) at = (at + 1) % axes->n_axes;
  }
  *why = SQA_OK;
  return true;
}
// 0 where a caller's prep can be used for heads of D elements
inline sqa_status check_prep(const sqa_head_prep& prep, int D, const sqa_rope_axes* axes, int32_t new_pos, int T, const sqa_batch_opts* opts) {
  if (!aligned16(prep.q_weight) || !aligned16(prep.k_weight) || !aligned16(prep.rope)) return SQA_ERR_SHAPE;
  if ((prep.q_weight || prep.k_weight) && !(prep.eps >= 0.f)) return SQA_ERR_SHAPE;
  if (prep.rope && (prep.n_pos < 1 || prep.rot_dim < 16 || prep.rot_dim % 16 || prep.rot_dim > D || (prep.interleaved != 0 && prep.interleaved != 1) ||
                    (!axes && !(opts && opts->new_pos_seq) && !(opts && opts->prompt_len) && (int64_t)new_pos + T > prep.n_pos)))
    return SQA_ERR_SHAPE;
  return SQA_OK;
}

}  // namespace sqa
