// The gated delta rule (include/lm_ops.h).
//
//   S <- e^g S;  u = beta (v - S' k);  S <- S + k u';  y = scale S' q
#include <algorithm>

#include "delta_scale.h"
#include "lm_common.h"

namespace lstm_int {
namespace {

struct DeltaArgs {
  const void *q, *k, *v;
  const float *g, *beta;
  const int32_t *lengths;
  const float *state;
  float *new_state;
  void *y;
  int64_t q_stride[3], k_stride[3], v_stride[3], y_stride[3], g_stride[3], beta_stride[3];
  int T, B, Hk, Hv, Dk, Dv;
  int normalize;
  float scale;
};

constexpr float kNormEps = 1e-6f;

// Step by step: a wave has 4 kLanes columns of one head's state in registers, lane (r = lane / kLanes, c = lane % kLanes)
// the rows kRows r .. kRows r + kRows - 1 of columns 4 c .. 4 c + 3.  S' k and S' q are taken of the state before the step,
// in one reduction over the lanes, and y = e^g S' q + (k' q) u follows from them: a step waits for one reduction.  A single
// step is bound by the state's way in and out.
template <class T, int kLanes, int kRows>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a) {
  constexpr int kColumns = 4 * kLanes;
  const int lane = threadIdx.x & 63;
  const int tiles = (a.Dv + kColumns - 1) / kColumns;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)a.B * a.Hv * tiles) return;
  const int tile = (int)(item % tiles), h = (int)(item / tiles % a.Hv), b = (int)(item / tiles / a.Hv);
  const int hk = h / (a.Hv / a.Hk);
  const int r0 = lane / kLanes * kRows, c0 = tile * kColumns + lane % kLanes * 4;
  const int nr = max(0, min(kRows, a.Dk - r0)), nc = max(0, min(4, a.Dv - c0));
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;

  f32x4 S[kRows];
  const int64_t at = (((int64_t)b * a.Hv + h) * a.Dk + r0) * a.Dv + c0;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    S[i] = {0, 0, 0, 0};
    if (a.state && i < nr) {
      const float *p = a.state + at + (int64_t)i * a.Dv;
      if (nc == 4) S[i] = *reinterpret_cast<const f32x4_any *>(p);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < nc) S[i][j] = p[j];
    }
  }
  const T *q = static_cast<const T *>(a.q) + b * a.q_stride[1] + hk * a.q_stride[2] + r0;
  const T *k = static_cast<const T *>(a.k) + b * a.k_stride[1] + hk * a.k_stride[2] + r0;
  const T *v = static_cast<const T *>(a.v) + b * a.v_stride[1] + h * a.v_stride[2] + c0;
  T *y = static_cast<T *>(a.y) + b * a.y_stride[1] + h * a.y_stride[2] + c0;
  const float *g = a.g + b * a.g_stride[1] + h * a.g_stride[2], *beta = a.beta + b * a.beta_stride[1] + h * a.beta_stride[2];

  for (int t = 0; t < len; ++t) {
    float kf[kRows], qf[kRows], vf[4];
    {
      Raw8<T> rk[(kRows + 7) / 8], rq[(kRows + 7) / 8];
#pragma unroll
      for (int i = 0; i < kRows; i += 8) {
        rk[i / 8].load(k + i + t * a.k_stride[0], min(nr - i, kRows < 8 ? kRows : 8));
        rq[i / 8].load(q + i + t * a.q_stride[0], min(nr - i, kRows < 8 ? kRows : 8));
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) kf[i] = (float)rk[i / 8].e[i % 8], qf[i] = (float)rq[i / 8].e[i % 8];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) vf[j] = j < nc ? (float)v[t * a.v_stride[0] + j] : 0.0f;
    const float decay = expf(g[t * a.g_stride[0]]), bt = beta[t * a.beta_stride[0]];

    float kk = 0, qq = 0, kq = 0;
    f32x4 pk = {0, 0, 0, 0}, pq = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      kk = __builtin_fmaf(kf[i], kf[i], kk);
      qq = __builtin_fmaf(qf[i], qf[i], qq);
      kq = __builtin_fmaf(kf[i], qf[i], kq);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pk[j] = __builtin_fmaf(S[i][j], kf[i], pk[j]);
        pq[j] = __builtin_fmaf(S[i][j], qf[i], pq[j]);
      }
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      kk += __shfl_xor(kk, m);
      qq += __shfl_xor(qq, m);
      kq += __shfl_xor(kq, m);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pk[j] += __shfl_xor(pk[j], m);
        pq[j] += __shfl_xor(pq[j], m);
      }
    }
    const float nk = a.normalize ? 1.0f / sqrtf(kk + kNormEps) : 1.0f, nq = (a.normalize ? 1.0f / sqrtf(qq + kNormEps) : 1.0f) * a.scale;
    f32x4 u, o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = bt * (vf[j] - nk * (decay * pk[j]));
      o[j] = nq * (decay * pq[j] + nk * kq * u[j]);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) S[i][j] = __builtin_fmaf(nk * kf[i], u[j], decay * S[i][j]);
    if (lane < kLanes)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < nc) y[t * a.y_stride[0] + j] = (T)o[j];
  }
  if (!a.new_state) return;
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (i < nr) {
      float *p = a.new_state + at + (int64_t)i * a.Dv;
      if (nc == 4) *reinterpret_cast<f32x4_any *>(p) = S[i];
      else
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < nc) p[j] = S[i][j];
    }
}

template <class T, int kLanes, int kRows>
int launch_step(const DeltaArgs &a, hipStream_t s) {
  const int64_t items = (int64_t)a.B * a.Hv * ((a.Dv + 4 * kLanes - 1) / (4 * kLanes));
  return launch(delta_step_kernel<T, kLanes, kRows>, dim3((unsigned)((items + 3) / 4)), dim3(256), s, a);
}

template <class T>
int launch_step(const DeltaArgs &a, hipStream_t s) {
  // 32 columns to a wave, whole lines of memory, where that leaves enough waves and registers: one step of 64 x 16 heads of
  // 128 x 128 takes 37 us with 16 columns and 30 with 32, 4.5 TB/s of state
  const bool wide = (int64_t)a.B * a.Hv * ((a.Dv + 31) / 32) >= 1024;
  if (a.Dk <= 64) return wide ? launch_step<T, 8, 8>(a, s) : launch_step<T, 4, 4>(a, s);
  if (a.Dk <= 128) return wide ? launch_step<T, 8, 16>(a, s) : launch_step<T, 4, 8>(a, s);
  return launch_step<T, 4, 16>(a, s);
}

// ---------------------------------------------------------------------------------------------------------------------
// Sequences, kChunk steps at a time.  With c_i the sum of g over the chunk's steps up to i, and S the state before it:
//   A_ij = beta_i e^(c_i - c_j) k_i'k_j  (j < i),   X = (1 + A)^-1 diag(beta)
//   u = X (v - diag(e^c) K S),   y = diag(e^c) Q S + P u,   P_ij = e^(c_i - c_j) q_i'k_j  (j <= i)
//   S <- e^(c_last) S + K' diag(e^(c_last - c)) u
// X and P do not depend on the state: delta_prep_kernel computes them for all chunks side by side.  delta_scan_kernel
// carries the state from chunk to chunk.  One kernel for both would read K and Q once less, and would either repeat the first
// part for each group of value columns or have it wait in front of every chunk.
//
// Products run on the fp16 MFMA, whose products are exact and whose sums are float32.  A float32 operand is scaled by a power
// of two -- each row of a left operand and each column of a right one by its own -- and taken as two fp16 parts: 22 bits of
// each element, down to a floor of 2^-25, where the largest is just below 2^15 (kTop, delta_scale.h; a column of the state
// 2^5 .. 2^15, keys 2^2 .. 2^3).  Of the products of parts the one of the two low ones, 2^-22 of the others, is left out.  bf16
// and fp16 keys and queries are one part.  Two or three MFMAs for one product, where the float32 MFMA takes 16 times the time.
// (Three bf16 parts, 24 bits, which need no scales, took three to six, and more vector instructions: 777 ragged steps of 5 x 6
// float32 heads 141 us, 96 so.)
//
// So a sum is as near as one of float32 products relative to the row and the column that it is made of, not to each of their
// elements: one far below its row's or column's largest is known to 2^-39 of that largest, in a key to 2^-27, in the state to
// 2^-30 (2^-36 where its scale is new).  A right-hand side's column has the 32 steps of a chunk, so that a value 2^17 times as
// large as the others costs these the first of their bits, earlier steps too, and a value 2^39 times as large all of them; a
// column of the state has all key rows.  (With all largest at 1 .. 2, a value 10^6 times as large left 5 bits of the steps
// before it.)
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kChunk = 32;
constexpr int kHeadsOfGrid = 1 << 15;  // blockIdx.y of the first kernel, blockIdx.z counts on
constexpr int kMatrix = 2 * 2 * 64 * 4;  // words of X or P in the workspace: two tiles of 16 rows, two parts, 16 bytes a lane
// factors of a chunk's steps: of K S, Q S and u for the state; 1 / scale of the rows of X and P; e^c_last; scales of the
// rows of K and Q
enum { kFk, kFq, kFu, kFx, kFp, kFwhole, kFactors, kSk = kFactors, kSq, kAllFactors };
constexpr int kItemWords = 2 * kMatrix + kAllFactors * kChunk;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <class T> constexpr int kParts = sizeof(T) == 4 ? 2 : 1;  // fp16 parts of a scaled key or query

// The MFMA's operand order: lane (i = lane % 16, g = lane / 16) of a 16 x 32 operand has the columns 4 g .. 4 g + 3 and
// 16 + 4 g .. 16 + 4 g + 3 of row i.  A result (column lane % 16, rows 4 g .. 4 g + 3) of two 16-row tiles then is the
// other operand of the next product as it lies in the registers.
union Frag {
  u32x4 w;
  bf16x8 b;
  f16x8 h;
};

__device__ inline f32x4 mfma(const Frag &a, const Frag &b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0); }

__device__ inline uint32_t bits_of(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// the largest over the four lanes of a column
__device__ inline uint32_t over_column(uint32_t v) {
  // the swaps exchange rows of 16 lanes (halves of the wave) between two registers: of v and v, each with its neighbour
  auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(s[0], s[1]);
  s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(s[0], s[1]);
}
__device__ inline float inverse_of_power(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }

// -1 in a register, which the compiler does not see through: a - h is then one instruction that takes the half as it is
__device__ inline float minus_one() {
  float v;
  asm("v_mov_b32 %0, -1.0" : "=v"(v));
  return v;
}
__device__ inline void split2(float a, float b, uint32_t &hi, uint32_t &lo, float minus) {
  const f16x2 h = __builtin_convertvector((f32x2{a, b}), f16x2);
  const f16x2 l = __builtin_convertvector((f32x2{__builtin_fmaf((float)h[0], minus, a), __builtin_fmaf((float)h[1], minus, b)}), f16x2);
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, l);
}
// x = part 0 + part 1, for |x| < 65504
__device__ inline void split8(f32x4 a, f32x4 b, Frag out[2], float minus) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t hi, lo;
    split2(a[2 * i], a[2 * i + 1], hi, lo, minus);
    out[0].w[i] = hi, out[1].w[i] = lo;
    split2(b[2 * i], b[2 * i + 1], hi, lo, minus);
    out[0].w[2 + i] = hi, out[1].w[2 + i] = lo;
  }
}

// four neighbouring elements of a row
template <class T>
struct Raw4 {
  union {
    uint32_t w[sizeof(T)];
    T e[4];
  };
  __device__ void load(const T *p) {
    if constexpr (sizeof(T) == 4) {
      const u32x4 v = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else {
      const u32x2_any v = *reinterpret_cast<const u32x2_any *>(p);
      w[0] = v[0], w[1] = v[1];
    }
  }
  // loaded from column col - by: what belongs at col on, zeros behind it
  __device__ void shift(int by) {
    if (by == 0) return;
    Raw4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T v = (T)0.0f;
#pragma unroll
      for (int j = i + 1; j < 4; ++j)
        if (j == i + by) v = e[j];
      o.e[i] = v;
    }
    *this = o;
  }
  __device__ void keep(bool yes) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) w[i] = yes ? w[i] : 0u;
  }
};

// Rows are read from column min(col, width - 4) on; what was there becomes what is at col, zeros behind the width.  Only
// widths that are no multiple of four have anything to shift.
template <class T, int kN>
__device__ inline void place(Raw4<T> (&rows)[kN], int col, int width) {
  if (width % 4) {
#pragma unroll
    for (int r = 0; r < kN; ++r) rows[r].shift(col - min(col, width - 4));
  } else {
#pragma unroll
    for (int r = 0; r < kN; ++r) rows[r].keep(col < width);
  }
}

struct ChunkArgs {
  DeltaArgs d;
  uint32_t *items;  // [B Hv][chunks][kItemWords]
  int chunks, heads;  // heads: value heads that a wave of the first kernel prepares, all of one key head
};

__device__ inline int length_of(const DeltaArgs &a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T; }

// products of inputs with each other, unscaled: bf16 and fp16 on their own MFMA; float32 in three bf16 parts that add up to
// it exactly
template <class T>
struct Inputs {
  static constexpr int kN = sizeof(T) == 4 ? 3 : 1;
  Frag f[kN];
  __device__ void set(int half, const Raw4<T> &r) {
    if constexpr (kN == 1) {
      f[0].w[2 * half] = r.w[0], f[0].w[2 * half + 1] = r.w[1];
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float a = r.e[2 * i], b = r.e[2 * i + 1];
#pragma unroll
        for (int p = 0; p < kN; ++p) {
          f[p].w[2 * half + i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
          a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
          b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
      }
    }
  }
  static __device__ f32x4 product(const Inputs &a, const Inputs &b, f32x4 c) {
#pragma unroll
    for (int i = kN - 1; i >= 0; --i)
#pragma unroll
      for (int j = kN - 1; j >= 0; --j)
        if (i + j < 3) {
          if constexpr (__is_same(T, _Float16)) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.f[i].h, b.f[j].h, c, 0, 0, 0);
          else c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.f[i].b, b.f[j].b, c, 0, 0, 0);
        }
    return c;
  }
};

// One wave per chunk and value head, or all of a key head's: X, P and the factors of its steps.  Vector instructions and
// the chain of the substitution bound it: 64 chunks of 8 x 16 key heads of 128, two value heads each, 84 us, 39 %
// of whose cycles issue vector instructions.
template <class T, int kDk, bool kWhole>  // kWhole: key_dim = kDk
__global__ __launch_bounds__(64) void delta_prep_kernel(ChunkArgs a) {
  constexpr int kLd = 36, kBlocks = kDk / 32;
  const DeltaArgs &d = a.d;
  __shared__ __attribute__((aligned(16))) float mat[2][kChunk * kLd];  // A, then X; P
  __shared__ double sum_g[kChunk];
  __shared__ float rate[kChunk], norm_k[kChunk], norm_q[kChunk];
  const int lane = threadIdx.x, i = lane & 15, g = lane >> 4;
  const int chunk = blockIdx.x;
  const int item_at = blockIdx.z * kHeadsOfGrid + blockIdx.y;  // of B Hv / heads
  const int bh0 = item_at * a.heads;
  if (bh0 >= d.B * d.Hv) return;
  const int b = bh0 / d.Hv, hk = bh0 % d.Hv / (d.Hv / d.Hk);
  const int t0 = chunk * kChunk, left = length_of(d, b) - t0;  // steps of the row from here on
  if (left <= 0) return;
  // rows behind the last step are that step again: their rate of writing is zero
  const T *kp = static_cast<const T *>(d.k) + b * d.k_stride[1] + hk * d.k_stride[2];
  const T *qp = static_cast<const T *>(d.q) + b * d.q_stride[1] + hk * d.q_stride[2];
  f32x4 kk[3] = {}, qk[3] = {};  // tiles (0,0), (1,0), (1,1)
  float sk[2] = {0, 0}, sq[2] = {0, 0};
  uint32_t mk[2] = {0, 0}, mq[2] = {0, 0};
  constexpr int kAtOnce = kBlocks * sizeof(T) > 4 ? 4 / sizeof(T) : kBlocks;
#pragma unroll
  for (int kb0 = 0; kb0 < kBlocks; kb0 += kAtOnce) {
    Raw4<T> rk[kAtOnce][2][2], rq[kAtOnce][2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int64_t t = t0 + min(16 * m + i, left - 1);
      const T *kr = kp + t * d.k_stride[0], *qr = qp + t * d.q_stride[0];
#pragma unroll
      for (int kb = 0; kb < kAtOnce; ++kb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int at = (kb0 + kb) * 32 + 16 * e, col = kWhole ? at + 4 * g : min(at + 4 * g, d.Dk - 4);
          rk[kb][m][e].load(kr + col);
          rq[kb][m][e].load(qr + col);
        }
    }
#pragma unroll
    for (int kb = 0; kb < kAtOnce; ++kb) {
      Inputs<T> kf[2], qf[2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = (kb0 + kb) * 32 + 16 * e + 4 * g;
          if constexpr (!kWhole) {
            place(reinterpret_cast<Raw4<T>(&)[1]>(rk[kb][m][e]), col, d.Dk);
            place(reinterpret_cast<Raw4<T>(&)[1]>(rq[kb][m][e]), col, d.Dk);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = (float)rk[kb][m][e].e[j], y = (float)rq[kb][m][e].e[j];
            sk[m] = __builtin_fmaf(x, x, sk[m]);
            sq[m] = __builtin_fmaf(y, y, sq[m]);
            mk[m] = max(mk[m], bits_of(x));
            mq[m] = max(mq[m], bits_of(y));
          }
          kf[m].set(e, rk[kb][m][e]);
          qf[m].set(e, rq[kb][m][e]);
        }
      kk[0] = Inputs<T>::product(kf[0], kf[0], kk[0]);
      qk[0] = Inputs<T>::product(qf[0], kf[0], qk[0]);
      kk[1] = Inputs<T>::product(kf[1], kf[0], kk[1]);
      qk[1] = Inputs<T>::product(qf[1], kf[0], qk[1]);
      kk[2] = Inputs<T>::product(kf[1], kf[1], kk[2]);
      qk[2] = Inputs<T>::product(qf[1], kf[1], qk[2]);
    }
  }
  float inv_sk[2], inv_sq[2], up_k[2], up_q[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    sk[m] += __shfl_xor(sk[m], 16);
    sk[m] += __shfl_xor(sk[m], 32);
    sq[m] += __shfl_xor(sq[m], 16);
    sq[m] += __shfl_xor(sq[m], 32);
    const Scale ks = scale_of<kKeyTop>(over_column(mk[m])), qs = scale_of<kTop>(over_column(mq[m]));
    inv_sk[m] = ks.down, inv_sq[m] = qs.down;
    if (g == 0) {
      norm_k[16 * m + i] = d.normalize ? 1.0f / sqrtf(sk[m] + kNormEps) : 1.0f;
      norm_q[16 * m + i] = (d.normalize ? 1.0f / sqrtf(sq[m] + kNormEps) : 1.0f) * d.scale;
    }
    up_k[m] = ks.up, up_q[m] = qs.up;
  }
  // what follows differs from value head to value head
#pragma unroll 1
  for (int n = 0; n < a.heads; ++n) {
    // the lane again, from nothing: places in LDS that are computed ahead of the loop would take half of the registers
    int lane = threadIdx.x;
    asm volatile("" : "+v"(lane));
    const int i = lane & 15, g = lane >> 4;
    const int bh = bh0 + n, h = bh % d.Hv;
    uint32_t *item = a.items + ((int64_t)bh * a.chunks + chunk) * kItemWords;
    float *factors = reinterpret_cast<float *>(item + 2 * kMatrix);
    double c = 0;
    float bt = 0;
    if ((lane & 31) < left) {
      const int64_t t = t0 + (lane & 31);
      const float gv = d.g[b * d.g_stride[1] + h * d.g_stride[2] + t * d.g_stride[0]];
      c = gv < -1000.0f ? -1000.0 : (double)gv;  // e^-1000 is zero; the sum stays a number
      bt = d.beta[b * d.beta_stride[1] + h * d.beta_stride[2] + t * d.beta_stride[0]];
    }
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      union { double v; int w[2]; } x, y;
      x.v = c;
      y.w[0] = __shfl_up(x.w[0], m, 32);
      y.w[1] = __shfl_up(x.w[1], m, 32);
      if ((lane & 31) >= m) c += y.v;
    }
    if (lane < 32) sum_g[lane] = c, rate[lane] = bt;
    if (g == 0)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        factors[kSk * kChunk + 16 * m + i] = up_k[m];
        factors[kSq * kChunk + 16 * m + i] = up_q[m];
      }
    __syncthreads();
    if (g < 2) {  // lane = step
      const double end = sum_g[kChunk - 1];
      const float e = expf((float)c), dk = g ? inv_sk[1] : inv_sk[0], dq = g ? inv_sq[1] : inv_sq[0];
      factors[kFk * kChunk + lane] = e * norm_k[lane] * dk;
      factors[kFq * kChunk + lane] = e * norm_q[lane] * dq;
      factors[kFu * kChunk + lane] = expf((float)(end - c)) * norm_k[lane] * dk;
      factors[kFwhole * kChunk + lane] = expf((float)end);
    }
#pragma unroll
    for (int tile = 0; tile < 3; ++tile) {
      const int tj = (tile == 2 ? 16 : 0) + i;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int ti = (tile ? 16 : 0) + 4 * g + r;
        const float e = ti >= tj ? expf((float)(sum_g[ti] - sum_g[tj])) * norm_k[tj] : 0.0f;
        mat[0][ti * kLd + tj] = ti > tj ? e * kk[tile][r] * norm_k[ti] * rate[ti] : 0.0f;
        mat[1][ti * kLd + tj] = ti >= tj ? e * qk[tile][r] * norm_q[ti] : 0.0f;
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) mat[1][(4 * g + r) * kLd + 16 + i] = 0;
    __syncthreads();
    // (1 + A)^-1: the 16 x 16 blocks on the diagonal by substitution, a lane a column; then the one below them
    {
      const int blk = g & 1;
      const float *A = mat[0] + 16 * blk * (kLd + 1);
      float x[16];
      int from = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float s0 = r == i ? 1.0f : 0.0f, s1 = 0;
#pragma unroll
        for (int m = 0; m < r; m += 4) {
          const f32x4 row = *reinterpret_cast<const f32x4 *>(A + from + r * kLd + m);
#pragma unroll
          for (int n = 0; n < 4; ++n)
            if (m + n < r) (n % 2 ? s1 : s0) = __builtin_fmaf(-row[n], x[m + n], n % 2 ? s1 : s0);
        }
        x[r] = s0 + s1;
        // the next four rows of A are read behind this one, not all sixteen at once: half of the registers
        if (r % 4 == 3) asm volatile("" : "+v"(from), "+v"(x[r]));
      }
      __syncthreads();
      if (g < 2)
#pragma unroll
        for (int r = 0; r < 16; ++r) mat[0][(16 * blk + r) * kLd + 16 * blk + i] = x[r];
    }
    __syncthreads();
    {
      f32x4 m1 = {0, 0, 0, 0}, m2 = {0, 0, 0, 0};
      const f32x4 below = *reinterpret_cast<const f32x4 *>(&mat[0][(16 + i) * kLd + 4 * g]);
      const f32x4 last = *reinterpret_cast<const f32x4 *>(&mat[0][(16 + i) * kLd + 16 + 4 * g]);
#pragma unroll
      for (int r = 0; r < 4; ++r) m1 = __builtin_amdgcn_mfma_f32_16x16x4f32(below[r], mat[0][(4 * g + r) * kLd + i], m1, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) m2 = __builtin_amdgcn_mfma_f32_16x16x4f32(last[r], m1[r], m2, 0, 0, 0);
      __syncthreads();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        mat[0][(16 + 4 * g + r) * kLd + i] = -m2[r];
        mat[0][(4 * g + r) * kLd + 16 + i] = 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f32x4 v[2];
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          v[e] = *reinterpret_cast<const f32x4 *>(&mat[w][(16 * m + i) * kLd + 16 * e + 4 * g]);
          if (w == 0) v[e] *= *reinterpret_cast<const f32x4 *>(&rate[16 * e + 4 * g]);
#pragma unroll
          for (int j = 0; j < 4; ++j) most = max(most, bits_of(v[e][j]));
        }
        const Scale s = scale_of<kTop>(over_column(most));  // lanes i, i + 16, ...: the row's
        Frag f[2];
        split8(v[0] * s.up, v[1] * s.up, f, minus_one());
#pragma unroll
        for (int p = 0; p < 2; ++p) *reinterpret_cast<u32x4 *>(item + w * kMatrix + ((m * 2 + p) * 64 + lane) * 4) = f[p].w;
        if (g == 0) factors[(w ? kFp : kFx) * kChunk + 16 * m + i] = s.down;
      }
    __syncthreads();  // mat and the sums are the next head's
  }
}

// A workgroup carries kMain * kCols * 16 columns of one head's state through the sequence: kMain waves have 16 kCols columns
// each, in the registers, for good; four more ("loaders") bring the next chunk's operands into LDS meanwhile, in parts and
// in the MFMA's order, with the chunk after it already requested.  kBuffers = 1 where two do not fit.
//
// With a workgroup on each compute unit it is bound by the issue of vector instructions: 1060 to a SIMD and chunk (parts of
// the state and their scales, the loaders' transposition), 53 % of all cycles, 67 % with the others; LDS 18 %, MFMA 24 %.
// 2048 steps of 8 x 32 heads of 128 x 128: 221 us, 3.5 us a chunk.  With fewer it is bound by the chain of a chunk, K S ->
// u -> S: 1.5 us for 32 steps, for which the scale of what is added to the state comes in front of P u (1.6 behind it).
template <class T, int kDk, int kMain, int kCols>
struct Scan {
  static constexpr int kP = kParts<T>, kBlocks = kDk / 32, kLoaders = 4, kColumns = 16 * kMain * kCols;
  static constexpr int kThreads = (kMain + kLoaders) * 64;
  struct Buffer {
    u32x4 k[2][kBlocks][kP][64], q[2][kBlocks][kP][64];  // rows of steps, by key column
    u32x4 kt[kDk / 16][kP][64];                          // rows of key columns, by step
    u32x4 x[2][2][64], p[2][2][64];
    u32x4 vt[kColumns / 16][sizeof(T) / 2][64];          // rows of value columns, by step: as they are
    float factor[kFactors][kChunk];
  };
  static constexpr int kBuffers = 2 * sizeof(Buffer) <= 160 * 1024 ? 2 : 1;
};

// Where lane (i, g)'s operand lies among the 64 of k, q, kt and vt: the writers, which have four rows of one g each, then
// meet in no bank, and a reader's order does not matter.
__device__ inline int slot_of(int i, int g) { return (i ^ g) + 16 * g; }

// column j of four rows of two words (four 16-bit elements each), as two words
__device__ inline u32x2_any column_of(const uint32_t w[4][2], int j) {
  const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
  return u32x2_any{__builtin_amdgcn_perm(w[1][j / 2], w[0][j / 2], pick), __builtin_amdgcn_perm(w[3][j / 2], w[2][j / 2], pick)};
}
__device__ inline void put8(u32x4 &to, int half, u32x2_any v) { reinterpret_cast<uint64_t *>(&to)[half] = __builtin_bit_cast(uint64_t, v); }

// four elements times a scale in kP fp16 parts, as two words each
template <int kP, class T>
__device__ inline void scaled_parts(const Raw4<T> &r, float s, uint32_t out[kP][2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float a = (float)r.e[2 * i] * s, b = (float)r.e[2 * i + 1] * s;
    if constexpr (kP == 1) out[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
    else split2(a, b, out[0][i], out[1][i], minus_one());
  }
}

template <class T, int kDk, int kMain, int kCols>
__device__ inline void scan_load(const ChunkArgs &a, typename Scan<T, kDk, kMain, kCols>::Buffer *buffer, int b, int h, int len, int chunks) {
  using S = Scan<T, kDk, kMain, kCols>;
  constexpr int kP = S::kP, kHalfWords = sizeof(T) / 2;
  constexpr int kKeyBlocks = 8 * (kDk / 4), kEach = (kKeyBlocks + 255) / 256, kValueBlocks = 8 * (S::kColumns / 4);
  const DeltaArgs &d = a.d;
  const int tid = threadIdx.x - kMain * 64, hk = h / (d.Hv / d.Hk);
  const T *kp = static_cast<const T *>(d.k) + b * d.k_stride[1] + hk * d.k_stride[2];
  const T *qp = static_cast<const T *>(d.q) + b * d.q_stride[1] + hk * d.q_stride[2];
  const T *vp = static_cast<const T *>(d.v) + b * d.v_stride[1] + h * d.v_stride[2];
  const uint32_t *item = a.items + (int64_t)(b * d.Hv + h) * a.chunks * kItemWords;
  // blocks of 4 steps x 4 columns: 4 x 16 of them to a wave, the steps' half above that, then the columns
  const int step = (tid / 64 % 2 * 4 + tid % 4) * 4;
  auto col_of = [&](int n) { return ((tid + 256 * n) / 128 * 16 + tid / 4 % 16) * 4; };
  // fewer than 16 blocks of value columns: the steps' half above them
  constexpr int kVc = S::kColumns / 4 < 16 ? S::kColumns / 4 : 16;
  const int v_step = (tid / (4 * kVc) % 2 * 4 + tid % 4) * 4, v_col = (tid / (8 * kVc) * kVc + tid / 4 % kVc) * 4;
  const int v_from = blockIdx.y * S::kColumns + v_col;
  struct Stage {
    Raw4<T> k[kEach][4], q[kEach][4], v[4];
    u32x4 m[2];
    f32x4 sk, sq;
    float f;
  };
  // where the first row of a block is in chunk 0, and where the sequence's last row is
  const T *k_at[kEach], *q_at[kEach], *k_end[kEach], *q_end[kEach];
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int col = min(col_of(n), d.Dk - 4);
    k_at[n] = kp + step * d.k_stride[0] + col;
    q_at[n] = qp + step * d.q_stride[0] + col;
    k_end[n] = kp + (int64_t)(len - 1) * d.k_stride[0] + col;
    q_end[n] = qp + (int64_t)(len - 1) * d.q_stride[0] + col;
  }
  const T *v_at = vp + v_step * d.v_stride[0] + min(v_from, d.Dv - 4), *v_end = vp + (int64_t)(len - 1) * d.v_stride[0] + min(v_from, d.Dv - 4);
  // rows behind the last step are that step again: one path for all chunks, so that nothing waits for a load but its use
  auto fetch = [&](Stage &s, int c) {
    c = min(c, chunks - 1);
    const int64_t t = (int64_t)c * kChunk;
    const int left = len - 1 - c * kChunk;
    const T *k_row[kEach], *q_row[kEach], *v_row = v_at + t * d.v_stride[0];
#pragma unroll
    for (int n = 0; n < kEach; ++n) k_row[n] = k_at[n] + t * d.k_stride[0], q_row[n] = q_at[n] + t * d.q_stride[0];
    // a selected address, not a branch around two loads
    auto either = [](bool yes, const T *a, const T *b) {
      uint64_t at = reinterpret_cast<uint64_t>(a);
      asm volatile("" : "+v"(at));
      at = yes ? at : reinterpret_cast<uint64_t>(b);
      return (const T *)reinterpret_cast<const __attribute__((address_space(1))) T *>(at);
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool in = step + r <= left;
#pragma unroll
      for (int n = 0; n < kEach; ++n) {
        s.k[n][r].load(either(in, k_row[n] + r * d.k_stride[0], k_end[n]));
        s.q[n][r].load(either(in, q_row[n] + r * d.q_stride[0], q_end[n]));
      }
      s.v[r].load(either(v_step + r <= left, v_row + r * d.v_stride[0], v_end));
    }
    const uint32_t *it = item + (int64_t)c * kItemWords;
    const float *factors = reinterpret_cast<const float *>(it + 2 * kMatrix);
    s.m[0] = *reinterpret_cast<const u32x4 *>(it + tid * 4);
    s.m[1] = *reinterpret_cast<const u32x4 *>(it + kMatrix + tid * 4);
    s.sk = *reinterpret_cast<const f32x4 *>(factors + kSk * kChunk + step);
    s.sq = *reinterpret_cast<const f32x4 *>(factors + kSq * kChunk + step);
    s.f = factors[tid % (kFactors * kChunk)];
  };
  auto put = [&](Stage &s, typename S::Buffer &o) {
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      const int col = col_of(n), m = step / 16, kb = col / 32, kg = col % 16 / 4, half = col % 32 / 16;
      if (col >= kDk) break;
      if (d.Dk < kDk) {
        place(s.q[n], col, d.Dk);
        place(s.k[n], col, d.Dk);
      }
      uint32_t w[kP][4][2];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint32_t v[kP][2];
        scaled_parts<kP>(s.q[n][r], s.sq[r], v);
#pragma unroll
        for (int p = 0; p < kP; ++p) put8(o.q[m][kb][p][slot_of(step % 16 + r, kg)], half, u32x2_any{v[p][0], v[p][1]});
        scaled_parts<kP>(s.k[n][r], s.sk[r], v);
#pragma unroll
        for (int p = 0; p < kP; ++p) {
          put8(o.k[m][kb][p][slot_of(step % 16 + r, kg)], half, u32x2_any{v[p][0], v[p][1]});
          w[p][r][0] = v[p][0], w[p][r][1] = v[p][1];
        }
      }
#pragma unroll
      for (int p = 0; p < kP; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) put8(o.kt[col / 16][p][slot_of(col % 16 + j, step % 16 / 4)], m, column_of(w[p], j));
    }
    if (kValueBlocks >= 256 || tid < kValueBlocks) {
      u32x4 *to = &o.vt[v_col / 16][0][0];
      if (d.Dv % 4) place(s.v, v_from, d.Dv);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = slot_of(v_col % 16 + j, v_step % 16 / 4);
        if constexpr (kHalfWords == 1) {
          uint32_t w[4][2];
#pragma unroll
          for (int r = 0; r < 4; ++r) w[r][0] = s.v[r].w[0], w[r][1] = s.v[r].w[1];
          put8(to[slot], v_step / 16, column_of(w, j));
        } else {
          to[v_step / 16 * 64 + slot] = u32x4{s.v[0].w[j], s.v[1].w[j], s.v[2].w[j], s.v[3].w[j]};
        }
      }
    }
    (&o.x[0][0][0])[tid] = s.m[0];
    (&o.p[0][0][0])[tid] = s.m[1];
    if (tid < kFactors * kChunk) o.factor[tid / 32][tid % 32] = s.f;
  };
  if (chunks == 0) {
    if constexpr (S::kBuffers == 2) __syncthreads();
    return;
  }
  if constexpr (S::kBuffers == 2) {
    Stage even, odd;
    fetch(even, 0);
    fetch(odd, 1);
    put(even, buffer[0]);
    fetch(even, 2);
    __syncthreads();
    // Two chunks at a time, without a branch: behind the end the last chunk comes again, into the buffer that nobody reads.
    // (With the branches, waits for one stage's loads became waits for the other's too.)
    for (int c = 0; c < chunks; c += 2) {  // main is at chunk c
      put(odd, buffer[1]);
      fetch(odd, c + 3);
      __syncthreads();
      put(even, buffer[0]);
      fetch(even, c + 4);
      __syncthreads();
    }
  } else {
    Stage s;
    fetch(s, 0);
    for (int c = 0; c < chunks; ++c) {
      put(s, buffer[0]);
      fetch(s, c + 1);
      __syncthreads();
      __syncthreads();
    }
  }
}

// c[n] += a[n] b over the parts that matter, the smallest products first, the chains side by side
template <int kPa, int kN>
__device__ inline void mfma_side_by_side(const Frag (*a)[kPa], const Frag *b, f32x4 **c) {
#pragma unroll
  for (int i = kPa - 1; i >= 0; --i)
#pragma unroll
    for (int j = 1; j >= 0; --j)
      if (i + j <= 1)
#pragma unroll
        for (int n = 0; n < kN; ++n) *c[n] = mfma(a[n][i], b[j], *c[n]);
}

// the largest |x| of eight and m; a NaN is passed over, and comes out of the products by itself
__device__ inline float largest8(f32x4 a, f32x4 b, float m) {
#pragma unroll
  for (int r = 0; r < 4; ++r) m = __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(a[r]), __builtin_fabsf(b[r])), m);
  return m;
}
__device__ inline uint32_t over_column(float m) { return over_column(__float_as_uint(m)); }

// bits of the largest of a column: what the products take as it is
constexpr uint32_t kLow = 0x42000000u, kHigh = 0x47000000u, kInf = 0x7f800000u;  // 2^5, 2^15, infinity
__device__ inline bool in_range(uint32_t bits) { return bits - kLow < kHigh - kLow; }

template <class T, int kDk, int kMain, int kCols>
__global__ __launch_bounds__((kMain + 4) * 64) void delta_scan_kernel(ChunkArgs a) {
  using S = Scan<T, kDk, kMain, kCols>;
  constexpr int kP = S::kP, kBlocks = S::kBlocks, kBuffers = S::kBuffers, kTiles = kDk / 16;
  const DeltaArgs &d = a.d;
  __shared__ typename S::Buffer buffer[kBuffers];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.x, b = bh / d.Hv, h = bh % d.Hv;
  const int len = length_of(d, b), chunks = (len + kChunk - 1) / kChunk;
  if (wave >= kMain) return scan_load<T, kDk, kMain, kCols>(a, buffer, b, h, len, chunks);

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, slot = slot_of(i, g);
  const float minus = minus_one();
  int col[kCols];
  f32x4 st[kCols][kTiles];  // the state times its column's scale, which changes where the column leaves 2^5 .. 2^15
  float up[kCols];
  const int64_t head = (int64_t)bh * d.Dk * d.Dv;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    up[n] = 1;
    col[n] = ((blockIdx.y * kMain + wave) * kCols + n) * 16 + i;
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * m + 4 * g + r;
        st[n][m][r] = d.state && row < d.Dk && col[n] < d.Dv ? d.state[head + (int64_t)row * d.Dv + col[n]] : 0.0f;
      }
  }
  T *y = static_cast<T *>(d.y) + b * d.y_stride[1] + h * d.y_stride[2];
  if constexpr (kBuffers == 2) __syncthreads();
  for (int c = 0; c < chunks; ++c) {
    if constexpr (kBuffers == 1) __syncthreads();
    const typename S::Buffer &o = buffer[kBuffers == 2 ? c & 1 : 0];
    uint32_t most[kCols];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      float top = 0;
#pragma unroll
      for (int m = 0; m < kTiles; m += 2) top = largest8(st[n][m], st[n][m + 1], top);
      most[n] = over_column(top);
      const bool fine = in_range(most[n]) || most[n] == 0;
      if (__any(!fine)) {
        const int e = exponent_of(__float_as_uint(up[n])), next = fine || most[n] >= kInf ? e : next_exponent(e, most[n], 0);
        const float by = power_of_two(min(next - e, 126));  // the rest next time
#pragma unroll
        for (int m = 0; m < kTiles; ++m) st[n][m] *= by;
        up[n] *= by;
        most[n] = most[n] < kInf ? __float_as_uint(__uint_as_float(most[n]) * by) : most[n];
      }
    }
    f32x4 rhs[kCols][2], out[kCols][2];
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
      for (int m = 0; m < 2; ++m) rhs[n][m] = out[n][m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      Frag f[4][kP];
#pragma unroll
      for (int p = 0; p < kP; ++p) {
        f[0][p].w = o.k[0][kb][p][slot], f[1][p].w = o.q[0][kb][p][slot];
        f[2][p].w = o.k[1][kb][p][slot], f[3][p].w = o.q[1][kb][p][slot];
      }
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        Frag s[2];
        split8(st[n][2 * kb], st[n][2 * kb + 1], s, minus);
        f32x4 *to[4] = {&rhs[n][0], &out[n][0], &rhs[n][1], &out[n][1]};
        mfma_side_by_side<kP, 4>(f, s, to);
      }
    }
    auto factor = [&](int f, int m) { return *reinterpret_cast<const f32x4 *>(&o.factor[f][16 * m + 4 * g]); };
    Frag part[2], x[2][2], p[2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int e = 0; e < 2; ++e) x[m][e].w = o.x[m][e][lane], p[m][e].w = o.p[m][e][lane];
    const float whole = o.factor[kFwhole][0];
    f32x4 u[kCols][2];
    Frag added[kCols][2];
    float keep[kCols];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      const float down = inverse_of_power(up[n]);
      Raw8<T> v;
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e) v.w[e] = o.vt[wave * kCols + n][e][slot];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const f32x4 fk = factor(kFk, m) * down, fq = factor(kFq, m) * down;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          rhs[n][m][r] = __builtin_fmaf(-fk[r], rhs[n][m][r], (float)v.e[4 * m + r]);
          out[n][m][r] *= fq[r];
        }
      }
      // u
      Scale s = scale_of<kTop>(over_column(largest8(rhs[n][0], rhs[n][1], 0.0f)));
      split8(rhs[n][0] * s.up, rhs[n][1] * s.up, part, minus);
      u[n][0] = u[n][1] = f32x4{0, 0, 0, 0};
      f32x4 *to[2] = {&u[n][0], &u[n][1]};
      mfma_side_by_side<2, 2>(x, part, to);
#pragma unroll
      for (int m = 0; m < 2; ++m) u[n][m] *= factor(kFx, m) * s.down;
      // What is added to the state has its scale, or changes it.  The scale is chosen by the largest of what is added and of what is
      // kept after the decay, and only then applied, to the one, and with the decay in one factor to the other: neither
      // a scale of a column that has faded nor a decay to all but nothing leads out of the range of a float.
      {
        const f32x4 w[2] = {u[n][0] * factor(kFu, 0), u[n][1] * factor(kFu, 1)};
        const uint32_t wm = over_column(largest8(w[0], w[1], 0.0f)), ws = __float_as_uint(__uint_as_float(wm) * (up[n] * (1 << kKeyTop)));
        const uint32_t kept = __float_as_uint(__uint_as_float(most[n]) * whole);
        const bool fine = in_range(max(ws, kept)) || (wm | kept) == 0;
        keep[n] = whole;
        if (__any(!fine)) {
          const bool as_it_is = fine || wm >= kInf || kept >= kInf;  // no scale would help
          const int e = exponent_of(__float_as_uint(up[n])), next = as_it_is ? e : next_exponent(e, kept, wm);
          keep[n] = as_it_is ? whole : scaled_whole(whole, next - e);
          up[n] = power_of_two(next);
        }
        split8(w[0] * up[n], w[1] * up[n], added[n], minus);
      }
      // P u
      s = scale_of<kTop>(over_column(largest8(u[n][0], u[n][1], 0.0f)));
      split8(u[n][0] * s.up, u[n][1] * s.up, part, minus);
      f32x4 pu[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      f32x4 *to2[2] = {&pu[0], &pu[1]};
      mfma_side_by_side<2, 2>(p, part, to2);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const f32x4 fp = factor(kFp, m) * s.down;
#pragma unroll
        for (int r = 0; r < 4; ++r) out[n][m][r] = __builtin_fmaf(pu[m][r], fp[r], out[n][m][r]);
      }
    }
#pragma unroll
    for (int m = 0; m < kTiles; m += 2) {
      Frag f[2][kP];
#pragma unroll
      for (int e = 0; e < kP; ++e) f[0][e].w = o.kt[m][e][slot], f[1][e].w = o.kt[m + 1][e][slot];
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        st[n][m] *= keep[n], st[n][m + 1] *= keep[n];
        f32x4 *to[2] = {&st[n][m], &st[n][m + 1]};
        mfma_side_by_side<kP, 2>(f, added[n], to);
      }
    }
    T *yc = y + (int64_t)(c * kChunk + 4 * g) * d.y_stride[0];
    const int left = len - c * kChunk - 4 * g;  // steps from this lane's first on
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      if (col[n] >= d.Dv) continue;
      if (c * kChunk + kChunk <= len) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r) yc[(int64_t)(16 * m + r) * d.y_stride[0] + col[n]] = (T)out[n][m][r];
      } else {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * m + r < left) yc[(int64_t)(16 * m + r) * d.y_stride[0] + col[n]] = (T)out[n][m][r];
      }
    }
    __syncthreads();
  }
  if constexpr (kBuffers == 2)
    if (chunks % 2) __syncthreads();  // the loaders go two chunks at a time
  if (!d.new_state) return;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    const float down = inverse_of_power(up[n]);
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * m + 4 * g + r;
        if (row < d.Dk && col[n] < d.Dv) d.new_state[head + (int64_t)row * d.Dv + col[n]] = st[n][m][r] * down;
      }
  }
}

template <class T, int kDk, int kMain, int kCols>
int launch_scan(const ChunkArgs &a, hipStream_t s) {
  const dim3 grid(a.d.B * a.d.Hv, (a.d.Dv + 16 * kMain * kCols - 1) / (16 * kMain * kCols));
  return launch(delta_scan_kernel<T, kDk, kMain, kCols>, grid, dim3((kMain + 4) * 64), s, a);
}

// As many columns to a workgroup as leave one for each compute unit: their operands come from memory once.  (2048 steps of
// 8 x 32 heads, 128 columns in four waves of 32, 64 columns in four of 16: 335 and 396 us; float32 426 and 532.  Eight waves
// of 16 were between the two.)
template <class T, int kDk>
int launch_scan(const ChunkArgs &a, hipStream_t s) {
  const int64_t heads = (int64_t)a.d.B * a.d.Hv;
  auto groups = [&](int columns) { return heads * ((a.d.Dv + columns - 1) / columns); };
  // 256 key columns: the state of 32 value columns and their products' operands are more than a wave has registers, and
  // in float32 LDS holds a chunk beside 16 value columns only
  if constexpr (kDk <= 128)
    if (groups(128) >= 256) return launch_scan<T, kDk, 4, 2>(a, s);
  if constexpr (kDk <= 128 || sizeof(T) == 2) {
    if (groups(64) >= 256) return launch_scan<T, kDk, 4, 1>(a, s);
    if (groups(32) >= 256) return launch_scan<T, kDk, 2, 1>(a, s);
  }
  return launch_scan<T, kDk, 1, 1>(a, s);
}

template <class T, int kDk>
int launch_chunks(const ChunkArgs &a, hipStream_t s) {
  const int items = a.d.B * a.d.Hv / a.heads;
  const dim3 grid(a.chunks, std::min(items, kHeadsOfGrid), (items + kHeadsOfGrid - 1) / kHeadsOfGrid);
  const int rc = a.d.Dk == kDk ? launch(delta_prep_kernel<T, kDk, true>, grid, dim3(64), s, a)
                               : launch(delta_prep_kernel<T, kDk, false>, grid, dim3(64), s, a);
  return rc != LSTM_INT_OK ? rc : launch_scan<T, kDk>(a, s);
}

template <class T>
int launch_chunks(const ChunkArgs &a, hipStream_t s) {
  return a.d.Dk <= 64 ? launch_chunks<T, 64>(a, s) : a.d.Dk <= 128 ? launch_chunks<T, 128>(a, s) : launch_chunks<T, 256>(a, s);
}

// A chunk takes the time of some twelve steps of few heads, sixteen of many: 16 heads of 128 x 128, 8, 12 and 16 steps: 17, 23
// and 29 us step by step, 20, 20 and 21 in one chunk; with 64 rows 57, 74 and 90, and 92, 93 and 93.  The loads of a chunk take
// four columns at once.
bool in_chunks(const delta_rule_args *p) { return p->steps >= 12 && p->key_dim >= 4 && p->value_dim >= 4; }

int check(const delta_rule_args *p) {
  if (!p || p->steps < 0 || p->batch < 0 || p->key_heads < 1 || p->value_heads < 1 || p->value_heads % p->key_heads || p->key_dim < 1 ||
      p->value_dim < 1 || !lm_type_bytes(p->dtype) || (p->normalize != 0 && p->normalize != 1))
    return LSTM_INT_E_INVALID_ARG;
  if (!__builtin_isfinite(p->scale)) return LSTM_INT_E_BAD_RANGE;
  if (p->key_dim > 256 || p->value_dim > 256 || (int64_t)p->batch * p->value_heads > 1 << 20 || p->steps > 1 << 24) return LSTM_INT_E_UNSUPPORTED;
  return LSTM_INT_OK;
}

}  // namespace
}  // namespace lstm_int

using namespace lstm_int;

extern "C" {

size_t delta_rule_workspace_bytes(const delta_rule_args *p) {
  if (check(p) != LSTM_INT_OK || !in_chunks(p)) return 0;
  return (size_t)p->batch * p->value_heads * ((p->steps + kChunk - 1) / kChunk) * kItemWords * sizeof(uint32_t);
}

int delta_rule_forward(int32_t device, const delta_rule_args *p, const void *q, const void *k, const void *v, const float *g,
                       const float *beta, const int32_t *lengths, const float *state, float *new_state, void *y, void *workspace,
                       size_t workspace_bytes, void *hip_stream) {
  const int rc = check(p);
  if (rc != LSTM_INT_OK) return rc;
  if (device < 0) return LSTM_INT_E_INVALID_ARG;
  if (p->batch == 0 || (p->steps == 0 && !new_state)) return LSTM_INT_OK;
  if (p->steps > 0 && (!q || !k || !v || !g || !beta || !y)) return LSTM_INT_E_INVALID_ARG;
  const size_t need = delta_rule_workspace_bytes(p);
  if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255))) return LSTM_INT_E_WORKSPACE;
  const int64_t extents[3] = {p->steps, p->batch, p->value_heads};
  for (int i = 0; i < 3; ++i)  // y: neighbours would be in each other's place
    if (p->steps && extents[i] > 1 && p->y_stride[i] < p->value_dim && p->y_stride[i] > -p->value_dim) return LSTM_INT_E_INVALID_ARG;
  DeltaArgs a{};
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.lengths = lengths; a.state = state; a.new_state = new_state; a.y = y;
  for (int i = 0; i < 3; ++i) {
    a.q_stride[i] = p->q_stride[i]; a.k_stride[i] = p->k_stride[i]; a.v_stride[i] = p->v_stride[i];
    a.y_stride[i] = p->y_stride[i]; a.g_stride[i] = p->g_stride[i]; a.beta_stride[i] = p->beta_stride[i];
  }
  a.T = p->steps; a.B = p->batch; a.Hk = p->key_heads; a.Hv = p->value_heads; a.Dk = p->key_dim; a.Dv = p->value_dim;
  a.normalize = p->normalize; a.scale = (float)p->scale;
  const DeviceScope scope(device);
  if (!scope.ok) return LSTM_INT_E_DEVICE;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  if (in_chunks(p)) {
    ChunkArgs c{a, static_cast<uint32_t *>(workspace), (p->steps + kChunk - 1) / kChunk, 1};
    // The products of keys and queries are the same for all value heads of a key head: a wave for all of them, as long as
    // that leaves the device full.  2048 steps, two value heads to each of 8 x 16 key heads 335 us instead of 348, of 4 x 16
    // 176 instead of 182; four to each of 8 x 8 292 instead of 308.
    if ((int64_t)p->batch * p->key_heads * c.chunks >= 4096) c.heads = p->value_heads / p->key_heads;
    return p->dtype == LM_F32 ? launch_chunks<float>(c, s) : p->dtype == LM_F16 ? launch_chunks<_Float16>(c, s) : launch_chunks<__bf16>(c, s);
  }
  return p->dtype == LM_F32 ? launch_step<float>(a, s) : p->dtype == LM_F16 ? launch_step<_Float16>(a, s) : launch_step<__bf16>(a, s);
}

}  // extern "C"
