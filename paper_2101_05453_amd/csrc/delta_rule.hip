// The gated delta rule (include/lm_ops.h).
//
//   S <- e^g S;  u = beta (v - S' k);  S <- S + k u';  y = scale S' q
#include <algorithm>

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

// Step by step: a wave has 16 columns of one head's state in registers, lane (r = lane / 4, c = lane % 4) the rows
// kRows r .. kRows r + kRows - 1 of columns 4 c .. 4 c + 3.  S' k and S' q are taken of the state before the step, in one
// reduction over the lanes, and y = e^g S' q + (k' q) u follows from them: a step waits for one reduction.
template <class T, int kRows>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a) {
  const int lane = threadIdx.x & 63;
  const int tiles = (a.Dv + 15) / 16;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)a.B * a.Hv * tiles) return;
  const int tile = (int)(item % tiles), h = (int)(item / tiles % a.Hv), b = (int)(item / tiles / a.Hv);
  const int hk = h / (a.Hv / a.Hk);
  const int r0 = (lane >> 2) * kRows, c0 = tile * 16 + (lane & 3) * 4;
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
    for (int m = 4; m < 64; m <<= 1) {
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
    if (lane < 4)
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

template <class T>
int launch_step(const DeltaArgs &a, hipStream_t s) {
  const int64_t items = (int64_t)a.B * a.Hv * ((a.Dv + 15) / 16);
  const dim3 grid((unsigned)((items + 3) / 4)), block(256);
  return a.Dk <= 64 ? launch(delta_step_kernel<T, 4>, grid, block, s, a)
                    : a.Dk <= 128 ? launch(delta_step_kernel<T, 8>, grid, block, s, a) : launch(delta_step_kernel<T, 16>, grid, block, s, a);
}

// ---------------------------------------------------------------------------------------------------------------------
// Sequences, kChunk steps at a time.  With c_i the sum of g over the chunk's steps up to i, and S the state before it:
//   A_ij = beta_i e^(c_i - c_j) k_i'k_j  (j < i),   X = (1 + A)^-1 diag(beta)
//   u = X (v - diag(e^c) K S),   y = diag(e^c) Q S + P u,   P_ij = e^(c_i - c_j) q_i'k_j  (j <= i)
//   S <- e^(c_last) S + K' diag(e^(c_last - c)) u
// X and P do not depend on the state: delta_prep_kernel computes them for all chunks side by side.  delta_scan_kernel
// carries the state from chunk to chunk.
//
// Products: on the bf16 MFMA, whose products are exact and whose sums are float32.  A float32 operand is taken as three
// bf16 parts that add up to it exactly (8 + 8 + 8 bits of its 24), and of the products of two operands' parts those are
// left out that are below 2^-24 of the largest: float32 results at three (a bf16 key with the state) to six MFMAs for
// one, where the float32 MFMA takes 16 times the time.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kChunk = 32;
constexpr int kMatrix = 2 * 64 * 8;                   // floats of X or P in the workspace: two tiles of 16 rows, 8 floats a lane
constexpr int kItemFloats = 2 * kMatrix + 4 * kChunk;  // X, P and four factors for each step
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <class T> constexpr int kParts = sizeof(T) == 4 ? 3 : __is_same(T, __bf16) ? 1 : 2;  // bf16 parts of an input

// The MFMA's operand order: lane (i = lane % 16, g = lane / 16) of a 16 x 32 operand has the columns 4 g .. 4 g + 3 and
// 16 + 4 g .. 16 + 4 g + 3 of row i.  A result (column lane % 16, rows 4 g .. 4 g + 3) of two 16-row tiles then is the
// other operand of the next product as it lies in the registers.
union Frag {
  u32x4 w;
  bf16x8 b;
};

__device__ inline f32x4 mfma(const Frag &a, const Frag &b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0); }

__device__ inline uint32_t high_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ inline float truncated(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// x = part 0 + part 1 + part 2, exactly
__device__ inline void split8(const float *x, Frag out[3]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
    out[0].w[i] = high_halves(a, b);
    a -= truncated(a);
    b -= truncated(b);
    out[1].w[i] = high_halves(a, b);
    out[2].w[i] = high_halves(a - truncated(a), b - truncated(b));
  }
}
__device__ inline void split8(f32x4 a, f32x4 b, Frag out[3]) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  split8(x, out);
}

// four neighbouring elements of a row, zeros behind n
template <class T>
struct Raw4 {
  union {
    uint32_t w[sizeof(T)];
    T e[4];
  };
  __device__ void load(const T *p, int n) {
    if (n >= 4) {
      if constexpr (sizeof(T) == 4) {
        const u32x4 v = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
      } else {
        const u32x2_any v = *reinterpret_cast<const u32x2_any *>(p);
        w[0] = v[0], w[1] = v[1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = i < n ? p[i] : (T)0.0f;
    }
  }
};

// part p of four values, as two words
template <int kP>
__device__ inline void parts4(const float *x, uint32_t out[kP][2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int p = 0; p < kP; ++p) {
      out[p][i] = high_halves(a, b);
      a -= truncated(a);
      b -= truncated(b);
    }
  }
}

// c += a b over the parts of both that matter
template <int kPa, int kPb>
__device__ inline f32x4 mfma_parts(const Frag *a, const Frag *b, f32x4 c) {
#pragma unroll
  for (int i = kPa - 1; i >= 0; --i)
#pragma unroll
    for (int j = kPb - 1; j >= 0; --j)
      if (i + j <= 2) c = mfma(a[i], b[j], c);
  return c;
}

struct ChunkArgs {
  DeltaArgs d;
  float *items;  // [B Hv][chunks][kItemFloats]
  int chunks;
};

__device__ inline int length_of(const DeltaArgs &a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T; }

// One wave per chunk and value head: X, P and the factors of its steps
//   e^c_i |k_i|^-1,  e^c_i |q_i|^-1 scale,  e^(c_last - c_i) |k_i|^-1,  e^c_last        (norms: 1 without normalize)
template <class T>
__global__ __launch_bounds__(64) void delta_prep_kernel(ChunkArgs a) {
  constexpr int kP = kParts<T>, kLd = 36;
  const DeltaArgs &d = a.d;
  __shared__ __attribute__((aligned(16))) float mat[2][kChunk * kLd];  // A, then X; P
  __shared__ double sum_g[kChunk];
  __shared__ float rate[kChunk], norm_k[kChunk], norm_q[kChunk];
  const int lane = threadIdx.x, i = lane & 15, g = lane >> 4;
  const int chunk = blockIdx.x;
  for (int bh = blockIdx.y; bh < d.B * d.Hv; bh += gridDim.y) {
    const int b = bh / d.Hv, h = bh % d.Hv, hk = h / (d.Hv / d.Hk);
    const int t0 = chunk * kChunk, left = length_of(d, b) - t0;  // steps of the row from here on
    if (left <= 0) continue;
    __syncthreads();
    {
      const int t = lane & 31;
      double c = 0;
      float bt = 0;
      if (t < left) {
        const float gv = d.g[b * d.g_stride[1] + h * d.g_stride[2] + (int64_t)(t0 + t) * d.g_stride[0]];
        c = gv < -1000.0f ? -1000.0 : (double)gv;  // e^-1000 is zero; the sum stays a number
        bt = d.beta[b * d.beta_stride[1] + h * d.beta_stride[2] + (int64_t)(t0 + t) * d.beta_stride[0]];
      }
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) {
        union { double v; int w[2]; } x, y;
        x.v = c;
        y.w[0] = __shfl_up(x.w[0], m, 32);
        y.w[1] = __shfl_up(x.w[1], m, 32);
        if (t >= m) c += y.v;
      }
      if (lane < 32) sum_g[t] = c, rate[t] = bt;
    }
    const T *kp = static_cast<const T *>(d.k) + b * d.k_stride[1] + hk * d.k_stride[2];
    const T *qp = static_cast<const T *>(d.q) + b * d.q_stride[1] + hk * d.q_stride[2];
    f32x4 kk[3] = {}, qk[3] = {};  // tiles (0,0), (1,0), (1,1)
    float sk[2] = {0, 0}, sq[2] = {0, 0};
    for (int kb = 0; kb < d.Dk; kb += 32) {
      Frag kf[2][kP], qf[2][kP];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int t = 16 * m + i;
        const bool in = t < left;
        const T *kr = kp + (int64_t)(t0 + t) * d.k_stride[0], *qr = qp + (int64_t)(t0 + t) * d.q_stride[0];
        Raw4<T> rk[2], rq[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = kb + 16 * e + 4 * g;
          rk[e].load(kr + col, in ? d.Dk - col : 0);
          rq[e].load(qr + col, in ? d.Dk - col : 0);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x[4], y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = (float)rk[e].e[j], y[j] = (float)rq[e].e[j];
            sk[m] = __builtin_fmaf(x[j], x[j], sk[m]);
            sq[m] = __builtin_fmaf(y[j], y[j], sq[m]);
          }
          uint32_t w[kP][2];
          parts4<kP>(x, w);
#pragma unroll
          for (int p = 0; p < kP; ++p) kf[m][p].w[2 * e] = w[p][0], kf[m][p].w[2 * e + 1] = w[p][1];
          parts4<kP>(y, w);
#pragma unroll
          for (int p = 0; p < kP; ++p) qf[m][p].w[2 * e] = w[p][0], qf[m][p].w[2 * e + 1] = w[p][1];
        }
      }
      kk[0] = mfma_parts<kP, kP>(kf[0], kf[0], kk[0]);
      kk[1] = mfma_parts<kP, kP>(kf[1], kf[0], kk[1]);
      kk[2] = mfma_parts<kP, kP>(kf[1], kf[1], kk[2]);
      qk[0] = mfma_parts<kP, kP>(qf[0], kf[0], qk[0]);
      qk[1] = mfma_parts<kP, kP>(qf[1], kf[0], qk[1]);
      qk[2] = mfma_parts<kP, kP>(qf[1], kf[1], qk[2]);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      sk[m] += __shfl_xor(sk[m], 16);
      sk[m] += __shfl_xor(sk[m], 32);
      sq[m] += __shfl_xor(sq[m], 16);
      sq[m] += __shfl_xor(sq[m], 32);
      if (g == 0) {
        norm_k[16 * m + i] = d.normalize ? 1.0f / sqrtf(sk[m] + kNormEps) : 1.0f;
        norm_q[16 * m + i] = (d.normalize ? 1.0f / sqrtf(sq[m] + kNormEps) : 1.0f) * d.scale;
      }
    }
    __syncthreads();
    float *item = a.items + ((int64_t)bh * a.chunks + chunk) * kItemFloats;
    if (lane < 32) {
      float *f = item + 2 * kMatrix;
      const double c = sum_g[lane], end = sum_g[kChunk - 1];
      const float e = expf((float)c);
      f[lane] = e * norm_k[lane];
      f[kChunk + lane] = e * norm_q[lane];
      f[2 * kChunk + lane] = expf((float)(end - c)) * norm_k[lane];
      f[3 * kChunk + lane] = expf((float)end);
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
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float s = r == i ? 1.0f : 0.0f;
#pragma unroll
        for (int m = 0; m < r; ++m) s = __builtin_fmaf(-A[r * kLd + m], x[m], s);
        x[r] = s;
      }
      __syncthreads();
      if (g < 2)
#pragma unroll
        for (int r = 0; r < 16; ++r) mat[0][(16 * blk + r) * kLd + 16 * blk + i] = x[r];
    }
    __syncthreads();
    {
      f32x4 m1 = {0, 0, 0, 0}, m2 = {0, 0, 0, 0};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        m1 = __builtin_amdgcn_mfma_f32_16x16x4f32(mat[0][(16 + i) * kLd + 4 * g + r], mat[0][(4 * g + r) * kLd + i], m1, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        m2 = __builtin_amdgcn_mfma_f32_16x16x4f32(mat[0][(16 + i) * kLd + 16 + 4 * g + r], m1[r], m2, 0, 0, 0);
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
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f32x4 v = *reinterpret_cast<const f32x4 *>(&mat[w][(16 * m + i) * kLd + 16 * e + 4 * g]);
          if (w == 0) v *= *reinterpret_cast<const f32x4 *>(&rate[16 * e + 4 * g]);
          *reinterpret_cast<f32x4 *>(item + w * kMatrix + (m * 64 + lane) * 8 + 4 * e) = v;
        }
  }
}

// A workgroup carries kMain * kCols * 16 columns of one head's state through the sequence: kMain waves have 16 kCols columns
// each, in the registers, for good; four more ("loaders") bring the next chunk's operands into LDS meanwhile, in parts and
// in the MFMA's order, with the chunk after it already requested.  kBuffers = 1 where two do not fit.
template <class T, int kDk, int kMain, int kCols>
struct Scan {
  static constexpr int kP = kParts<T>, kBlocks = kDk / 32, kLoaders = 4, kColumns = 16 * kMain * kCols;
  static constexpr int kThreads = (kMain + kLoaders) * 64;
  struct Buffer {
    u32x4 k[2][kBlocks][kP][64], q[2][kBlocks][kP][64];  // rows of steps, by key column
    u32x4 kt[kDk / 16][kP][64];                          // rows of key columns, by step
    u32x4 x[2][3][64], p[2][3][64];
    u32x4 vt[kColumns / 16][sizeof(T) / 2][64];          // rows of value columns, by step: as they are
    float factor[4][kChunk];
  };
  static constexpr int kBuffers = 2 * sizeof(Buffer) <= 160 * 1024 ? 2 : 1;
};

// Where lane (i, g)'s operand lies among the 64 of k, q, kt and vt: the writers, which have four rows of one g each, then
// meet in no bank, and a reader's order does not matter.
__device__ inline int slot_of(int i, int g) { return (i ^ g) + 16 * g; }

// A block of four steps x four columns of a matrix [T, width]
template <class T>
struct Block4 {
  Raw4<T> row[4];
  // four columns from col on, where there are that many; else the last four of the row, which shifted() puts in place
  __device__ void fetch(const T *p, int64_t stride, int t, int last, int col, int width) {
    const T *at = p + min(col, width - 4);
#pragma unroll
    for (int r = 0; r < 4; ++r) row[r].load(at + (int64_t)min(t + r, last) * stride, 4);
  }
  // columns beyond the width as zeros
  __device__ void shift(int col, int width) {
    const int s = col - min(col, width - 4);
    if (s == 0) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      Raw4<T> o;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        T v = (T)0.0f;
#pragma unroll
        for (int j = i + 1; j < 4; ++j)
          if (j == i + s) v = row[r].e[j];
        o.e[i] = v;
      }
      row[r] = o;
    }
  }
  // part p of row r, as two words
  template <int kP>
  __device__ void parts(int r, uint32_t out[kP][2]) const {
    if constexpr (kP == 1) {
      out[0][0] = row[r].w[0], out[0][1] = row[r].w[1];
    } else {
      const float x[4] = {(float)row[r].e[0], (float)row[r].e[1], (float)row[r].e[2], (float)row[r].e[3]};
      parts4<kP>(x, out);
    }
  }
};

// column j of four rows of two words (four 16-bit elements each), as two words
__device__ inline u32x2_any column_of(const uint32_t w[4][2], int j) {
  const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
  return u32x2_any{__builtin_amdgcn_perm(w[1][j / 2], w[0][j / 2], pick), __builtin_amdgcn_perm(w[3][j / 2], w[2][j / 2], pick)};
}
__device__ inline void put8(u32x4 &to, int half, u32x2_any v) { reinterpret_cast<uint64_t *>(&to)[half] = __builtin_bit_cast(uint64_t, v); }

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
  const float *item = a.items + (int64_t)(b * d.Hv + h) * a.chunks * kItemFloats;
  // block id: 4 x 16 blocks to a wave, the steps' half above that, then the columns
  auto step_of = [](int id) { return (id / 64 % 2 * 4 + id % 4) * 4; };
  auto col_of = [](int id) { return (id / 128 * 16 + id / 4 % 16) * 4; };
  // fewer than 16 blocks of value columns: the steps' half above them
  constexpr int kVc = S::kColumns / 4 < 16 ? S::kColumns / 4 : 16;
  const int v_step = (tid / (4 * kVc) % 2 * 4 + tid % 4) * 4, v_col = (tid / (8 * kVc) * kVc + tid / 4 % kVc) * 4;
  const int v_from = blockIdx.y * S::kColumns + v_col;
  struct Stage {
    Block4<T> k[kEach], q[kEach], v;
    f32x4 m[2];
    float f;
  };
  auto fetch = [&](Stage &s, int c) {
    c = min(c, chunks - 1);
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      const int id = kKeyBlocks < 256 ? tid % kKeyBlocks : tid + 256 * n;
      s.k[n].fetch(kp, d.k_stride[0], c * kChunk + step_of(id), len - 1, col_of(id), d.Dk);
      s.q[n].fetch(qp, d.q_stride[0], c * kChunk + step_of(id), len - 1, col_of(id), d.Dk);
    }
    s.v.fetch(vp, d.v_stride[0], c * kChunk + v_step, len - 1, v_from, d.Dv);
    const float *it = item + (int64_t)c * kItemFloats;
#pragma unroll
    for (int e = 0; e < 2; ++e) s.m[e] = *reinterpret_cast<const f32x4 *>(it + tid * 8 + 4 * e);
    s.f = it[2 * kMatrix + (tid & 127)];
  };
  auto put = [&](Stage &s, typename S::Buffer &o) {
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      const int id = tid + 256 * n;
      if (kKeyBlocks < 256 && id >= kKeyBlocks) break;
      const int step = step_of(id), col = col_of(id), m = step / 16, kb = col / 32, kg = col % 16 / 4, half = col % 32 / 16;
      s.q[n].shift(col, d.Dk);
      s.k[n].shift(col, d.Dk);
      uint32_t w[kP][4][2];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint32_t v[kP][2];
        s.q[n].template parts<kP>(r, v);
#pragma unroll
        for (int p = 0; p < kP; ++p) put8(o.q[m][kb][p][slot_of(step % 16 + r, kg)], half, u32x2_any{v[p][0], v[p][1]});
        s.k[n].template parts<kP>(r, v);
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
      s.v.shift(v_from, d.Dv);
      u32x4 *to = &o.vt[v_col / 16][0][0];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = slot_of(v_col % 16 + j, v_step % 16 / 4);
        if constexpr (kHalfWords == 1) {
          uint32_t w[4][2];
#pragma unroll
          for (int r = 0; r < 4; ++r) w[r][0] = s.v.row[r].w[0], w[r][1] = s.v.row[r].w[1];
          put8(to[slot], v_step / 16, column_of(w, j));
        } else {
          to[v_step / 16 * 64 + slot] = u32x4{s.v.row[0].w[j], s.v.row[1].w[j], s.v.row[2].w[j], s.v.row[3].w[j]};
        }
      }
    }
    Frag f[3];
    split8(s.m[0], s.m[1], f);
    u32x4(*to)[3][64] = tid < 128 ? o.x : o.p;
#pragma unroll
    for (int p = 0; p < 3; ++p) to[tid / 64 % 2][p][tid & 63] = f[p].w;
    if (tid < 128) o.factor[tid / 32][tid % 32] = s.f;
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
    for (int c = 0;; c += 2) {  // main is at chunk c
      if (c + 1 < chunks) put(odd, buffer[1]);
      fetch(odd, c + 3);
      __syncthreads();
      if (c + 1 >= chunks) break;
      if (c + 2 < chunks) put(even, buffer[0]);
      fetch(even, c + 4);
      __syncthreads();
      if (c + 2 >= chunks) break;
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
    for (int j = 2; j >= 0; --j)
      if (i + j <= 2)
#pragma unroll
        for (int n = 0; n < kN; ++n) *c[n] = mfma(a[n][i], b[j], *c[n]);
}

template <class T, int kDk, int kMain, int kCols>
__global__ __launch_bounds__((kMain + 4) * 64) void delta_scan_kernel(ChunkArgs a) {
  using S = Scan<T, kDk, kMain, kCols>;
  constexpr int kP = S::kP, kBlocks = S::kBlocks, kBuffers = S::kBuffers;
  const DeltaArgs &d = a.d;
  __shared__ typename S::Buffer buffer[kBuffers];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.x, b = bh / d.Hv, h = bh % d.Hv;
  const int len = length_of(d, b), chunks = (len + kChunk - 1) / kChunk;
  if (wave >= kMain) return scan_load<T, kDk, kMain, kCols>(a, buffer, b, h, len, chunks);

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, slot = slot_of(i, g);
  int col[kCols];
  f32x4 st[kCols][kDk / 16];
  const int64_t head = (int64_t)bh * d.Dk * d.Dv;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    col[n] = ((blockIdx.y * kMain + wave) * kCols + n) * 16 + i;
#pragma unroll
    for (int m = 0; m < kDk / 16; ++m)
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
        Frag s[3];
        split8(st[n][2 * kb], st[n][2 * kb + 1], s);
        f32x4 *to[4] = {&rhs[n][0], &out[n][0], &rhs[n][1], &out[n][1]};
        mfma_side_by_side<kP, 4>(f, s, to);
      }
    }
    Frag part[kCols][3], x[2][3];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int p = 0; p < 3; ++p) x[m][p].w = o.x[m][p][lane];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      Raw8<T> v;
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e) v.w[e] = o.vt[wave * kCols + n][e][slot];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const f32x4 fk = *reinterpret_cast<const f32x4 *>(&o.factor[0][16 * m + 4 * g]), fq = *reinterpret_cast<const f32x4 *>(&o.factor[1][16 * m + 4 * g]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          rhs[n][m][r] = __builtin_fmaf(-fk[r], rhs[n][m][r], (float)v.e[4 * m + r]);
          out[n][m][r] *= fq[r];
        }
      }
    }
    f32x4 u[kCols][2];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      split8(rhs[n][0], rhs[n][1], part[n]);
      u[n][0] = u[n][1] = f32x4{0, 0, 0, 0};
      f32x4 *to[2] = {&u[n][0], &u[n][1]};
      mfma_side_by_side<3, 2>(x, part[n], to);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int p = 0; p < 3; ++p) x[m][p].w = o.p[m][p][lane];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      split8(u[n][0], u[n][1], part[n]);
      f32x4 *to[2] = {&out[n][0], &out[n][1]};
      mfma_side_by_side<3, 2>(x, part[n], to);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const f32x4 fu = *reinterpret_cast<const f32x4 *>(&o.factor[2][16 * m + 4 * g]);
#pragma unroll
      for (int n = 0; n < kCols; ++n) u[n][m] *= fu;
    }
    const float whole = o.factor[3][0];
#pragma unroll
    for (int n = 0; n < kCols; ++n) split8(u[n][0], u[n][1], part[n]);
#pragma unroll
    for (int m = 0; m < kDk / 16; m += 2) {
      Frag f[2][kP];
#pragma unroll
      for (int p = 0; p < kP; ++p) f[0][p].w = o.kt[m][p][slot], f[1][p].w = o.kt[m + 1][p][slot];
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        st[n][m] *= whole, st[n][m + 1] *= whole;
        f32x4 *to[2] = {&st[n][m], &st[n][m + 1]};
        mfma_side_by_side<kP, 2>(f, part[n], to);
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
  if (!d.new_state) return;
#pragma unroll
  for (int n = 0; n < kCols; ++n)
#pragma unroll
    for (int m = 0; m < kDk / 16; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * m + 4 * g + r;
        if (row < d.Dk && col[n] < d.Dv) d.new_state[head + (int64_t)row * d.Dv + col[n]] = st[n][m][r];
      }
}

template <class T, int kDk, int kMain, int kCols>
int launch_scan(const ChunkArgs &a, hipStream_t s) {
  const dim3 grid(a.d.B * a.d.Hv, (a.d.Dv + 16 * kMain * kCols - 1) / (16 * kMain * kCols));
  return launch(delta_scan_kernel<T, kDk, kMain, kCols>, grid, dim3((kMain + 4) * 64), s, a);
}

// As many columns to a workgroup as leave one for each compute unit: their operands come from memory once
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

template <class T>
int launch_chunks(const ChunkArgs &a, hipStream_t s) {
  const int rc = launch(delta_prep_kernel<T>, dim3(a.chunks, std::min(a.d.B * a.d.Hv, 65535)), dim3(64), s, a);
  if (rc != LSTM_INT_OK) return rc;
  return a.d.Dk <= 64 ? launch_scan<T, 64>(a, s) : a.d.Dk <= 128 ? launch_scan<T, 128>(a, s) : launch_scan<T, 256>(a, s);
}

bool in_chunks(const delta_rule_args *p) { return p->steps >= kChunk && p->key_dim >= 4 && p->value_dim >= 4; }

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
  return (size_t)p->batch * p->value_heads * ((p->steps + kChunk - 1) / kChunk) * kItemFloats * sizeof(float);
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
    const ChunkArgs c{a, static_cast<float *>(workspace), (p->steps + kChunk - 1) / kChunk};
    return p->dtype == LM_F32 ? launch_chunks<float>(c, s) : p->dtype == LM_F16 ? launch_chunks<_Float16>(c, s) : launch_chunks<__bf16>(c, s);
  }
  return p->dtype == LM_F32 ? launch_step<float>(a, s) : p->dtype == LM_F16 ? launch_step<_Float16>(a, s) : launch_step<__bf16>(a, s);
}

}  // extern "C"
