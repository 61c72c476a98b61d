// Products with 4-bit weights (include/lm_ops.h).
//
//   y[m, n] = a[m] sum_g s[n, g] (sum_{k in g} x[m, k] w[n, k] - zero_point sum_{k in g} w[n, k]) + bias[n]
//
// The weights lie in the order in which the MFMA takes them: 16 outputs x 128 inputs are the 16 bytes of each of 64 lanes, a
// wave's load is 1 KB in one piece.  A nibble becomes an int8 operand by a mask: (v & 0xf0) is 16 w, so the high nibbles of
// a register serve one product and the low ones, shifted, another; the factor 16 is in the scales.  A group's sum is int32
// and exact, and begins with what the zero point takes off.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "lm_common.h"

namespace lstm_int {
namespace {

constexpr int kTile = 16, kChunk = 128;  // outputs and inputs of one 1 KB piece of weights

// The 128 codes q of one output and chunk to their places in the piece of the output's tile.  Lane (n % 16, kg) has 16 bytes; a
// byte's high nibble is of one product, the low one of the next: inputs 16 kg + e of 64 each, or, in groups of 32, inputs
// 8 kg + e of 32 each, two products after the other (an MFMA never spans two groups).
void w4_pack(const int8_t q[kChunk], int n, int group, uint8_t *piece) {
  const int depth = group == 32 ? 32 : 64, per_lane = depth / 4;
  for (int kg = 0; kg < 4; ++kg) {
    uint8_t *to = piece + (kg * 16 + n % kTile) * 16;
    for (int j = 0; j < kChunk / depth; j += 2) {
      const int8_t *high = q + j * depth + kg * per_lane, *low = high + depth;
      for (int e = 0; e < per_lane; ++e) to[j / 2 * per_lane + e] = (uint8_t)((uint8_t)high[e] << 4 | (low[e] & 15));
    }
  }
}

struct W4Args {
  const uint32_t *w;
  const float *s;       // [tile][group][16], times 1/16
  const int16_t *sums;  // [tile][group][16]: 16 sum of a group's codes
  const float *bias;    // [tiles * 16] or NULL
  const int8_t *x;
  const float *row_scales;
  void *y;
  int64_t x_stride, y_stride;
  int M, N, K, tiles, chunks, groups;  // groups: of all chunks
  int zero_point, split, across;  // across: workgroups over the outputs; blockIdx.x goes over them first
  float scale;
};

typedef int64_t i64;

// n bytes of a row of x from k on, zeros behind its end
template <class V, int n>
__device__ inline V load_x(const int8_t *row, int k, int K) {
  union { int8_t b[n]; V v; } r;
#pragma unroll
  for (int i = 0; i < n; ++i) r.b[i] = k + i < K ? row[k + i] : 0;
  return r.v;
}

constexpr uint32_t kHigh = 0xf0f0f0f0u;
// A group's sum c, |c| <= 255 * 128 * 128 < 2^22, begins at the bits of the float 1.5 * 2^23: the result's bits then are
// the float 1.5 * 2^23 + c.
constexpr float kMagic = 12582912.0f;
constexpr int kMagicBits = 0x4b400000;

// What the groups of a chunk begin with and are scaled by, for outputs 4 kg .. 4 kg + 3 of a tile
template <int kGroup, bool kZero>
struct Scales {
  static constexpr int kN = kChunk / kGroup;
  f32x4 s[kN];
  i32x4 begin[kN];
  // s, sums: of the chunk's first group
  __device__ void load(const float *sp, const int16_t *sums, int zp) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      s[j] = *reinterpret_cast<const f32x4 *>(sp + j * kTile);
      begin[j] = i32x4{kMagicBits, kMagicBits, kMagicBits, kMagicBits};
      if constexpr (kZero) {
        const u32x2_any v = *reinterpret_cast<const u32x2_any *>(sums + j * kTile);
#pragma unroll
        for (int r = 0; r < 4; ++r) begin[j][r] = kMagicBits - zp * ((int)(v[r / 2] << (r % 2 ? 0 : 16)) >> 16);
      }
    }
  }
};

__device__ inline f32x4 add_scaled(i32x4 c, f32x4 s, f32x4 acc) {
#pragma unroll
  for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(__int_as_float(c[r]) - kMagic, s[r], acc[r]);
  return acc;
}

// acc += the groups of a chunk, 16 outputs x 16 rows: v the weights as they lie in memory; x the rows' operands of 64
// inputs each (groups of 32: of 32 each)
template <int kGroup, bool kZero>
__device__ inline f32x4 w4_chunk(f32x4 acc, u32x4 v, const i32x4 x[2], const Scales<kGroup, kZero> &sc) {
  const i32x4 hi = (i32x4)(v & kHigh), lo = (i32x4)((v << 4) & kHigh);
  if constexpr (kGroup == 64) {
    acc = add_scaled(__builtin_amdgcn_mfma_i32_16x16x64_i8(hi, x[0], sc.begin[0], 0, 0, 0), sc.s[0], acc);
    return add_scaled(__builtin_amdgcn_mfma_i32_16x16x64_i8(lo, x[1], sc.begin[1], 0, 0, 0), sc.s[1], acc);
  } else {
    const i32x4 c = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi, x[0], sc.begin[0], 0, 0, 0);
    return add_scaled(__builtin_amdgcn_mfma_i32_16x16x64_i8(lo, x[1], c, 0, 0, 0), sc.s[0], acc);
  }
}
template <bool kZero>
__device__ inline f32x4 w4_chunk(f32x4 acc, u32x4 v, const i64 x[4], const Scales<32, kZero> &sc) {
  union { u32x4 v; i64 q[2]; } hi, lo;
  hi.v = v & kHigh;
  lo.v = (v << 4) & kHigh;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    acc = add_scaled(__builtin_amdgcn_mfma_i32_16x16x32_i8(j & 1 ? lo.q[j / 2] : hi.q[j / 2], x[j], sc.begin[j], 0, 0, 0), sc.s[j], acc);
  return acc;
}

// one row's operands of a chunk, lane kg = lane / 16
template <int kGroup>
struct RowOperands {
  i32x4 x[2];
  __device__ void load(const int8_t *row, int k0, int kg, int K) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = k0 + 64 * j + 16 * kg;
      x[j] = k0 + kChunk <= K ? (i32x4)*reinterpret_cast<const u32x4_any *>(row + k) : load_x<i32x4, 16>(row, k, K);
    }
  }
};
template <>
struct RowOperands<32> {
  i64 x[4];
  __device__ void load(const int8_t *row, int k0, int kg, int K) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + 32 * j + 8 * kg;
      union { u32x2_any u; i64 v; } r;
      if (k0 + kChunk <= K) r.u = *reinterpret_cast<const u32x2_any *>(row + k);
      else r.v = load_x<i64, 8>(row, k, K);
      x[j] = r.v;
    }
  }
};

__device__ inline float row_scale(const W4Args &a, int64_t m) { return a.row_scales ? a.row_scales[m < a.M ? m : a.M - 1] : a.scale; }
__device__ inline f32x4 bias_of(const W4Args &a, int n) { return a.bias ? *reinterpret_cast<const f32x4 *>(a.bias + n) : f32x4{0, 0, 0, 0}; }

template <class T>
__device__ inline void w4_store(const W4Args &a, f32x4 acc, float am, f32x4 bias, int64_t m, int n) {
  T *y = static_cast<T *>(a.y) + m * a.y_stride + n;
  union {
    T e[4];
    uint32_t w[sizeof(T)];
  } o;
#pragma unroll
  for (int r = 0; r < 4; ++r) o.e[r] = (T)(am * acc[r] + bias[r]);
  if (n + 4 <= a.N) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4_any *>(y) = u32x4{o.w[0], o.w[1], o.w[2], o.w[3]};
    else *reinterpret_cast<u32x2_any *>(y) = u32x2_any{o.w[0], o.w[1]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < a.N) y[r] = o.e[r];
  }
}

// Few rows: a wave has 16 outputs x 16 kRows rows and every split-th chunk of the inputs, kAhead of them requested before
// the first is used; the parts of a tile meet in LDS, in the order of the waves.  Bound by the weights' way from memory where
// there are many (2 x 4096 -> 32000, groups of 64: 19 us, 4.0 TB/s), by a launch and one round of loads where there are few
// (1 x 2048 -> 2048 3.1 us, 32 x 4096 -> 4096 7.9).
template <int kGroup, int kRows, bool kZero, class T>
__global__ __launch_bounds__(512) void w4_rows_kernel(W4Args a) {
  // four chunks ahead where registers allow: 1 x 4096 -> 64000 35.0 us, two ahead 37.1; else two: 7 x 640 -> 32003 in groups of
  // 32 8.2 us, four ahead 10.2, 128 x 4096 -> 4096 20.9 and 22.4
  constexpr int kAhead = kRows == 4 || kGroup == 32 ? 2 : 4, per_chunk = kChunk / kGroup;
  __shared__ f32x4 part[8][kRows][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x % a.across * (8 / a.split) + wave / a.split, p = wave % a.split;
  const int kg = lane >> 4;
  const int64_t m0 = (int64_t)(blockIdx.x / a.across) * 16 * kRows + (lane & 15);
  f32x4 acc[kRows] = {};
  if (tile < a.tiles) {
    const int8_t *xrow[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) xrow[i] = a.x + (m0 + 16 * i < a.M ? m0 + 16 * i : a.M - 1) * a.x_stride;
    const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w) + (int64_t)tile * a.chunks * 64 + lane;
    const float *s = a.s + (int64_t)tile * a.groups * kTile + 4 * kg;
    const int16_t *sums = a.sums + (int64_t)tile * a.groups * kTile + 4 * kg;
    for (int c0 = p; c0 < a.chunks; c0 += a.split * kAhead) {
      u32x4 v[kAhead];
      Scales<kGroup, kZero> sc[kAhead];
      RowOperands<kGroup> x[kAhead][kRows];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int c = c0 + n * a.split;
        if (c >= a.chunks) break;
        v[n] = __builtin_nontemporal_load(w + (int64_t)c * 64);
        sc[n].load(s + c * per_chunk * kTile, sums + c * per_chunk * kTile, a.zero_point);
#pragma unroll
        for (int i = 0; i < kRows; ++i) x[n][i].load(xrow[i], c * kChunk, kg, a.K);
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        if (c0 + n * a.split >= a.chunks) break;
#pragma unroll
        for (int i = 0; i < kRows; ++i) acc[i] = w4_chunk(acc[i], v[n], x[n][i].x, sc[n]);
      }
    }
  }
  if (a.split > 1) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (p) return;
    for (int j = 1; j < a.split; ++j)
#pragma unroll
      for (int i = 0; i < kRows; ++i) acc[i] += part[wave + j][i][lane];
  }
  if (tile >= a.tiles) return;
  const f32x4 bias = bias_of(a, tile * kTile + 4 * kg);
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (m0 + 16 * i < a.M) w4_store<T>(a, acc[i], row_scale(a, m0 + 16 * i), bias, m0 + 16 * i, tile * kTile + 4 * kg);
}

// Many rows: a workgroup of eight waves has 128 rows x 128 outputs, a wave 64 x 32 of them.  A chunk's operands and scales
// go through LDS, two chunks deep.  Needs two chunks or more.  Bound by the latency of a chunk's loads and the stores, with 16
// waves on a compute unit: 16384 x 640 -> 8192 166 us, 1.0 POP/s (before the stores went through LDS 192, of which 150 without
// them and 177 without the products); 4096 x 4096 -> 4096 105 us, 1.3 POP/s.  More in flight by way of registers needs
// more than there are (two stages: 295 us); loads straight into LDS were not tried.  The first product in groups of 32: 253 us,
// and 446 with a zero point, where 21 registers are spilled.
template <int kGroup, bool kZero, class T>
__global__ __launch_bounds__(512, 4) void w4_block_kernel(W4Args a) {
  constexpr int per_chunk = kChunk / kGroup;
  // results on their way out: rows of 128, a half of them at a time in float32, 16 bytes apart from multiples of all banks
  constexpr int kOutRows = sizeof(T) == 4 ? 64 : 128, kOutLd = 128 + 16 / sizeof(T);
  __shared__ union {
    struct {
      u32x4 xs[2][8][2][64];  // [row tile][64 inputs][operand order]
      u32x4 ws[2][8][64];     // [output tile]
      f32x4 ss[2][8 * per_chunk * 4];
      u32x4 zs[2][8 * per_chunk * 2];
    };
    T out[kOutRows][kOutLd];
  } lds;
  auto &xs = lds.xs;
  auto &ws = lds.ws;
  auto &ss = lds.ss;
  auto &zs = lds.zs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = lane >> 4, i16 = lane & 15;
  const int nb = blockIdx.x % a.across;
  const int64_t m0 = (int64_t)(blockIdx.x / a.across) * 128;
  const int nt0 = (wave & 3) * 2, mt0 = (wave >> 2) * 4, tile0 = nb * 8 + nt0;

  // a wave brings row tile `wave` and output tile `wave`
  const int64_t mine = m0 + wave * 16 + i16;
  const int8_t *xrow = a.x + (mine < a.M ? mine : a.M - 1) * a.x_stride;
  const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w) + (int64_t)(nb * 8 + wave) * a.chunks * 64;
  // scales and sums: the first threads hold one vector each, the others fetch one of those too (no branch around a load)
  constexpr int kS = 8 * per_chunk * 4, kZ = 8 * per_chunk * 2;
  const int st = tid % kS, zt = tid % kZ;
  const f32x4 *sp = reinterpret_cast<const f32x4 *>(a.s) + ((int64_t)(nb * 8 + st / (per_chunk * 4)) * a.groups * 4 + st % (per_chunk * 4));
  const u32x4 *zp = reinterpret_cast<const u32x4 *>(a.sums) + ((int64_t)(nb * 8 + zt / (per_chunk * 2)) * a.groups * 2 + zt % (per_chunk * 2));
  RowOperands<64> xr;
  u32x4 wr, zr;
  f32x4 sr;
  auto fetch_weights = [&](int c) {
    wr = (w + (int64_t)c * 64)[(unsigned)lane];
    sr = sp[c * per_chunk * 4];
    if constexpr (kZero) zr = zp[c * per_chunk * 2];
  };
  auto put = [&](int b) {
    xs[b][wave][0][lane] = (u32x4)xr.x[0], xs[b][wave][1][lane] = (u32x4)xr.x[1];
    ws[b][wave][lane] = wr;
    if (tid < kS) ss[b][tid] = sr;
    if (kZero && tid < kZ) zs[b][tid] = zr;
  };

  f32x4 acc[2][4] = {};  // [output tile][row tile]
  auto compute = [&](int b) {
    RowOperands<kGroup> x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int8_t *t = reinterpret_cast<const int8_t *>(xs[b][mt0 + i]);
      if constexpr (kGroup == 32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // 16 bytes of row i16 are those of piece 2 j + kg / 2, of which this lane has one half
          const int piece = 2 * j + kg / 2;
          x[i].x[j] = *reinterpret_cast<const i64 *>(t + (piece * 16 + i16) * 16 + kg % 2 * 8);
        }
      } else {
        x[i].x[0] = reinterpret_cast<const i32x4 *>(t)[lane], x[i].x[1] = reinterpret_cast<const i32x4 *>(t)[64 + lane];
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Scales<kGroup, kZero> sc;
      const int at = (nt0 + j) * per_chunk * kTile + 4 * kg;
      sc.load(reinterpret_cast<const float *>(ss[b]) + at, reinterpret_cast<const int16_t *>(zs[b]) + at, a.zero_point);
      const u32x4 v = ws[b][nt0 + j][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = w4_chunk(acc[j][i], v, x[i].x, sc);
      // keeps the products of the tile behind this one, and their registers, behind it
      asm volatile("" : "+v"(acc[j][0]), "+v"(acc[j][1]), "+v"(acc[j][2]), "+v"(acc[j][3]));
    }
  };
  // step 0 is the last chunk, which may be short; step n is chunk n - 1, a whole one
  xr.load(xrow, (a.chunks - 1) * kChunk, kg, a.K);
  fetch_weights(a.chunks - 1);
  put(0);
  __syncthreads();
  for (int n = 0; n < a.chunks; ++n) {
    const int next = n + 1 < a.chunks ? n : n - 1;  // behind the end: the last whole chunk again
#pragma unroll
    for (int j = 0; j < 2; ++j) xr.x[j] = (i32x4)*reinterpret_cast<const u32x4_any *>(xrow + next * kChunk + 64 * j + 16 * kg);
    fetch_weights(next);
    compute(n & 1);
    put((n + 1) & 1);
    __syncthreads();
  }
  f32x4 bias[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) bias[j] = bias_of(a, (tile0 + j) * kTile + 4 * kg);
  // through LDS into whole rows: a lane's four outputs of each of 16 rows are pieces of 32 bytes in memory (16384 x 640 ->
  // 8192: 192 us so, 166 as rows of 256 bytes)
#pragma unroll
  for (int half = 0; half < 128 / kOutRows; ++half) {
    if (half) __syncthreads();
    if (kOutRows == 128 || wave >> 2 == half)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = (mt0 + i) * 16 + i16;
        const float am = row_scale(a, m0 + m);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          T *to = &lds.out[m % kOutRows][(nt0 + j) * kTile + 4 * kg];
#pragma unroll
          for (int r = 0; r < 4; ++r) to[r] = (T)(am * acc[j][i][r] + bias[j][r]);
        }
      }
    __syncthreads();
    constexpr int kPiece = 16 / sizeof(T), kPieces = 128 / kPiece;  // of a row
#pragma unroll
    for (int e = 0; e < kOutRows * kPieces / 512; ++e) {
      const int id = e * 512 + tid, row = id / kPieces, at = id % kPieces * kPiece, n = nb * 128 + at;
      const int64_t m = m0 + half * kOutRows + row;
      if (m >= a.M || n >= a.N) continue;
      T *y = static_cast<T *>(a.y) + m * a.y_stride + n;
      const T *from = &lds.out[row][at];
      if (n + kPiece <= a.N) *reinterpret_cast<u32x4_any *>(y) = *reinterpret_cast<const u32x4 *>(from);
      else
#pragma unroll
        for (int r = 0; r < kPiece; ++r)
          if (n + r < a.N) y[r] = from[r];
    }
  }
}

template <int kGroup, bool kZero, class T>
int launch_w4(W4Args a, hipStream_t s) {
  // A chunk of blocks takes what some 900 pieces of 64 rows x 16 outputs take by themselves, spread over the device.  us, rows
  // / blocks, at 900 and on both sides: 4096 inputs and outputs, 192 and 256 rows 30 / 33 and 39 / 33; 640 inputs, 8192
  // outputs, 64 and 96 rows 6.1 / 7.1 and 9.5 / 7.6; 1024 and 1024, 512 rows 8.7 / 10.8; 512 and 32000, 32 rows 9.1 / 6.5;
  // the same in groups of 32, where both take twice as long.
  const bool blocks = a.M > 16 && a.chunks > 1 && (int64_t)((a.M + 63) / 64) * a.tiles > 900;
  int rows = blocks ? 128 : a.M <= 16 ? 16 : a.M <= 32 ? 32 : 64;
  const int tiles = blocks ? 8 : 8 / a.split;
  a.across = (a.tiles + tiles - 1) / tiles;
  // fewer rows to a wave where that takes a workgroup to more of the compute units: 1821 x 6592 -> 64 29 us in 64s, 17 so;
  // 64 x 1024 -> 1024 5.3 and 3.3
  while (!blocks && rows > 16 && (int64_t)a.across * ((a.M + rows - 1) / rows) < 256) rows /= 2;
  const int64_t count = (int64_t)a.across * ((a.M + rows - 1) / rows);  // one dimension: the others end at 65536,
  if (count > UINT32_MAX / 512) return LSTM_INT_E_UNSUPPORTED;          // and this one at 2^32 threads
  const dim3 grid((unsigned)count), block(512);
  return blocks       ? launch(w4_block_kernel<kGroup, kZero, T>, grid, block, s, a)
         : rows == 16 ? launch(w4_rows_kernel<kGroup, 1, kZero, T>, grid, block, s, a)
         : rows == 32 ? launch(w4_rows_kernel<kGroup, 2, kZero, T>, grid, block, s, a)
                      : launch(w4_rows_kernel<kGroup, 4, kZero, T>, grid, block, s, a);
}

template <int kGroup, class T>
int launch_w4(const W4Args &a, hipStream_t s) {
  return a.zero_point ? launch_w4<kGroup, true, T>(a, s) : launch_w4<kGroup, false, T>(a, s);
}

template <class T>
int launch_w4(const W4Args &a, int group, hipStream_t s) {
  return group == 32 ? launch_w4<32, T>(a, s) : group == 64 ? launch_w4<64, T>(a, s) : launch_w4<128, T>(a, s);
}

}  // namespace
}  // namespace lstm_int

using namespace lstm_int;

struct w4_linear_model {
  int32_t K = 0, N = 0, group = 0, groups = 0, device = -1;
  int32_t tiles = 0, chunks = 0, dev_groups = 0;
  std::vector<int8_t> codes;
  std::vector<float> scales;
  uint8_t *base = nullptr;
  size_t o_s = 0, o_sums = 0, o_bias = 0;
  bool bias = false;
};

extern "C" {

int w4_linear_prepare(const w4_linear_params *p, int32_t device, w4_linear_model **out) {
  if (!out) return LSTM_INT_E_INVALID_ARG;
  *out = nullptr;
  if (!p || p->inputs < 1 || p->outputs < 1 || (p->group_size != 32 && p->group_size != 64 && p->group_size != 128) || device < -1)
    return LSTM_INT_E_INVALID_ARG;
  if (p->W ? p->codes || p->scales : !p->codes || !p->scales) return LSTM_INT_E_INVALID_ARG;
  const int K = p->inputs, N = p->outputs, G = p->group_size;
  if (K > 1 << 17 || N > 1 << 24) return LSTM_INT_E_UNSUPPORTED;
  w4_linear_model *m = new (std::nothrow) w4_linear_model();
  if (!m) return LSTM_INT_E_OUT_OF_MEMORY;
  int rc = LSTM_INT_OK;
  try {
    const int groups = (K + G - 1) / G;
    m->K = K; m->N = N; m->group = G; m->groups = groups; m->device = device;
    m->codes.resize((size_t)N * K);
    m->scales.resize((size_t)N * groups);
    bool finite = true, in_range = true;
    for (int n = 0; n < N; ++n)
      for (int g = 0; g < groups; ++g) {
        const size_t at = (size_t)n * K + (size_t)g * G, to = (size_t)n * groups + g;
        const int len = std::min(G, K - g * G);
        int8_t *q = &m->codes[at];
        if (p->W) {
          float most = 0;
          for (int i = 0; i < len; ++i) {
            finite &= std::isfinite(p->W[at + i]);
            most = std::max(most, std::fabs(p->W[at + i]));
          }
          const float s = most / 7;
          m->scales[to] = s;
          // a subnormal scale is coarse: its codes are held to the range
          for (int i = 0; i < len; ++i)
            q[i] = s > 0 && finite ? (int8_t)std::max(-8.0f, std::min(7.0f, std::round(p->W[at + i] / s))) : (int8_t)0;
        } else {
          m->scales[to] = p->scales[to];
          finite &= std::isfinite(p->scales[to]);
          for (int i = 0; i < len; ++i) {
            q[i] = p->codes[at + i];
            in_range &= q[i] >= -8 && q[i] <= 7;
          }
        }
      }
    if (p->bias)
      for (int n = 0; n < N; ++n) finite &= std::isfinite(p->bias[n]);
    if (!in_range) rc = LSTM_INT_E_INVALID_ARG;
    else if (!finite) rc = LSTM_INT_E_BAD_RANGE;
    if (rc == LSTM_INT_OK && device >= 0) {
      // whole chunks of inputs, whole pieces of 128 outputs; zeros behind the ends
      m->tiles = (N + 127) / 128 * 8;
      m->chunks = (K + kChunk - 1) / kChunk;
      m->dev_groups = m->chunks * (kChunk / G);
      const size_t per_tile = (size_t)m->dev_groups * kTile, tiles = m->tiles;
      m->o_s = tiles * m->chunks * 1024;
      m->o_sums = m->o_s + tiles * per_tile * 4;
      m->o_bias = (m->o_sums + tiles * per_tile * 2 + 255) & ~(size_t)255;
      m->bias = p->bias != nullptr;
      std::vector<uint8_t> img(m->o_bias + (m->bias ? tiles * kTile * 4 : 0), 0);
      float *s = reinterpret_cast<float *>(img.data() + m->o_s);
      int16_t *sums = reinterpret_cast<int16_t *>(img.data() + m->o_sums);
      for (int n = 0; n < N; ++n) {
        const size_t tile = n / kTile;
        for (int c = 0; c < m->chunks; ++c) {
          int8_t q[kChunk] = {};
          std::memcpy(q, &m->codes[(size_t)n * K + (size_t)c * kChunk], std::min(kChunk, K - c * kChunk));
          w4_pack(q, n, G, img.data() + (tile * m->chunks + c) * 1024);
          for (int g = c * (kChunk / G), i = 0; i < kChunk; ++g, i += G) {
            int sum = 0;
            for (int e = 0; e < G; ++e) sum += q[i + e];
            sums[tile * per_tile + (size_t)g * kTile + n % kTile] = (int16_t)(16 * sum);
            if (g < groups) s[tile * per_tile + (size_t)g * kTile + n % kTile] = m->scales[(size_t)n * groups + g] / 16;
          }
        }
        if (m->bias) reinterpret_cast<float *>(img.data() + m->o_bias)[n] = p->bias[n];
      }
      const DeviceScope scope(device);
      if (!scope.ok) rc = LSTM_INT_E_DEVICE;
      else if (hipMalloc(reinterpret_cast<void **>(&m->base), img.size()) != hipSuccess) {
        m->base = nullptr;
        (void)hipGetLastError();  // said here
        rc = LSTM_INT_E_OUT_OF_MEMORY;
      } else if (hipMemcpy(m->base, img.data(), img.size(), hipMemcpyHostToDevice) != hipSuccess) {
        rc = LSTM_INT_E_DEVICE;
      }
    }
  } catch (const std::bad_alloc &) {
    rc = LSTM_INT_E_OUT_OF_MEMORY;
  } catch (...) {
    rc = LSTM_INT_E_DEVICE;
  }
  if (rc != LSTM_INT_OK) {
    w4_linear_destroy(m);
    return rc;
  }
  *out = m;
  return LSTM_INT_OK;
}

int w4_linear_get_quant(const w4_linear_model *m, w4_linear_quant *out) {
  if (!m || !out) return LSTM_INT_E_INVALID_ARG;
  *out = {m->K, m->N, m->group, m->groups, m->codes.data(), m->scales.data()};
  return LSTM_INT_OK;
}

int w4_linear_forward(const w4_linear_model *m, const int8_t *x, int64_t x_stride, int64_t rows, const float *row_scales, float scale,
                      int32_t zero_point, void *y, int64_t y_stride, int32_t dtype, void *hip_stream) {
  if (!m || rows < 0 || !lm_type_bytes(dtype) || zero_point < -128 || zero_point > 127) return LSTM_INT_E_INVALID_ARG;
  if (rows == 0) return LSTM_INT_OK;
  if (!x || !y || (rows > 1 && (x_stride < m->K || y_stride < m->N))) return LSTM_INT_E_INVALID_ARG;
  if (m->device < 0) return LSTM_INT_E_DEVICE;
  if (rows > 1 << 24) return LSTM_INT_E_UNSUPPORTED;
  W4Args a{};
  a.w = reinterpret_cast<const uint32_t *>(m->base);
  a.s = reinterpret_cast<const float *>(m->base + m->o_s);
  a.sums = reinterpret_cast<const int16_t *>(m->base + m->o_sums);
  a.bias = m->bias ? reinterpret_cast<const float *>(m->base + m->o_bias) : nullptr;
  a.x = x; a.row_scales = row_scales; a.y = y; a.x_stride = x_stride; a.y_stride = y_stride;
  a.M = (int)rows; a.N = m->N; a.K = m->K; a.tiles = (m->N + kTile - 1) / kTile; a.chunks = m->chunks; a.groups = m->dev_groups;
  a.zero_point = zero_point; a.scale = scale;
  a.split = 1;
  // Waves share a tile's inputs until there are six to a compute unit.  One row of 4096 inputs, us: 8192 outputs by four waves
  // 6.2, by two 9.5; 16384 by two 10.4, by one 16.2; 28000 by two 18.7, by one 17.7; 2048 x 2048 by eight 3.2, by one 7.0.
  while (a.split < 8 && a.split * 2 <= a.chunks && (int64_t)a.tiles * a.split < 1536) a.split *= 2;
  const DeviceScope scope(m->device);
  if (!scope.ok) return LSTM_INT_E_DEVICE;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  return dtype == LM_F32 ? launch_w4<float>(a, m->group, s)
                         : dtype == LM_F16 ? launch_w4<_Float16>(a, m->group, s) : launch_w4<__bf16>(a, m->group, s);
}

void w4_linear_destroy(w4_linear_model *m) {
  if (!m) return;
  if (m->base) {
    const DeviceScope scope(m->device);
    (void)hipFree(m->base);
  }
  delete m;
}

}  // extern "C"
