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
#include <new>
#include <vector>

#include "lm_common.h"

namespace lstm_int {
namespace {

constexpr int kTile = 16, kChunk = 128;  // outputs and inputs of one 1 KB piece of weights

// where weight (n, k) lies: piece (n / 16, k / 128); byte and nibble within it
struct W4Place {
  int byte;
  bool high;
};
W4Place w4_place(int n, int k, int group) {
  const int depth = group == 32 ? 32 : 64;  // inputs of one MFMA, which never spans two groups
  const int kk = k % kChunk, j = kk / depth, in = kk % depth, per_lane = depth / 4;
  const int lane = in / per_lane * 16 + n % kTile, e = in % per_lane;
  return {lane * 16 + j / 2 * 8 + e, j % 2 == 0};
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
  int zero_point, split;
  float scale;
};

typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef int64_t i64;

// 16 bytes of a row of x from k on, zeros behind its end
__device__ inline i32x4 load_x16(const int8_t *row, int k, int K) {
  if (k + 16 <= K) return (i32x4)*reinterpret_cast<const u32x4_any *>(row + k);
  union { int8_t b[16]; i32x4 v; } r;
#pragma unroll
  for (int i = 0; i < 16; ++i) r.b[i] = k + i < K ? row[k + i] : 0;
  return r.v;
}
__device__ inline i64 load_x8(const int8_t *row, int k, int K) {
  union { int8_t b[8]; u32x2_any u; i64 v; } r;
  if (k + 8 <= K) {
    r.u = *reinterpret_cast<const u32x2_any *>(row + k);
    return r.v;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) r.b[i] = k + i < K ? row[k + i] : 0;
  return r.v;
}

// one chunk of 128 inputs for 16 outputs x 16 rows: acc += sum of its groups, scaled
template <int kGroup>
__device__ inline void w4_chunk(f32x4 &acc, u32x4 wv, const int8_t *xrow, int k0, int kg, int K, const float *s, const int16_t *sums,
                                int zp) {
  constexpr uint32_t kHigh = 0xf0f0f0f0u;
  const i32x4 hi = (i32x4)(wv & kHigh), lo = (i32x4)((wv << 4) & kHigh);
  auto begin = [&](int g) {
    i32x4 c = {0, 0, 0, 0};
    if (zp) {
      const int16_t *p = sums + g * kTile;
#pragma unroll
      for (int r = 0; r < 4; ++r) c[r] = -zp * (int)p[r];
    }
    return c;
  };
  auto add = [&](i32x4 c, int g) {
    const f32x4 sv = *reinterpret_cast<const f32x4 *>(s + g * kTile);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf((float)c[r], sv[r], acc[r]);
  };
  if constexpr (kGroup == 32) {
    const i64 h[2] = {(i64)((uint32_t)hi[0] | (uint64_t)(uint32_t)hi[1] << 32), (i64)((uint32_t)hi[2] | (uint64_t)(uint32_t)hi[3] << 32)};
    const i64 l[2] = {(i64)((uint32_t)lo[0] | (uint64_t)(uint32_t)lo[1] << 32), (i64)((uint32_t)lo[2] | (uint64_t)(uint32_t)lo[3] << 32)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const i64 xv = load_x8(xrow, k0 + 32 * j + 8 * kg, K);
      add(__builtin_amdgcn_mfma_i32_16x16x32_i8(j & 1 ? l[j / 2] : h[j / 2], xv, begin(j), 0, 0, 0), j);
    }
  } else {
    const i32x4 x0 = load_x16(xrow, k0 + 16 * kg, K), x1 = load_x16(xrow, k0 + 64 + 16 * kg, K);
    if constexpr (kGroup == 64) {
      add(__builtin_amdgcn_mfma_i32_16x16x64_i8(hi, x0, begin(0), 0, 0, 0), 0);
      add(__builtin_amdgcn_mfma_i32_16x16x64_i8(lo, x1, begin(1), 0, 0, 0), 1);
    } else {
      const i32x4 c = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi, x0, begin(0), 0, 0, 0);
      add(__builtin_amdgcn_mfma_i32_16x16x64_i8(lo, x1, c, 0, 0, 0), 0);
    }
  }
}

template <class T>
__device__ inline void w4_store(const W4Args &a, f32x4 acc, int64_t m, int n) {
  const float am = a.row_scales ? a.row_scales[m] : a.scale;
  T *y = static_cast<T *>(a.y) + m * a.y_stride + n;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n + r < a.N) y[r] = (T)(am * acc[r] + (a.bias ? a.bias[n + r] : 0.0f));
}

// Few rows: a wave has 16 outputs x 16 rows and every split-th chunk of the inputs.
template <int kGroup, class T>
__global__ __launch_bounds__(512) void w4_rows_kernel(W4Args a) {
  __shared__ f32x4 part[8][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x * (8 / a.split) + wave / a.split, p = wave % a.split;
  const int kg = lane >> 4;
  const int64_t m = (int64_t)blockIdx.y * 16 + (lane & 15);
  const int8_t *xrow = a.x + (m < a.M ? m : a.M - 1) * a.x_stride;
  f32x4 acc = {0, 0, 0, 0};
  if (tile < a.tiles) {
    constexpr int per_chunk = kChunk / kGroup;
    const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w) + (int64_t)tile * a.chunks * 64 + lane;
    const float *s = a.s + (int64_t)tile * a.groups * kTile + 4 * kg;
    const int16_t *sums = a.sums + (int64_t)tile * a.groups * kTile + 4 * kg;
    for (int c = p; c < a.chunks; c += a.split)
      w4_chunk<kGroup>(acc, w[c * 64], xrow, c * kChunk, kg, a.K, s + c * per_chunk * kTile, sums + c * per_chunk * kTile, a.zero_point);
  }
  if (a.split > 1) {
    part[wave][lane] = acc;
    __syncthreads();
    if (p) return;
    for (int i = 1; i < a.split; ++i) acc += part[wave + i][lane];
  }
  if (tile < a.tiles && m < a.M) w4_store<T>(a, acc, m, tile * kTile + 4 * kg);
}

template <class T>
int launch_rows(const W4Args &a, int group, hipStream_t s) {
  const int per_block = 8 / a.split;
  const dim3 grid((a.tiles + per_block - 1) / per_block, (a.M + 15) / 16), block(512);
  return group == 32 ? launch(w4_rows_kernel<32, T>, grid, block, s, a)
                     : group == 64 ? launch(w4_rows_kernel<64, T>, grid, block, s, a) : launch(w4_rows_kernel<128, T>, grid, block, s, a);
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
      std::vector<W4Place> place((size_t)kTile * kChunk);
      for (int n = 0; n < kTile; ++n)
        for (int k = 0; k < kChunk; ++k) place[n * kChunk + k] = w4_place(n, k, G);
      for (int n = 0; n < N; ++n) {
        const size_t tile = n / kTile;
        const W4Place *pl = &place[(size_t)(n % kTile) * kChunk];
        for (int g = 0; g < groups; ++g) {
          int sum = 0;
          for (int k = g * G; k < std::min(K, (g + 1) * G); ++k) {
            const int q = m->codes[(size_t)n * K + k];
            const W4Place w = pl[k % kChunk];
            img[(tile * m->chunks + k / kChunk) * 1024 + w.byte] |= (uint8_t)((q & 15) << (w.high ? 4 : 0));
            sum += q;
          }
          s[tile * per_tile + (size_t)g * kTile + n % kTile] = m->scales[(size_t)n * groups + g] / 16;
          sums[tile * per_tile + (size_t)g * kTile + n % kTile] = (int16_t)(16 * sum);
        }
        if (m->bias) reinterpret_cast<float *>(img.data() + m->o_bias)[n] = p->bias[n];
      }
      const DeviceScope scope(device);
      if (!scope.ok) rc = LSTM_INT_E_DEVICE;
      else if (hipMalloc(reinterpret_cast<void **>(&m->base), img.size()) != hipSuccess) {
        m->base = nullptr;
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
  while (a.split < 8 && a.split * 2 <= a.chunks && (int64_t)a.tiles * ((rows + 15) / 16) * a.split < 4096) a.split *= 2;
  const DeviceScope scope(m->device);
  if (!scope.ok) return LSTM_INT_E_DEVICE;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  return dtype == LM_F32 ? launch_rows<float>(a, m->group, s)
                         : dtype == LM_F16 ? launch_rows<_Float16>(a, m->group, s) : launch_rows<__bf16>(a, m->group, s);
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
