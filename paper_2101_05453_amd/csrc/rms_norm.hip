// Root-mean-square norm into int8 codes (include/lm_ops.h).
//
//   r = x + residual;  n = r / sqrt(mean(r^2) + eps) * weight [* gate * sigma(gate)];  codes = floor(n / s + 1/2)
//
// One pass over memory: a row stays in the registers of one, four or sixteen waves, eight neighbouring columns ("a chunk")
// per lane and slot, as it lies in memory, from its load to the store of its codes.  What is summed and compared is double
// precision: the products are then exact enough that a code at the border between two is the one of the definition.
#include "lm_common.h"

namespace lstm_int {
namespace {

// A half and a little: the square root cancels in n / s, so that values half way between two codes do occur (a row whose
// largest is 127, say); n / s is right to 2^-45, and what is half way goes up.
constexpr double kHalf = 0.5 + 0x1p-40;

constexpr int kSlots = 4;  // chunks per lane: 2048 columns per wave

struct NormArgs {
  const void *x, *residual, *gate;
  const float *weight;
  int8_t *codes;
  float *scales;
  void *y, *new_residual;
  int64_t x_stride, residual_stride, gate_stride, new_residual_stride;
  int rows, cols, groups, D;
  int lanes, per_group;  // groups > 1: a group takes `lanes` (a power of two) lanes and per_group slots of them
  int slots;
  int zero_point;
  double eps, scale, inv_d;
};

__device__ inline double shfl_xor_d(double v, int mask) {
  union { double d; int i[2]; } a, b;
  a.d = v;
  b.i[0] = __shfl_xor(a.i[0], mask);
  b.i[1] = __shfl_xor(a.i[1], mask);
  return b.d;
}

template <class T, int kWaves, bool kGate>
__global__ __launch_bounds__(kWaves == 16 ? 1024 : 256) void rms_norm_kernel(NormArgs a) {
  constexpr int kBlockWaves = kWaves == 16 ? 16 : 4;
  __shared__ double part[2][kBlockWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % kWaves;
  const int64_t row_at = (int64_t)blockIdx.x * (kBlockWaves / kWaves) + wave / kWaves;
  const bool live = row_at < a.rows;
  const int64_t row = live ? row_at : a.rows - 1;  // waves behind the last row follow it and store nothing
  const bool whole = a.groups == 1;

  int col[kSlots], count[kSlots], first[kSlots];  // first: the chunk's column within its group
  bool last[kSlots];                              // the last slot of a group
  {
    int it = 0, c = 0;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      int group, chunk;
      if (whole) {
        group = 0;
        chunk = (s * kWaves + w) * 64 + lane;
        last[s] = s == kSlots - 1;
      } else {
        group = (it * kWaves + w) * (64 / a.lanes) + lane / a.lanes;
        chunk = c * a.lanes + lane % a.lanes;
        last[s] = c == a.per_group - 1;
        if (++c == a.per_group) c = 0, ++it;
      }
      first[s] = chunk * 8;
      col[s] = group * a.D + chunk * 8;
      count[s] = s < a.slots && group < a.groups ? max(0, min(8, a.D - chunk * 8)) : 0;
    }
  }

  const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_stride : nullptr;
  Raw8<T> rx[kSlots], rr[kSlots], rg[kGate ? kSlots : 1];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (count[s] > 0) rx[s].load(x + col[s], count[s]);
    if (count[s] > 0 && res) rr[s].load(res + col[s], count[s]);
    if constexpr (kGate)
      if (count[s] > 0) rg[s].load(static_cast<const T *>(a.gate) + row * a.gate_stride + col[s], count[s]);
  }

  double n[kSlots][8], inv[kSlots], sum = 0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (count[s] > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // elements behind the end are zeros
        double r = (double)(float)rx[s].e[i];
        if (res) r += (double)(float)rr[s].e[i];
        n[s][i] = r;
        sum = __builtin_fma(r, r, sum);
      }
    }
    inv[s] = 0;
    if (!whole && last[s]) {
      for (int m = a.lanes >> 1; m > 0; m >>= 1) sum += shfl_xor_d(sum, m);
      inv[s] = 1.0 / sqrt(sum * a.inv_d + a.eps);
      sum = 0;
    }
  }
  if (whole) {
    for (int m = 32; m > 0; m >>= 1) sum += shfl_xor_d(sum, m);
    if constexpr (kWaves > 1) {
      if (lane == 0) part[0][wave] = sum;
      __syncthreads();
      sum = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) sum += part[0][wave - w + i];
    }
    const double v = 1.0 / sqrt(sum * a.inv_d + a.eps);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) inv[s] = v;
  } else {
#pragma unroll
    for (int s = kSlots - 2; s >= 0; --s)
      if (!last[s]) inv[s] = inv[s + 1];
  }

  if (live && a.new_residual) {
    T *out = static_cast<T *>(a.new_residual) + row * a.new_residual_stride;
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
      if (count[s] > 0) {
        Raw8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.e[i] = (T)(float)n[s][i];
        o.store(out + col[s], count[s]);
      }
  }

  double most = 0;
  bool bad = false;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (count[s] <= 0) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= count[s]) continue;
      double v = n[s][i] * inv[s] * (double)a.weight[first[s] + i];
      if constexpr (kGate) {
        const double z = (double)(float)rg[s].e[i];
        v *= z / (1.0 + exp(-z));
      }
      n[s][i] = v;
      bad |= !__builtin_isfinite(v);
      most = fmax(most, fabs(v));
    }
  }

  if (live && a.y) {
    T *y = static_cast<T *>(a.y) + row * a.cols;
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
      if (count[s] > 0) {
        Raw8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.e[i] = (T)(float)n[s][i];
        o.store(y + col[s], count[s]);
      }
  }
  if (!a.codes) return;

  double mul = 0, div = a.scale;
  if (a.scale == 0) {
    if (bad) most = __builtin_inf();
    for (int m = 32; m > 0; m >>= 1) most = fmax(most, shfl_xor_d(most, m));
    if constexpr (kWaves > 1) {
      if (lane == 0) part[1][wave] = most;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) most = fmax(most, part[1][wave - w + i]);
    }
    bad = !__builtin_isfinite(most);
    mul = most > 0 && !bad ? 127.0 / most : 0.0;
    if (live && lane == 0 && w == 0) a.scales[row] = bad ? __builtin_nanf("") : (float)(most / 127.0);
  }
  if (!live) return;
  int8_t *codes = a.codes + row * a.cols;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (count[s] <= 0) continue;
    union { int8_t q[8]; u32x2_any v; } o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double v;
      if (a.scale == 0) {
        v = bad ? 0.0 : floor(n[s][i] * mul + kHalf);
      } else {
        v = floor(n[s][i] / div + 0.5) + a.zero_point;
        v = v != v ? 0.0 : fmin(fmax(v, -128.0), 127.0);
      }
      o.q[i] = (int8_t)(int)v;
    }
    if (count[s] == 8) {
      *reinterpret_cast<u32x2_any *>(codes + col[s]) = o.v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count[s]) codes[col[s] + i] = o.q[i];
    }
  }
}

template <class T, int kWaves>
int launch_norm(const NormArgs &a, hipStream_t s) {
  constexpr int threads = kWaves == 16 ? 1024 : 256, per_block = threads / 64 / kWaves;
  const dim3 grid((a.rows + per_block - 1) / per_block);
  return a.gate ? launch(rms_norm_kernel<T, kWaves, true>, grid, dim3(threads), s, a)
                : launch(rms_norm_kernel<T, kWaves, false>, grid, dim3(threads), s, a);
}

template <class T>
int launch_norm(const NormArgs &a, int waves, hipStream_t s) {
  return waves == 1 ? launch_norm<T, 1>(a, s) : waves == 4 ? launch_norm<T, 4>(a, s) : launch_norm<T, 16>(a, s);
}

// Slots that a row takes with `waves` waves
int slots_of(const NormArgs &a, int waves) {
  const int chunks = (a.D + 7) / 8;
  if (a.groups == 1) return (chunks + 64 * waves - 1) / (64 * waves);
  const int at_once = waves * (64 / a.lanes);
  return (a.groups + at_once - 1) / at_once * a.per_group;
}

}  // namespace
}  // namespace lstm_int

using namespace lstm_int;

extern "C" int rms_norm_forward(int32_t device, const rms_norm_args *p, const void *x, const void *residual, const void *gate,
                                const float *weight, int8_t *codes, float *scales, void *y, void *new_residual, void *hip_stream) {
  if (!p || device < 0 || p->rows < 0 || p->cols < 0 || p->groups < 1 || p->cols % p->groups || !lm_type_bytes(p->dtype))
    return LSTM_INT_E_INVALID_ARG;
  if (!(p->eps > 0) || !__builtin_isfinite(p->eps) || !(p->scale >= 0) || !__builtin_isfinite(p->scale)) return LSTM_INT_E_BAD_RANGE;
  if (p->rows == 0 || p->cols == 0) return LSTM_INT_OK;
  if (!x || !weight || (!codes && !y) || (codes && p->scale == 0 && !scales) || (new_residual && !residual)) return LSTM_INT_E_INVALID_ARG;
  if (p->zero_point < -128 || p->zero_point > 127) return LSTM_INT_E_INVALID_ARG;
  if (p->rows > 1 && (p->x_stride < p->cols || (residual && p->residual_stride < p->cols) || (gate && p->gate_stride < p->cols) ||
                      (new_residual && p->new_residual_stride < p->cols)))
    return LSTM_INT_E_INVALID_ARG;
  const int D = p->cols / p->groups;
  if (p->rows > INT32_MAX || p->cols > 32768 || (p->groups > 1 && (p->cols > 8192 || D < 8 || D > 2048))) return LSTM_INT_E_UNSUPPORTED;

  NormArgs a{};
  a.x = x; a.residual = residual; a.gate = gate; a.weight = weight;
  a.codes = codes; a.scales = scales; a.y = y; a.new_residual = new_residual;
  a.x_stride = p->x_stride; a.residual_stride = p->residual_stride; a.gate_stride = p->gate_stride;
  a.new_residual_stride = p->new_residual_stride;
  a.rows = (int)p->rows; a.cols = p->cols; a.groups = p->groups; a.D = D;
  a.zero_point = p->zero_point; a.eps = p->eps; a.scale = p->scale; a.inv_d = 1.0 / a.D;
  const int chunks = (a.D + 7) / 8;
  a.lanes = 1;
  while (a.lanes < 64 && a.lanes < chunks) a.lanes *= 2;
  a.per_group = (chunks + a.lanes - 1) / a.lanes;
  int waves = 1;
  while (waves < 16 && slots_of(a, waves) > kSlots) waves *= 4;
  // few rows: more waves for each, as long as they shorten it
  while (waves < 16 && a.rows * (int64_t)waves < 1024 && slots_of(a, waves) > 1) waves *= 4;
  a.slots = slots_of(a, waves);
  if (a.slots > kSlots) return LSTM_INT_E_UNSUPPORTED;

  const DeviceScope scope(device);
  if (!scope.ok) return LSTM_INT_E_DEVICE;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  return p->dtype == LM_F32 ? launch_norm<float>(a, waves, s)
                            : p->dtype == LM_F16 ? launch_norm<_Float16>(a, waves, s) : launch_norm<__bf16>(a, waves, s);
}
