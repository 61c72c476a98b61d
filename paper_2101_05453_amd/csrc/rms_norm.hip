// Root-mean-square norm into int8 codes (include/lm_ops.h).
//
//   r = x + residual;  n = r / sqrt(mean(r^2) + eps) * weight [* gate * sigma(gate)];  codes = floor(n / s + 1/2)
//
// One pass over memory: a row stays in the registers of one, four or sixteen waves, eight neighbouring columns ("a chunk")
// per lane and slot, as it lies in memory, from its load to the store of its codes.  A code at the border between two has
// to be the definition's, so sums of squares are double precision and n is evaluated twice: in float32 for every element,
// and in double precision for the few that this leaves open -- the row's largest, which the scale is made of, and those
// whose n / s comes out within its rounding of a border.  (In double precision throughout, 8192 x 4096 in heads of 128 with a
// gate took 129 us.)
//
// Bound by memory where it is large and plain: 8192 x 4096 bf16 with a residual 52 to 56 us, 4.5 TB/s; by vector instructions
// with a gate, 71 an element, which are active in 76 % of all cycles: the same in heads of 128, 71 us, 2.4 TB/s (without the gate
// 49); by the chain load, sum, largest, store where it is small: one row of 2048 5 us.
#include <algorithm>

#include "lm_common.h"

namespace lstm_int {
namespace {

// A half and a little: the square root cancels in n / s, so that values half way between two codes do occur (a row whose
// largest is 127, say); n / s is right to 2^-45, and what is half way goes up.
constexpr double kHalf = 0.5 + 0x1p-40;

constexpr int kMostSlots = 4;  // chunks per lane: 2048 columns per wave

// Workgroups along blockIdx.x, blockIdx.y counts on: a dimension of a launch ends at 2^32 threads
constexpr int kGridBlocks = 1 << 21;

struct NormArgs {
  const void *x, *residual, *gate;
  const float *weight;
  int8_t *codes;
  float *scales;
  void *y, *new_residual;
  int64_t x_stride, residual_stride, gate_stride, new_residual_stride;
  int rows, cols, groups, D;
  int lanes, per_group;  // a group takes `lanes` (a power of two) lanes and per_group slots of them
  int row_lanes;         // lanes of a wave that a row takes: 64, or `lanes` where a wave has several rows
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

// With a gate, five waves to a SIMD: float32, 4096 x 2048, 24.9 us; 26.4 at four, which the compiler takes by itself
template <class T, int kWaves, int kSlots, bool kGate>
__global__ __launch_bounds__(kWaves == 16 ? 1024 : 256, kWaves != 16 && kSlots == 1 && kGate ? 5 : 1) void rms_norm_kernel(NormArgs a) {
  constexpr int kBlockWaves = kWaves == 16 ? 16 : 4;
  __shared__ double part[3][kBlockWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % kWaves;
  const bool whole = a.groups == 1;
  const int row_lane = lane & (a.row_lanes - 1);
  const int64_t rows_at = ((int64_t)blockIdx.y * kGridBlocks + blockIdx.x) * (kBlockWaves / kWaves) + wave / kWaves;
  const int64_t row_at = rows_at * (64 / a.row_lanes) + lane / a.row_lanes;
  const bool live = row_at < a.rows;
  const int64_t row = live ? row_at : a.rows - 1;  // lanes behind the last row follow it and store nothing

  // a slot's chunk: its column, its column within the group, the columns it has
  struct Place {
    int col, first, count;
  };
  auto place = [&](int s) {
    int group = 0, chunk;
    if (whole) {
      chunk = (s * kWaves + w) * a.row_lanes + row_lane;
    } else {
      group = (s / a.per_group * kWaves + w) * (64 / a.lanes) + lane / a.lanes;
      chunk = s % a.per_group * a.lanes + lane % a.lanes;
    }
    return Place{group * a.D + chunk * 8, chunk * 8, s < a.slots && group < a.groups ? max(0, min(8, a.D - chunk * 8)) : 0};
  };
  Place at[kSlots];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) at[s] = place(s);

  const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_stride : nullptr;
  const T *gate = kGate ? static_cast<const T *>(a.gate) + row * a.gate_stride : nullptr;
  Raw8<T> rx[kSlots], rr[kSlots], rg[kGate ? kSlots : 1];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (at[s].count <= 0) continue;
    rx[s].load(x + at[s].col, at[s].count);
    if (res) rr[s].load(res + at[s].col, at[s].count);
    if constexpr (kGate) rg[s].load(gate + at[s].col, at[s].count);
  }

  double inv[kSlots], sum = 0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    if (at[s].count > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // elements behind the end are zeros
        double r = (double)(float)rx[s].e[i];
        if (res) r += (double)(float)rr[s].e[i];
        sum = __builtin_fma(r, r, sum);
      }
    }
    inv[s] = 0;
    if (!whole && s % a.per_group == a.per_group - 1) {
      for (int m = a.lanes >> 1; m > 0; m >>= 1) sum += shfl_xor_d(sum, m);
      inv[s] = 1.0 / sqrt(sum * a.inv_d + a.eps);
      sum = 0;
    }
  }
  if (whole) {
    for (int m = a.row_lanes >> 1; m > 0; m >>= 1) sum += shfl_xor_d(sum, m);
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
      if (s % a.per_group != a.per_group - 1) inv[s] = inv[s + 1];
  }
  auto inv_of = [&](int s) {  // s known at run time only
    double v = inv[0];
#pragma unroll
    for (int k = 1; k < kSlots; ++k)
      if (s == k) v = inv[k];
    return v;
  };
  // n in double precision, of memory again: for single elements, by their number
  auto n64 = [&](const Place &p, double iv, int i) {
    double v = (double)(float)x[p.col + i];
    if (res) v += (double)(float)res[p.col + i];
    v = v * iv * (double)a.weight[p.first + i];
    if constexpr (kGate) {
      const double z = (double)(float)gate[p.col + i];
      v *= z / (1.0 + exp(-z));
    }
    return v;
  };

  if (a.y) {
    T *y = static_cast<T *>(a.y) + row * a.cols;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (at[s].count <= 0) continue;
      Raw8<float> wt;
      Raw8<T> o;
      wt.load(a.weight + at[s].first, at[s].count);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        double v = (double)(float)rx[s].e[i];
        if (res) v += (double)(float)rr[s].e[i];
        v = v * inv[s] * (double)wt.e[i];
        if constexpr (kGate) {
          const double z = (double)(float)rg[s].e[i];
          v *= z / (1.0 + exp(-z));
        }
        o.e[i] = (T)(float)v;
      }
      if (live) o.store(y + at[s].col, at[s].count);
    }
  }

  if (a.codes) {
    // n in float32, at most ten roundings off where no product on the way leaves float32's normal range.  One that does is
    // below 2^-126, so what becomes of it is below 2^-94 and next to nothing (in_float, usable), unless its weight or gate is
    // beyond 2^16: `far` is the largest of them.
    float n[kSlots][8], far = 0;
    uint32_t largest = 0;  // bits of the largest |n|; of a NaN, if there is one
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (at[s].count <= 0) continue;
      const float iv = (float)inv[s];
      Raw8<float> wt;
      wt.load(a.weight + at[s].first, at[s].count);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v = (float)rx[s].e[i];
        if (res) v += (float)rr[s].e[i];
        v = v * iv * wt.e[i];
        far = __builtin_fmaxf(far, fabsf(wt.e[i]));
        if constexpr (kGate) {
          const float z = (float)rg[s].e[i];
          far = __builtin_fmaxf(far, fabsf(z));
          // e^-z = 2^(t + lo), t the rounded product; from 2^128 on infinity as it is, and the factor zero (lo times it is NaN)
          constexpr float kLog2e = -1.44269504f, kLow = -1.92596299e-8f, kLn2 = 0.693147181f;
          const float t = z * kLog2e, lo = __builtin_fmaf(z, kLow, __builtin_fmaf(z, kLog2e, -t));
          const float e = __builtin_amdgcn_exp2f(t);
          v *= z * __builtin_amdgcn_rcpf(1.0f + (fabsf(t) < 128.0f ? __builtin_fmaf(e, lo * kLn2, e) : e));
        }
        n[s][i] = v;
        largest = max(largest, __float_as_uint(v) & 0x7fffffffu);
      }
    }

    if (far > 0x1p16f) largest = 0x7f800000u;
    // v = n / s + 1/2 decides its floor where it is further from a border than ten roundings of it
    auto decided = [](float v) { return fabsf(v - floorf(v) - 0.5f) < __builtin_fmaf(fabsf(v), -0x1p-20f, 0.5f - 0x1p-20f); };
    static_assert(kSlots * 8 <= 32, "a bit for each element of a lane");
    int8_t *codes = a.codes + row * a.cols;
    auto store = [&](const Place &p, const int8_t q[8]) {
      if (!live) return;
      if (p.count == 8) {
        union { int8_t b[8]; u32x2_any v; } o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.b[i] = q[i];
        *reinterpret_cast<u32x2_any *>(codes + p.col) = o.v;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < p.count) codes[p.col + i] = q[i];
      }
    };
    uint32_t open = 0;  // elements whose code float32 does not decide
    if (a.scale != 0) {
      const float mul = (float)(1.0 / a.scale);
      const bool usable = mul >= 0x1p-80f && mul <= 0x1p80f && largest < 0x7f800000u;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        if (at[s].count <= 0) continue;
        int8_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float m = fabsf(n[s][i]), v = n[s][i] * mul + 0.5f, f = floorf(v);
          // beyond 512 the code is at an end whatever v is; a product below float32's normal range is next to no border
          const bool sure = usable && m <= 0x1p80f && (m >= 0x1p-80f || m == 0) && (fabsf(v) > 512.0f || decided(v));
          if (!sure && i < at[s].count) open |= 1u << (8 * s + i);
          q[i] = (int8_t)min(max((int)fminf(fmaxf(f, -512.0f), 512.0f) + a.zero_point, -128), 127);
        }
        store(at[s], q);
      }
#pragma unroll 1
      for (; open; open &= open - 1) {
        const int k = __builtin_ctz(open);
        const Place p = place(k / 8);
        const double e = floor(n64(p, inv_of(k / 8), k % 8) / a.scale + 0.5) + a.zero_point;
        if (live) codes[p.col + k % 8] = (int8_t)(e != e ? 0 : (int)fmin(fmax(e, -128.0), 127.0));
      }
    } else {
      uint32_t row_largest = largest;
      for (int m = a.row_lanes >> 1; m > 0; m >>= 1) row_largest = max(row_largest, (uint32_t)__shfl_xor((int)row_largest, m));
      if constexpr (kWaves > 1) {
        if (lane == 0) part[1][wave] = row_largest;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) row_largest = max(row_largest, (uint32_t)part[1][wave - w + i]);
      }
      // a NaN, or numbers that float32 may not hold to all their bits or that come of such: the whole row in double precision
      const float top = __uint_as_float(row_largest);
      const bool in_float = top >= 0x1p-80f && top <= 0x1p80f;
      const float from = in_float ? top * (1 - 0x1p-18f) : -1.0f;  // what may be the largest
      if (!(__uint_as_float(largest) < from))
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < at[s].count && !(fabsf(n[s][i]) < from)) open |= 1u << (8 * s + i);
      double most = 0;
#pragma unroll 1
      for (; open; open &= open - 1) {
        const int k = __builtin_ctz(open);
        const double v = fabs(n64(place(k / 8), inv_of(k / 8), k % 8));
        most = fmax(most, v <= 0x1p1020 ? v : __builtin_inf());
      }
      for (int m = a.row_lanes >> 1; m > 0; m >>= 1) most = fmax(most, shfl_xor_d(most, m));
      if constexpr (kWaves > 1) {
        if (lane == 0) part[2][wave] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) most = fmax(most, part[2][wave - w + i]);
      }
      const bool bad = !__builtin_isfinite(most);
      const double mul = most > 0 && !bad ? 127.0 / most : 0.0;
      if (live && row_lane == 0 && w == 0) a.scales[row] = bad ? __builtin_nanf("") : (float)(most / 127.0);
      const float mul32 = in_float ? (float)mul : 0.0f;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        if (at[s].count <= 0) continue;
        int8_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = __builtin_fmaf(n[s][i], mul32, 0.5f);  // in_float: within -127 .. 128
          if (i < at[s].count && !decided(v)) open |= 1u << (8 * s + i);
          q[i] = (int8_t)(in_float ? (int)floorf(v) : 0);
        }
        if (!in_float) open |= bad ? 0u : ((1u << at[s].count) - 1) << (8 * s);
        store(at[s], q);
      }
      if (bad) open = 0;
#pragma unroll 1
      for (; open; open &= open - 1) {
        const int k = __builtin_ctz(open);
        const Place p = place(k / 8);
        const double e = floor(n64(p, inv_of(k / 8), k % 8) * mul + kHalf);
        if (live) codes[p.col + k % 8] = (int8_t)(int)e;
      }
    }
  }

  // last: it may be in the place of x or of the residual
  if (live && a.new_residual) {
    T *out = static_cast<T *>(a.new_residual) + row * a.new_residual_stride;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (at[s].count <= 0) continue;
      Raw8<T> o;
      // the float32 sum: of two 16-bit numbers it is exact wherever the next rounding could see a difference
#pragma unroll
      for (int i = 0; i < 8; ++i) o.e[i] = (T)((float)rx[s].e[i] + (float)rr[s].e[i]);
      o.store(out + at[s].col, at[s].count);
    }
  }
}

template <class T, int kWaves, int kSlots>
int launch_norm(const NormArgs &a, hipStream_t s) {
  constexpr int threads = kWaves == 16 ? 1024 : 256;
  const int per_block = threads / 64 / kWaves * (64 / a.row_lanes);
  const int64_t blocks = ((int64_t)a.rows + per_block - 1) / per_block;
  const dim3 grid((unsigned)std::min<int64_t>(blocks, kGridBlocks), (unsigned)((blocks + kGridBlocks - 1) / kGridBlocks));
  return a.gate ? launch(rms_norm_kernel<T, kWaves, kSlots, true>, grid, dim3(threads), s, a)
                : launch(rms_norm_kernel<T, kWaves, kSlots, false>, grid, dim3(threads), s, a);
}

template <class T, int kWaves>
int launch_norm(const NormArgs &a, hipStream_t s) {
  return a.slots == 1 ? launch_norm<T, kWaves, 1>(a, s) : a.slots == 2 || kWaves == 1 ? launch_norm<T, kWaves, 2>(a, s)
                      : launch_norm<T, kWaves, kWaves == 1 ? 2 : kMostSlots>(a, s);
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
  // As few waves to a row as hold it.  One wave alone takes two slots at most: with four of them, and half as many waves on a
  // compute unit, 1500 and 4096 bf16 rows of 2048 take 25 and 31 us, as four waves of a slot 11 and 21 (16384 rows 66, 65).
  // Four waves do better than 16 at four slots too: 4096 and 16384 rows of 8192 65 and 240 us, by 16 waves 73 and 296.
  while (waves < 16 && slots_of(a, waves) > (waves == 1 ? 2 : kMostSlots)) waves *= 4;
  // Few rows: more waves for each, as long as they shorten it.  64 rows of 1024 7.0 us by one wave, 5.7 by four, 64 of 4096 7.3
  // by four, 6.7 by 16; 272 rows of 4096 8.0 by four, 10.0 by 16; 4096 rows of 1024 11.8 by one, 17.7 by four.
  while (waves < 16 && a.rows * (int64_t)waves < 1024 && slots_of(a, waves) > 1) waves *= 4;
  a.slots = slots_of(a, waves);
  a.row_lanes = a.groups == 1 && waves == 1 && a.slots == 1 ? a.lanes : 64;  // short rows: several to a wave (65536 x 128: 18 us, one to a wave 59)
  if (a.slots > kMostSlots) return LSTM_INT_E_UNSUPPORTED;

  const DeviceScope scope(device);
  if (!scope.ok) return LSTM_INT_E_DEVICE;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  return p->dtype == LM_F32 ? launch_norm<float>(a, waves, s)
                            : p->dtype == LM_F16 ? launch_norm<_Float16>(a, waves, s) : launch_norm<__bf16>(a, waves, s);
}
