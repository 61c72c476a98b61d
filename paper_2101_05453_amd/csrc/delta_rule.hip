// The gated delta rule (include/lm_ops.h).
//
//   S <- e^g S;  u = beta (v - S' k);  S <- S + k u';  y = scale S' q
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
      // a decay of zero clears the state, whatever it holds
      const float old = decay == 0.0f ? 0.0f : decay * pk[j], oldq = decay == 0.0f ? 0.0f : decay * pq[j];
      u[j] = bt * (vf[j] - nk * old);
      o[j] = nq * (oldq + nk * kq * u[j]);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) S[i][j] = __builtin_fmaf(nk * kf[i], u[j], decay == 0.0f ? 0.0f : decay * S[i][j]);
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
  if (check(p) != LSTM_INT_OK) return 0;
  return 0;
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
  return p->dtype == LM_F32 ? launch_step<float>(a, s) : p->dtype == LM_F16 ? launch_step<_Float16>(a, s) : launch_step<__bf16>(a, s);
}

}  // extern "C"
