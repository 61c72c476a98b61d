// What the operators of include/lm_ops.h share: element types, loads of any alignment, the device of a call.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lm_ops.h"

namespace lstm_int {

// The calling thread's current device is `device` while this lives, and what it was before afterwards.
struct DeviceScope {
  int prev = -1;
  bool ok = false, changed = false;
  explicit DeviceScope(int device) {
    if (device < 0 || hipGetDevice(&prev) != hipSuccess) return;
    if (prev == device) {
      ok = true;
      return;
    }
    ok = changed = hipSetDevice(device) == hipSuccess;
    if (!ok) (void)hipGetLastError();  // said by the call's code, not by a later call's
  }
  ~DeviceScope() {
    if (changed) (void)hipSetDevice(prev);
  }
};

// One launch; the code is that of this launch, not of an earlier call's error.
template <class... P, class... A>
int launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s, A... args) {
  static_assert(sizeof...(P) == sizeof...(A), "one argument for each parameter");
  return [&](P... typed) {
    void *ptrs[] = {&typed...};
    if (hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, ptrs, 0, s) == hipSuccess) return LSTM_INT_OK;
    (void)hipGetLastError();
    return LSTM_INT_E_DEVICE;
  }(args...);
}

inline int lm_type_bytes(int dtype) { return dtype == LM_F32 ? 4 : dtype == LM_F16 || dtype == LM_BF16 ? 2 : 0; }

// Vectors at addresses of element alignment only: the hardware takes them at any, in one access.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// n <= 8 of eight neighbouring elements of type T, as they lie in memory
template <class T>
struct Raw8 {
  static constexpr int kWords = sizeof(T) * 8 / 16;
  union {
    u32x4 w[kWords];
    T e[8];
  };
  __device__ void load(const T *p, int n) {
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const u32x4_any *>(p)[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : (T)0.0f;
    }
  }
  __device__ void store(T *p, int n) const {
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) reinterpret_cast<u32x4_any *>(p)[i] = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = e[i];
    }
  }
};

}  // namespace lstm_int
