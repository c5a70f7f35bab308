// What the attention kernels with roles share.
#pragma once

#include <cuda_fp16.h>

#include "paged.h"
#include "umma.cuh"

namespace spla {

// Warp-uniform bounded wait that also ends when another role has given up.
__device__ __forceinline__ bool pm_wait_slow(uint64_t* bar, uint32_t parity, int limit, volatile int* abort_flag) {
  if (limit <= 0) limit = kWaitLimitDefault;
  for (int it = 0; it < limit; ++it) {
    if (__all_sync(0xffffffffu, mbar_wait(bar, parity, 1))) return true;
    if (it > 64) __nanosleep(64);
    if ((it & 63) == 63 && warp_aborted(abort_flag)) return false;
  }
  return false;
}
__device__ __forceinline__ bool pm_wait(uint64_t* bar, uint32_t parity, int limit, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, 1)) || pm_wait_slow(bar, parity, limit, abort_flag);
}

constexpr float kCapNear = 0.375f;                 // up to here tanh goes by a polynomial: u (c0 + c1 u^2 + c2 u^4 + c3 u^6), interpolated at Chebyshev nodes, 6e-8 off
constexpr float kTanh0 = 0.99999994f, kTanh1 = -0.33331972f, kTanh2 = 0.13284431f, kTanh3 = -0.048268907f;
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// The smaller one, NaN if either is.
__device__ __forceinline__ float min_or_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Four e4m3 values as two pairs of fp16.
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// bits a .. e - 1 of a word (a, e in any range)
__device__ __forceinline__ uint32_t bits_between(int a, int e) {
  const uint32_t below_e = e >= 32 ? 0xffffffffu : e <= 0 ? 0u : (1u << e) - 1u;
  const uint32_t below_a = a >= 32 ? 0xffffffffu : a <= 0 ? 0u : (1u << a) - 1u;
  return below_e & ~below_a;
}

}  // namespace spla
