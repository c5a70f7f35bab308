// Queries for the tensor-core attention over 8-bit pages: bf16 rows as two parts of 8 bits, whose products with e4m3 keys are the row's own.
//
// A row is scaled by a power of two, so that its largest magnitude is in [128, 256); the first part is each channel rounded to e4m3, which takes the first four
// of bf16's eight bits, the second what that leaves, as e5m2: three bits and a sign, all there is left down to 2^-14 of the row's largest channel,
// within 2^-21 of it below.  Bound by memory: 4 bytes in and out per channel (a prompt of 8192 tokens, 32 heads of 128: @split).
#include <cuda_fp8.h>

#include "paged_tiles.cuh"

namespace spla {

namespace {

// Four bf16 values times `mul` (a power of two) as four e4m3 and, of what that leaves, four e5m2.  An infinity is left to the second type, which has one.
__device__ __forceinline__ void split_e4m3(uint32_t w0, uint32_t w1, float mul, bool finite, uint32_t& first, uint32_t& second) {
  float x[4] = {bf16_lo(w0) * mul, bf16_hi(w0) * mul, bf16_lo(w1) * mul, bf16_hi(w1) * mul};
  uint32_t infinite = 0u;
  if (!finite)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (fabsf(x[i]) == INFINITY) {
        infinite |= (x[i] > 0.f ? 0x7cu : 0xfcu) << (8 * i);
        x[i] = 0.f;
      }
  const uint32_t h = __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3) |
                     (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2], x[3]), __NV_SATFINITE, __NV_E4M3) << 16;
  uint32_t lo, hi;
  widen(h, lo, hi);
  first = h;
  second = infinite | __nv_cvt_float2_to_fp8x2(make_float2(x[0] - __low2float(*reinterpret_cast<const __half2*>(&lo)), x[1] - __high2float(*reinterpret_cast<const __half2*>(&lo))), __NV_SATFINITE, __NV_E5M2) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2] - __low2float(*reinterpret_cast<const __half2*>(&hi)), x[3] - __high2float(*reinterpret_cast<const __half2*>(&hi))), __NV_SATFINITE, __NV_E5M2) << 16;
}
constexpr int kSplitThreads = 256;
template <int D>
__global__ void __launch_bounds__(kSplitThreads) paged_split_kernel(const __nv_bfloat16* q, long long q_stride, int Hq, long long rows, unsigned char* parts, signed char* exps) {
  constexpr int LANES = D / 8, AT_ONCE = kSplitThreads / LANES, ROWS = 4;        // of a row; rows of a block at once, and one after the other
  pdl_wait();
  pdl_launch_dependents();
  const int l = threadIdx.x % LANES;
  const long long first = (long long)blockIdx.x * (AT_ONCE * ROWS) + threadIdx.x / LANES;
  uint4 v[ROWS];
#pragma unroll
  for (int x = 0; x < ROWS; ++x) {
    const long long r = first + x * AT_ONCE;
    v[x] = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows) v[x] = *reinterpret_cast<const uint4*>(q + r / Hq * q_stride + (r % Hq) * D + l * 8);
  }
#pragma unroll
  for (int x = 0; x < ROWS; ++x) {
    const long long r = first + x * AT_ONCE;
    const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
    float top = 0.f;
    bool finite = true;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float lo = fabsf(bf16_lo(w[y])), hi = fabsf(bf16_hi(w[y]));
      if (lo < INFINITY) top = fmaxf(top, lo); else finite = false;
      if (hi < INFINITY) top = fmaxf(top, hi); else finite = false;
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int e = top > 0.f ? max((__float_as_int(top) >> 23) - 127 - 7, -100) : 0;
    const float mul = power_of_two(-e);
    uint2 a, b;
    split_e4m3(w[0], w[1], mul, finite, a.x, b.x);
    split_e4m3(w[2], w[3], mul, finite, a.y, b.y);
    if (r < rows) {
      *reinterpret_cast<uint2*>(parts + r * (2 * D) + l * 8) = a;
      *reinterpret_cast<uint2*>(parts + r * (2 * D) + D + l * 8) = b;
      if (l == 0) exps[r] = (signed char)e;
    }
  }
}

}  // namespace

size_t paged_split_bytes(const PagedLayout& pl, int total_new, size_t* exps) {
  const size_t rows = (size_t)total_new * pl.Hq;
  *exps = rows * 2 * pl.d;                                                         // (their place: behind the parts)
  return rows * 2 * pl.d + rows;
}

cudaError_t launch_paged_split(const PagedLayout& pl, const void* q, long long q_stride, int total_new, unsigned char* parts, signed char* exps, cudaStream_t s) {
  const long long rows = (long long)total_new * pl.Hq;
  const int at_once = kSplitThreads / (pl.d / 8) * 4;
  return launch_ex(pl.d == 128 ? paged_split_kernel<128> : paged_split_kernel<64>, dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(kSplitThreads), 0, s, 0, true,
                   (const __nv_bfloat16*)q, q_stride, pl.Hq, rows, parts, exps);
}

}  // namespace spla
