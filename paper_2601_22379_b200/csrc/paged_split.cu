// What comes before the tensor-core attention over 8-bit pages: queries as two parts of 8 bits, or keys and values in bf16.
//
// Queries: bf16 rows as two parts of 8 bits, whose products with e4m3 keys are the row's own.
//
// A row is scaled by a power of two, so that its largest magnitude is in [128, 256); the first part is each channel rounded to e4m3, which takes the first four
// of bf16's eight bits, the second what that leaves, as e5m2: three bits and a sign, all there is left down to 2^-14 of the row's largest channel,
// within 2^-21 of it below.  Bound by memory: 4 bytes in and out per channel (8192 tokens, 32 heads of 128: 134 MB).
// Keys and values: e4m3 times a power of two is exact in bf16.  Three bytes a value, 0.14 ns for a token and KV head of 128.  Where a call has many rows for each key this is little
// beside what the kernel for bf16 pages does faster: no widening on the way, no scales in the softmax, one product of queries and keys for two.
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


// Cached tokens of the sequences that have new ones, as bf16 pages of 128 tokens and their page table.  With a window: the tiles of the sinks (`first` of
// them) and those from the first token's window on, which is all that any row walks.  Block (page, head).  The rows behind the end stay as they are.
template <int D>
__global__ void __launch_bounds__(kSplitThreads) paged_widen_kernel(const __grid_constant__ PagedBatch pb, const __grid_constant__ PagedLayout pl,
                                                                    const __grid_constant__ PagedPages pages, int cols, int slots, int first, int window,
                                                                    __nv_bfloat16* k, __nv_bfloat16* v, int* table) {
  constexpr int PIECES = D / 16, EACH = kWidePage * PIECES / kSplitThreads;       // of a row; of a thread
  __shared__ long long rows[kWidePage / 16];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, b = blockIdx.x / slots, slot = blockIdx.x - b * slots, h = blockIdx.y;
  const PagedSeq s = paged_seq(pb, pl.status, b);
  if (s.n == 0) return;
  const int from = window > 0 ? max(0, s.L - s.n - window + 1) / kWidePage : 0;    // the first tile of a window
  const int tile = slot < first ? slot : max(from, first) + slot - first, tok0 = tile * kWidePage;
  if (tok0 >= s.L) return;
  if (tid == 0 && h == 0) table[(long long)b * cols + tile] = blockIdx.x;
  if (tid < kWidePage >> pl.log_p && tok0 + (tid << pl.log_p) < s.L) rows[tid] = paged_row(pb, pl, b, h, (tok0 >> pl.log_p) + tid);
  __syncthreads();
  uint4 w[2][EACH];
  float mul[2][EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int piece = tid + x * kSplitThreads, r = piece / PIECES, c = piece % PIECES * 16;
    long long row = tok0 + r < s.L ? rows[r >> pl.log_p] : -1;
    if (row >= 0) row += r & (pl.P - 1);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      w[y][x] = make_uint4(0u, 0u, 0u, 0u);                                        // (a page number outside the pool: zeros)
      mul[y][x] = 1.f;
      if (row >= 0) {
        w[y][x] = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(y ? pages.v : pages.k) + row * D + c);
        mul[y][x] = paged_scale(y ? pages.v_scales : pages.k_scales, row);
      }
    }
  }
  const long long row0 = ((long long)blockIdx.x * pl.Hkv + h) * kWidePage;
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const int piece = tid + x * kSplitThreads, r = piece / PIECES, c = piece % PIECES * 16;
    if (tok0 + r >= s.L) continue;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t from[4] = {w[y][x].x, w[y][x].y, w[y][x].z, w[y][x].w};
      uint32_t to[8];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        uint32_t lo, hi;
        widen(from[z], lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), e = __half22float2(*reinterpret_cast<const __half2*>(&hi));
        to[2 * z] = pack_bf16(a.x * mul[y][x], a.y * mul[y][x]);
        to[2 * z + 1] = pack_bf16(e.x * mul[y][x], e.y * mul[y][x]);
      }
      uint4* at = reinterpret_cast<uint4*>((y ? v : k) + (row0 + r) * D + c);
      at[0] = make_uint4(to[0], to[1], to[2], to[3]);
      at[1] = make_uint4(to[4], to[5], to[6], to[7]);
    }
  }
}

}  // namespace

PagedWide paged_wide(const PagedLayout& pl, const PagedBatch& pb, int window, int sinks) {
  PagedWide w = {};
  w.cols = (pb.max_len + kWidePage - 1) / kWidePage;
  w.first = window > 0 ? (int)(((long long)sinks + kWidePage - 1) / kWidePage) : 0;
  const long long reach = w.first + ((long long)pb.max_new + window - 1 + kWidePage - 1) / kWidePage + 1;   // tiles of the sinks, of the window of all new tokens
  w.slots = window > 0 && reach < w.cols ? (int)reach : w.cols;
  const long long pages = (long long)pb.batch * w.slots;
  const size_t tokens = (size_t)pages * pl.Hkv * kWidePage;
  w.pl = pl;
  w.pl.P = kWidePage;
  w.pl.log_p = 7;
  static_assert(kWidePage == 1 << 7, "tokens of a page");
  w.pl.n_pages = (int)pages;
  w.pl.page_stride = (long long)pl.Hkv * kWidePage;
  w.pl.head_stride = kWidePage;
  w.v_at = tokens * pl.d * 2;
  w.table_at = 2 * w.v_at;
  w.bytes = w.table_at + (size_t)pb.batch * w.cols * 4;
  w.fits = (double)pages * pl.Hkv * kWidePage < 2147483392.0;                      // (2^31 - 256)
  return w;
}

cudaError_t launch_paged_widen(const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, const PagedWide& w, int window, void* to, cudaStream_t s) {
  unsigned char* at = reinterpret_cast<unsigned char*>(to);
  return launch_ex(pl.d == 128 ? paged_widen_kernel<128> : paged_widen_kernel<64>, dim3((unsigned)w.pl.n_pages, (unsigned)pl.Hkv), dim3(kSplitThreads), 0, s, 0, true, pb, pl,
                   pages, w.cols, w.slots, w.first, window, (__nv_bfloat16*)at, (__nv_bfloat16*)(at + w.v_at), (int*)(at + w.table_at));
}

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
