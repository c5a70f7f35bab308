// What the kernels that rotate heads share: a thread's piece of a head, its loads and stores, sines and cosines.
#pragma once

#include <cuda_fp8.h>

#include "paged.h"

namespace spla {

// VEC channels as they lie: VEC x sizeof(T) = 16 bytes, or one channel.
__device__ __forceinline__ void load_raw(const void* p, uint32_t (&w)[4]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
__device__ __forceinline__ void load_raw(const float* p, uint32_t (&w)[1]) { w[0] = *reinterpret_cast<const uint32_t*>(p); }
__device__ __forceinline__ void load_raw(const __nv_bfloat16* p, uint32_t (&w)[1]) { w[0] = *reinterpret_cast<const uint16_t*>(p); }
template <typename T, int VEC, int W>
__device__ __forceinline__ void unpack(const uint32_t (&w)[W], float (&x)[VEC]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = __uint_as_float(w[i]);
  } else if constexpr (VEC == 1) {
    x[0] = bf16_lo(w[0]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
  }
}
template <int VEC>
__device__ __forceinline__ void store_piece(float* p, const float (&x)[VEC]) {
  if constexpr (VEC == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = x[i];
  }
}
template <int VEC>
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, const float (&x)[VEC]) {
  if constexpr (VEC == 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = __float2bfloat16_rn(x[i]);
  }
}

// Angle of a position: sine and cosine of 2 pi frac(position x freq).
__device__ __forceinline__ float2 turn_of(unsigned long long freq, int position, float amplitude, bool back) {
  const unsigned long long phase = (unsigned long long)(long long)position * freq;
  const float half_turns = (float)(int)(phase >> 32) * (1.f / 2147483648.f);       // [-1, 1]
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c * amplitude, (back ? -s : s) * amplitude);
}

// The VEC pairs of a thread's piece, turned.  a, b: its two runs of VEC channels (pair i is (a_i, b_i), or where neighbours are paired
// (a_0, a_1), (a_2, a_3), .. (b_0, b_1), ..); tab: the sines of its first two pairs, the next two `stride` further.
template <int VEC>
__device__ __forceinline__ void turn_piece(float* a, float* b, const float4* tab, int stride, bool interleaved) {
#pragma unroll
  for (int j = 0; j < VEC / 2; ++j) {
    const float4 cs = tab[j * stride];
    if (interleaved) {                                     // a then b hold neighbouring pairs (x, y), (x, y), ...
      float* v = 4 * j < VEC ? a + 4 * j : b + 4 * j - VEC;
      const float x0 = v[0], y0 = v[1], x1 = v[2], y1 = v[3];
      v[0] = x0 * cs.x - y0 * cs.y; v[1] = y0 * cs.x + x0 * cs.y;
      v[2] = x1 * cs.z - y1 * cs.w; v[3] = y1 * cs.z + x1 * cs.w;
    } else {
      const float x0 = a[2 * j], y0 = b[2 * j], x1 = a[2 * j + 1], y1 = b[2 * j + 1];
      a[2 * j] = x0 * cs.x - y0 * cs.y; b[2 * j] = y0 * cs.x + x0 * cs.y;
      a[2 * j + 1] = x1 * cs.z - y1 * cs.w; b[2 * j + 1] = y1 * cs.z + x1 * cs.w;
    }
  }
}

// ---- a row: one head of one token, held by `width` neighbouring lanes ---------------------------------------------------
// Wide: VEC pairs a lane (two runs of 16 bytes), as above.
template <typename T, int VEC>
struct WideRow {
  static constexpr int CH = 2 * VEC, WORDS = 8;             // channels of a lane; 32-bit words that they come in
  int ca, cb, piece, rot_pieces;
  bool here, turns, interleaved;
  __device__ __forceinline__ WideRow(const RopeTable& rt, int lane_of_row) {
    const int pairs = rt.rot / 2;
    rot_pieces = pairs / VEC;
    piece = lane_of_row;
    here = piece < rt.dim / CH;
    turns = piece < rot_pieces;
    interleaved = rt.interleaved != 0;
    if (!turns) { ca = rt.rot + (piece - rot_pieces) * 2 * VEC; cb = ca + VEC; }
    else if (interleaved) { ca = piece * 2 * VEC; cb = ca + VEC; }
    else { ca = piece * VEC; cb = ca + pairs; }
  }
  __device__ __forceinline__ int channel(int i) const { return i < VEC ? ca + i : cb + i - VEC; }
  __device__ __forceinline__ void load(const T* row, uint32_t (&w)[WORDS]) const {
    load_raw(row + ca, *reinterpret_cast<uint32_t(*)[4]>(w));
    load_raw(row + cb, *reinterpret_cast<uint32_t(*)[4]>(w + 4));
  }
  __device__ __forceinline__ void values(const uint32_t (&w)[WORDS], float (&x)[CH]) const {
    unpack<T, VEC>(*reinterpret_cast<const uint32_t(*)[4]>(w), *reinterpret_cast<float(*)[VEC]>(x));
    unpack<T, VEC>(*reinterpret_cast<const uint32_t(*)[4]>(w + 4), *reinterpret_cast<float(*)[VEC]>(x + VEC));
  }
  __device__ __forceinline__ void weights(const float* w, float (&y)[CH]) const {   // (shared memory)
#pragma unroll
    for (int i = 0; i < CH; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(w + (here ? channel(i) : 0));
      y[i] = v.x; y[i + 1] = v.y; y[i + 2] = v.z; y[i + 3] = v.w;
    }
  }
  // Pair i into a token's table of sines: two pairs' cosines, then their sines; the pieces side by side, so that a warp's loads are contiguous.
  static __device__ __forceinline__ void put(float2* table, int i, int pairs, float2 cs) {
    const int pc = i / VEC, j = i % VEC;
    float* at = reinterpret_cast<float*>(table) + ((j >> 1) * (pairs / VEC) + pc) * 4 + (j & 1);
    at[0] = cs.x;
    at[2] = cs.y;
  }
  __device__ __forceinline__ void turn(float (&x)[CH], const float2* table, float*) const {   // two pairs at a time
    if (!turns) return;
    const float4* tab = reinterpret_cast<const float4*>(table) + piece;
    if (interleaved) {
#pragma unroll
      for (int j = 0; j < VEC / 2; ++j) two(tab[j * rot_pieces], x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
    } else {
#pragma unroll
      for (int j = 0; j < VEC / 2; ++j) two(tab[j * rot_pieces], x[2 * j], x[VEC + 2 * j], x[2 * j + 1], x[VEC + 2 * j + 1]);
    }
  }
  static __device__ __forceinline__ void two(float4 cs, float& a0, float& b0, float& a1, float& b1) {
    const float2 c = make_float2(cs.x, cs.y), s = make_float2(cs.z, cs.w), a = make_float2(a0, a1), b = make_float2(b0, b1);
    const float2 y = __ffma2_rn(make_float2(-b.x, -b.y), s, __fmul2_rn(a, c)), z = __ffma2_rn(a, s, __fmul2_rn(b, c));
    a0 = y.x; a1 = y.y; b0 = z.x; b1 = z.y;
  }
  __device__ __forceinline__ void store(T* row, const float (&x)[CH]) const {
    store_piece<VEC>(row + ca, *reinterpret_cast<const float(*)[VEC]>(x));
    store_piece<VEC>(row + cb, *reinterpret_cast<const float(*)[VEC]>(x + VEC));
  }
};

// Any address and any rotated part: a warp holds a row, lane l its channels l, l + 32, ...; partners meet in shared memory.
template <typename T, int N>
struct LooseRow {
  static constexpr int CH = N, WORDS = N;
  int lane, dim, rot;
  bool here, interleaved;
  __device__ __forceinline__ LooseRow(const RopeTable& rt, int lane_of_row) : lane(lane_of_row), dim(rt.dim), rot(rt.rot), here(true), interleaved(rt.interleaved != 0) {}
  __device__ __forceinline__ int channel(int i) const { return lane + 32 * i; }
  __device__ __forceinline__ void load(const T* row, uint32_t (&w)[WORDS]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      w[i] = 0u;
      if (channel(i) < dim) load_raw(row + channel(i), *reinterpret_cast<uint32_t(*)[1]>(w + i));
    }
  }
  __device__ __forceinline__ void values(const uint32_t (&w)[WORDS], float (&x)[CH]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) unpack<T, 1>(*reinterpret_cast<const uint32_t(*)[1]>(w + i), *reinterpret_cast<float(*)[1]>(x + i));
  }
  __device__ __forceinline__ void weights(const float* w, float (&y)[CH]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = channel(i) < dim ? w[channel(i)] : 0.f;
  }
  static __device__ __forceinline__ void put(float2* table, int i, int, float2 cs) { table[i] = cs; }
  __device__ __forceinline__ void turn(float (&x)[CH], const float2* table, float* row) const {   // whole warps; row: its own dim floats
    const int pairs = rot / 2;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (channel(i) < rot) row[channel(i)] = x[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = channel(i);
      if (c >= rot) continue;
      const bool second = interleaved ? c & 1 : c >= pairs;
      const float2 cs = table[interleaved ? c >> 1 : second ? c - pairs : c];
      const float other = row[interleaved ? c ^ 1 : second ? c - pairs : c + pairs];
      x[i] = second ? x[i] * cs.x + other * cs.y : x[i] * cs.x - other * cs.y;
    }
  }
  __device__ __forceinline__ void store(T* row, const float (&x)[CH]) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (channel(i) < dim) store_piece<1>(row + channel(i), *reinterpret_cast<const float(*)[1]>(x + i));
  }
};

// Sum over the `width` neighbouring lanes of a row (a power of two); the same in all of them.
__device__ __forceinline__ float row_sum(float v, int width) {
  if (width == 8) {                                         // (the usual one)
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  } else {
#pragma unroll 1
    for (int o = width >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  return v;
}
// 1 / sqrt(mean x^2 + eps)
template <int CH>
__device__ __forceinline__ float row_rms(const float (&x)[CH], int width, float per_channel, float eps) {
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < CH; i += 2) s = __ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(x[i], x[i + 1]), s);
  return rsqrtf(fmaf(row_sum(s.x + s.y, width), per_channel, eps));
}
// x = x f w
template <int CH>
__device__ __forceinline__ void row_scale(float (&x)[CH], float f, const float (&w)[CH]) {
#pragma unroll
  for (int i = 0; i < CH; i += 2) {
    const float2 y = __fmul2_rn(__fmul2_rn(make_float2(x[i], x[i + 1]), make_float2(f, f)), make_float2(w[i], w[i + 1]));
    x[i] = y.x;
    x[i + 1] = y.y;
  }
}

// Sines and cosines of nt tokens for the rows of class ROW, by all threads of the CTA: table[t * pairs ..].  `position`: of token t.
template <class ROW, typename F>
__device__ __forceinline__ void fill_turns(const RopeTable& rt, float2* table, int nt, int tid, int threads, bool back, F position) {
  const unsigned long long* freq = rt.freq;
  asm("" : "+l"(freq));                                     // (an ordinary load: a constant one takes a turn per thread)
  const int pairs = rt.rot / 2;
  for (int x = tid; x < nt * pairs; x += threads) {
    const int t = x / pairs, i = x - t * pairs;
    ROW::put(table + t * pairs, i, pairs, turn_of(freq[i], position(t), rt.amplitude, back));
  }
}

// Whether the wide rows serve this rotation (the addresses are the caller's to check).
inline bool wide_rotation(const RopeTable& rt, int elem) {
  const int two = 32 / elem;                                // channels of a lane
  return rt.dim % two == 0 && rt.rot % two == 0;
}
inline bool wide_strides(const void* p, int elem, long long s0, long long s1, long long s2) {
  const long long v = 16 / elem;
  return (uintptr_t)p % 16 == 0 && s0 % v == 0 && s1 % v == 0 && s2 % v == 0;
}

}  // namespace spla
