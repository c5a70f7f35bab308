// The append to a paged cache that norms and quantises on the way, and reading cached tokens back.
//
// 8-bit pages hold e4m3 values and a power-of-two scale 2^e for every 16 tokens of a head (a block):  e is the least integer with
// max |x| <= 448 2^e over the block's tokens, between -40 and 40.  Powers of two cost no accuracy (a floating format's steps are relative), a
// value times its scale is exact in bf16, and a block that is begun in one call and grown in the next is rescaled exactly but for values
// below 2^-6 of the new scale, which lose bits at the format's end: e only grows, so that any cutting of the tokens into calls ends with the same scale.
//
// A run is the new tokens of one block: at most 16 rows of one sequence.  A CTA takes the runs that start in its rows; a warp takes a run of one
// head (or a single new token of several heads), holds it in registers, norms and turns it, finds the largest magnitude by shuffles and
// stores.  Queries go the same way without the scale.  New values are read once, written once; a block's earlier tokens are touched only when
// its scale grows.
//
// What bounds it: the first loads of a CTA come behind a search for its sequences and the page table's entries, which are dependent loads; then memory.  A prompt of 32768 tokens of 32 + 8 + 8
// heads of 128 in bf16: 166 us in a graph (112 at a copy's rate), 16384 in fp32, pages of 16: 43 (27), turns of 50 to 700 tokens x 16 61 (23), a token for each of 64
// sequences 14 (launch 8).  Steps: a body for each kind of head, so that rows without norm or turn skip them, and packed arithmetic 242 -> 164 us (prompt).
// Reading back: 131072 tokens, 8 heads of 128: 154 us (123), 32000 tokens in pages of 16 54 (30).  Norms on the way into pages of 16 and 32 bits (without them rope.cu's times, in
// brackets, then the floor): a prompt of 32768 in bf16 156 (141; 123), turns 53 (37; 23), in fp32 72 (66; 47), 16384 in fp32 in pages of 16 47 (43; 31).
#include <type_traits>

#include "rope_device.cuh"

namespace spla {

namespace {

constexpr int kStoreThreads = 256;
constexpr int kStoreTokens = 16;                           // rows of a CTA, at most: 15 more may belong to its last run
constexpr int kStoreReach = 2 * kStoreTokens;

struct StoreLaunch {
  const void *q, *k, *v;
  void* q_out;
  long long q_stride, k_stride, v_stride, q_out_stride;    // elements between tokens
  int n_q, n_kv;                                           // heads of this launch (0: not in it)
  const float *q_weight, *k_weight;                        // null: not normed
  float eps;
  const int* positions;
  int tb, heads_per_y;
  PagedBatch pb;
  PagedLayout pl;
  void *k_pages, *v_pages;
  unsigned char *k_scales, *v_scales;                      // of 8-bit pages
  int turn;
};

// Least e with top <= 448 2^e: top = m 2^x with m in [1/2, 1), 448 = 7/8 2^9.
__device__ __forceinline__ int scale_exponent(float top) {
  const int bits = __float_as_int(top), e = (bits >> 23) - 126 - 9 + ((bits & 0x7fffff) > 0x600000);
  return min(max(e, kExpMin), kExpMax);
}
// (an ordinary load: the byte is written later in the same kernel)
__device__ __forceinline__ int held_exponent(const unsigned char* p) { return min(max((int)*p - 127, kExpMin), kExpMax); }

// Two values as e4m3, to nearest, those above 448 as 448; the lower one in the lower byte.
__device__ __forceinline__ unsigned pack_e4m3(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 unpack_e4m3(unsigned two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(__half2(h));
}
// Bytes of a lane's channels: n contiguous ones.
template <int N>
__device__ __forceinline__ void store_bytes(unsigned char* p, const float* x, float mul) {
  if constexpr (N == 1) {
    *p = (unsigned char)pack_e4m3(x[0] * mul, 0.f);
  } else {
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      w[i] = pack_e4m3(x[4 * i] * mul, x[4 * i + 1] * mul) | pack_e4m3(x[4 * i + 2] * mul, x[4 * i + 3] * mul) << 16;
    if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
}
// ... rounded again to a larger scale
template <int N>
__device__ __forceinline__ void rescale_bytes(unsigned char* p, float mul) {
  if constexpr (N == 1) {
    *p = (unsigned char)pack_e4m3(unpack_e4m3(*p).x * mul, 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      uint32_t* at = reinterpret_cast<uint32_t*>(p) + i;
      const uint32_t w = *at;
      const float2 a = unpack_e4m3(w & 0xffffu), b = unpack_e4m3(w >> 16);
      *at = pack_e4m3(a.x * mul, a.y * mul) | pack_e4m3(b.x * mul, b.y * mul) << 16;
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_row8(const WideRow<T, VEC>& row, unsigned char* p, const float (&x)[2 * VEC], float mul) {
  store_bytes<VEC>(p + row.ca, x, mul);
  store_bytes<VEC>(p + row.cb, x + VEC, mul);
}
template <typename T, int VEC>
__device__ __forceinline__ void rescale_row8(const WideRow<T, VEC>& row, unsigned char* p, float mul) {
  rescale_bytes<VEC>(p + row.ca, mul);
  rescale_bytes<VEC>(p + row.cb, mul);
}
template <typename T, int N>
__device__ __forceinline__ void store_row8(const LooseRow<T, N>& row, unsigned char* p, const float (&x)[N], float mul) {
#pragma unroll
  for (int i = 0; i < N; ++i) store_bytes<1>(p + row.channel(i), x + i, mul);
}
template <typename T, int N>
__device__ __forceinline__ void rescale_row8(const LooseRow<T, N>& row, unsigned char* p, float mul) {
#pragma unroll
  for (int i = 0; i < N; ++i) rescale_bytes<1>(p + row.channel(i), mul);
}

// Where the tokens tok0 .. of a CTA lie: sequence's first row and the row behind its last, position (-1: of no sequence), cache row of head 0 (-1: none).
struct StorePlaces {
  long long cache_row[kStoreReach];
  int pos[kStoreReach], turn_pos[kStoreReach], row0[kStoreReach], row_end[kStoreReach];
};
__device__ __forceinline__ void find_places(StorePlaces& at, const PagedBatch& pb, const PagedLayout& pl, const int* positions, int tok0, int nt, int tid) {
  constexpr int kWarps = kStoreThreads / 32, kEach = kStoreReach / kWarps;
  const int lane = tid & 31, warp = tid >> 5;
  if (warp >= nt) return;                                  // a warp's tokens: warp, warp + 8, ...
  const int who = paged_owner<kEach>(pb, tok0 + warp, kWarps, lane), t = warp + lane * kWarps, tok = tok0 + t;
  if (lane < kEach && t < nt) {
    PagedSeq s{0, 0, 0, false};
    if (who >= 0) s = paged_seq(pb, pl.status, who);
    const bool there = s.n > 0 && tok >= s.row0 && tok < s.row0 + s.n;
    int pos = -1;
    long long r = -1;
    if (there) {
      pos = s.L - s.n + (tok - s.row0);
      r = paged_row(pb, pl, who, 0, pos >> pl.log_p);
      if (r >= 0) r += pos & (pl.P - 1);
    }
    at.pos[t] = pos;
    at.turn_pos[t] = positions && there ? __ldg(positions + tok) : pos;
    at.row0[t] = s.row0;
    at.row_end[t] = s.row0 + s.n;
    at.cache_row[t] = r;
  }
}

// T: new tokens and queries; E8: 8-bit pages (otherwise T); S: rows that a warp holds side by side.
template <typename T, class ROW, bool E8, int D>
__global__ void __launch_bounds__(kStoreThreads, 2) store_kernel(const __grid_constant__ StoreLaunch r, const __grid_constant__ RopeTable rt) {
  constexpr int CH = ROW::CH, WORDS = ROW::WORDS, W = D / CH, S = 32 / W, PASSES = kStoreTokens / S;
  constexpr bool loose = W == 32 && WORDS == CH;
  __shared__ __align__(16) float2 table[(kStoreReach - 1) * (D / 2)];
  __shared__ __align__(16) float w_s[2][D];
  __shared__ float rows_s[loose ? kStoreThreads / 32 : 1][loose ? D : 1];
  __shared__ StorePlaces at;
  __shared__ int run_at[kStoreTokens], run_len[kStoreTokens], n_runs_s;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, slot = lane / W;
  const int tok0 = blockIdx.x * r.tb, n_own = min(r.tb, r.pb.total_new - tok0), nt = min(n_own + kStoreTokens - 1, r.pb.total_new - tok0);
  const ROW row(rt, lane % W);
  float* own_row = rows_s[loose ? warp : 0];
  if (blockIdx.x == 0 && blockIdx.y == 0)                  // every sequence's numbers are looked at once, those without tokens too
    for (int b = tid; b < r.pb.batch; b += kStoreThreads) paged_seq(r.pb, r.pl.status, b);
  find_places(at, r.pb, r.pl, r.positions, tok0, nt, tid);
  for (int x = tid; x < 2 * D; x += kStoreThreads) {
    const float* w = x < D ? r.q_weight : r.k_weight;
    if (w) w_s[x / D][x % D] = __ldg(w + x % D);
  }
  __syncthreads();
  if (warp == 0) {
    const int t = lane;
    bool starts = false;
    int len = 0;
    if (t < n_own && at.pos[t] >= 0) {
      starts = at.pos[t] % kStoreTokens == 0 || tok0 + t == at.row0[t];
      len = min(kStoreTokens - at.pos[t] % kStoreTokens, at.row_end[t] - (tok0 + t));
    }
    const unsigned all = __ballot_sync(0xffffffffu, starts);
    if (starts) {
      const int i = __popc(all & ((1u << lane) - 1));
      run_at[i] = t;
      run_len[i] = len;
    }
    if (lane == 0) n_runs_s = __popc(all);
  }
  if (r.turn) fill_turns<ROW>(rt, table, nt, tid, kStoreThreads, false, [&](int t) { return at.turn_pos[t]; });
  __syncthreads();
  const int n_runs = n_runs_s, pairs = rt.rot / 2, h_first = blockIdx.y * r.heads_per_y, h_end = min(h_first + r.heads_per_y, r.n_q + 2 * r.n_kv);
  // heads of the queries, the keys, the values that are this block's
  int h0[3], hn[3];
#pragma unroll
  for (int g = 0; g < 3; ++g) {
    const int before = g == 0 ? 0 : g == 1 ? r.n_q : r.n_q + r.n_kv, n = g == 0 ? r.n_q : r.n_kv;
    h0[g] = min(max(h_first - before, 0), n);
    hn[g] = min(max(h_end - before, 0), n) - h0[g];
  }
  int before = 0;                                          // pieces of work of the runs before, modulo the warps
  for (int run = 0; run < n_runs; ++run) {
    const int t0 = run_at[run], len = run_len[run], many = len == 1 ? S : 1;
    const int off = at.pos[t0] % kStoreTokens, first = many > 1 ? 0 : slot;          // the lane's first token; the next is S further
    const long long cache_row0 = at.cache_row[t0];         // (a run lies in one page)
    // one head of the run (`many` heads of its one token) of the queries (GI 0), the keys (1) or the values (2); N rows a lane, at most
    auto piece = [&](auto group_c, auto norm_c, auto rows_c, int h) {
      constexpr int GI = decltype(group_c)::value, N = decltype(rows_c)::value;
      constexpr bool NORM = decltype(norm_c)::value;
      h += many > 1 ? slot : 0;
      const bool head = h < h0[GI] + hn[GI];
      const long long stride = GI == 0 ? r.q_stride : GI == 1 ? r.k_stride : r.v_stride;
      const T* in = reinterpret_cast<const T*>(GI == 0 ? r.q : GI == 1 ? r.k : r.v) + (long long)h * D + (tok0 + t0 + first) * stride;
      const int mine = head ? many > 1 ? 1 : (len - first + S - 1) / S : 0;   // rows of the lane
      uint32_t raw[N][WORDS];
#pragma unroll
      for (int p = 0; p < N; ++p)
        if (p < mine) {
          row.load(in, raw[p]);
          in += S * stride;
        } else {
#pragma unroll
          for (int i = 0; i < WORDS; ++i) raw[p][i] = 0u;
        }
      unsigned char* scale_at = nullptr;
      int e_old = kExpMin;
      const long long crow = GI == 0 || cache_row0 < 0 ? -1 : cache_row0 + (long long)h * r.pl.head_stride;
      if constexpr (E8 && GI > 0) {
        if (head && crow >= 0) {
          scale_at = (GI == 1 ? r.k_scales : r.v_scales) + (crow >> 4);
          if (off > 0) e_old = held_exponent(scale_at);
        }
        __syncwarp();                                      // (all lanes have read the byte before one writes it)
      }
      const float2* tab = table + (t0 + first) * pairs;
      T* out = GI == 0 ? reinterpret_cast<T*>(r.q_out) + (tok0 + t0 + first) * r.q_out_stride + (long long)h * D
                       : E8 ? nullptr : reinterpret_cast<T*>(GI == 1 ? r.k_pages : r.v_pages) + (crow + first) * D;
      const long long out_stride = GI == 0 ? S * r.q_out_stride : S * D;
      auto finished = [&](float (&x)[CH], int p) {         // (whole warps)
        row.values(raw[p], x);
        if constexpr (NORM) {
          const float rms = row_rms(x, W, 1.f / D, r.eps);
          float w[CH];
          row.weights(w_s[GI], w);
          row_scale(x, rms, w);
        }
        if (GI < 2 && r.turn) row.turn(x, tab + (p < mine ? S * p * pairs : 0), own_row);
      };
      if constexpr (GI == 0 || !E8) {
#pragma unroll
        for (int p = 0; p < N; ++p) {
          float x[CH];
          finished(x, p);
          if (p < mine && (GI == 0 || crow >= 0)) row.store(out, x);
          out += out_stride;
        }
      } else {
        float x[N][CH], top = 0.f;
#pragma unroll
        for (int p = 0; p < N; ++p) {
          finished(x[p], p);
#pragma unroll
          for (int i = 0; i < CH; i += 2) top = fmaxf(top, fmaxf(fabsf(x[p][i]), fabsf(x[p][i + 1])));   // (NaN takes no part)
        }
        // the lanes of a row, and where the rows are one head's tokens, all of them
        auto over_rows = [&](float v) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const float other = __shfl_xor_sync(0xffffffffu, v, o);
            if (o < W || many == 1) v = fmaxf(v, other);
          }
          return v;
        };
        top = over_rows(top);
        if (__any_sync(0xffffffffu, top == INFINITY)) {    // infinities take no part in the scale either, and have no place in the format: NaN
          float fine = 0.f;
#pragma unroll
          for (int p = 0; p < N; ++p)
#pragma unroll
            for (int i = 0; i < CH; ++i) {
              if (fabsf(x[p][i]) == INFINITY) x[p][i] = __int_as_float(0x7fffffff);
              fine = fmaxf(fine, fabsf(x[p][i]));
            }
          top = over_rows(fine);
        }
        if (scale_at) {
          unsigned char* page = reinterpret_cast<unsigned char*>(GI == 1 ? r.k_pages : r.v_pages) + crow * D;
          const int e = max(scale_exponent(top), e_old);
          if (off > 0 && e > e_old) {                      // the tokens before: rounded again, each row by the lanes that hold one
            const float less = power_of_two(e_old - e);
#pragma unroll 1
            for (int t = first; t < off; t += many > 1 ? 1 : S) rescale_row8(row, page + (t - off) * D, less);
          }
          const float mul = power_of_two(-e);
#pragma unroll
          for (int p = 0; p < N; ++p)
            if (p < mine) store_row8(row, page + (first + S * p) * D, x[p], mul);
          if ((many > 1 ? lane % W : lane) == 0) *scale_at = (unsigned char)(e + 127);
        }
      }
    };
    auto heads = [&](auto rows_c) {
      constexpr std::integral_constant<int, 0> queries{};
      constexpr std::integral_constant<int, 1> keys{};
      constexpr std::integral_constant<int, 2> vals{};
      constexpr std::true_type normed{};
      constexpr std::false_type plain{};
      const int n0 = (hn[0] + many - 1) / many, n1 = n0 + (hn[1] + many - 1) / many, n2 = n1 + (hn[2] + many - 1) / many;
      for (int u = (warp - before) & 7; u < n2; u += kStoreThreads / 32) {
        if (u < n0) {
          if (r.q_weight) piece(queries, normed, rows_c, h0[0] + u * many); else piece(queries, plain, rows_c, h0[0] + u * many);
        } else if (u < n1) {
          if (r.k_weight) piece(keys, normed, rows_c, h0[1] + (u - n0) * many); else piece(keys, plain, rows_c, h0[1] + (u - n0) * many);
        } else {
          piece(vals, plain, rows_c, h0[2] + (u - n1) * many);
        }
      }
      before += n2;
    };
    if (len <= S) heads(std::integral_constant<int, 1>{}); else heads(std::integral_constant<int, PASSES>{});
  }
}

// Cached tokens as rows: TC (bf16, fp32 or an e4m3 byte) -> TO.  A thread takes 16 channels of one head of one token.
template <typename TC, typename TO, int D>
__global__ void __launch_bounds__(kStoreThreads) read_kernel(const __grid_constant__ PagedBatch pb, const __grid_constant__ PagedLayout pl, const TC* k_pages,
                                                             const TC* v_pages, const unsigned char* k_scales, const unsigned char* v_scales, TO* k_out,
                                                             TO* v_out, int tb, int heads_per_y) {
  __shared__ StorePlaces at;
  constexpr int PIECES = D / 16;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, tok0 = blockIdx.x * tb, nt = min(tb, pb.total_new - tok0);
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = tid; b < pb.batch; b += kStoreThreads) paged_seq(pb, pl.status, b);
  find_places(at, pb, pl, nullptr, tok0, nt, tid);
  __syncthreads();
  const int h0 = blockIdx.y * heads_per_y, heads = min(heads_per_y, 2 * pl.Hkv - h0), each = heads * PIECES;
#pragma unroll 4
  for (int x = tid; x < nt * each; x += kStoreThreads) {
    const int t = x / each, y = x - t * each, hh = h0 + y / PIECES, c = y % PIECES * 16, is_v = hh >= pl.Hkv, h = is_v ? hh - pl.Hkv : hh;
    if (at.pos[t] < 0) continue;                           // (a row of no sequence)
    const long long row = at.cache_row[t] < 0 ? -1 : at.cache_row[t] + h * pl.head_stride;
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
    if (row >= 0) {
      const TC* from = (is_v ? v_pages : k_pages) + row * D + c;
      if constexpr (sizeof(TC) == 1) {
        const uint4 w = *reinterpret_cast<const uint4*>(from);
        const float mul = paged_scale(is_v ? v_scales : k_scales, row);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = unpack_e4m3(ws[i] & 0xffffu), b = unpack_e4m3(ws[i] >> 16);
          v[4 * i] = a.x * mul; v[4 * i + 1] = a.y * mul; v[4 * i + 2] = b.x * mul; v[4 * i + 3] = b.y * mul;
        }
      } else {
        constexpr int VEC = 16 / (int)sizeof(TC);
#pragma unroll
        for (int i = 0; i < 16; i += VEC) {
          uint32_t w[4];
          load_raw(from + i, w);
          unpack<TC, VEC>(w, *reinterpret_cast<float(*)[VEC]>(v + i));
        }
      }
    }
    TO* out = (is_v ? v_out : k_out) + ((long long)(tok0 + t) * pl.Hkv + h) * D + c;
    constexpr int VO = 16 / (int)sizeof(TO);
#pragma unroll
    for (int i = 0; i < 16; i += VO) store_piece<VO>(out + i, *reinterpret_cast<const float(*)[VO]>(v + i));
  }
}

template <typename T, class ROW, bool E8, int D>
cudaError_t store_launch(StoreLaunch r, const RopeTable& rt, cudaStream_t s) {
  const int heads = r.n_q + 2 * r.n_kv, sm = device_sm_count();
  // rows of a CTA: 16, fewer where SMs would idle; then, up to two rounds of CTAs, the heads are shared out to four (turns of 50 to 700 x 16 74 -> 61 us; from more
  // rounds on the sines of a token, which every CTA forms again, cost more than they bring: 16384 tokens in fp32 43 -> 49)
  int tb = kStoreTokens;
  while (tb > 1 && (r.pb.total_new + tb - 1) / tb < 2 * sm) tb /= 2;
  const int blocks = (r.pb.total_new + tb - 1) / tb;
  int ys = 1;
  if (blocks < 4 * sm) {
    ys = (8 * sm + blocks - 1) / blocks;
    const int most = (heads + 7) / 8;                      // a head for every warp
    if (ys > most) ys = most;
  }
  r.tb = tb;
  r.heads_per_y = (heads + ys - 1) / ys;
  return launch_ex(store_kernel<T, ROW, E8, D>, dim3(blocks, (heads + r.heads_per_y - 1) / r.heads_per_y), dim3(kStoreThreads), 0, s, 0, true, r, rt);
}
template <typename T, bool E8, int D>
cudaError_t store_rows(const StoreLaunch& r, const RopeTable& rt, bool wide, cudaStream_t s) {
  return wide ? store_launch<T, WideRow<T, 16 / (int)sizeof(T)>, E8, D>(r, rt, s) : store_launch<T, LooseRow<T, D / 32>, E8, D>(r, rt, s);
}
template <typename T>
cudaError_t store_type(const StoreLaunch& r, const RopeTable& rt, bool e8, bool wide, cudaStream_t s) {
  if (r.pl.d == 128) return e8 ? store_rows<T, true, 128>(r, rt, wide, s) : store_rows<T, false, 128>(r, rt, wide, s);
  return e8 ? store_rows<T, true, 64>(r, rt, wide, s) : store_rows<T, false, 64>(r, rt, wide, s);
}
template <typename TC, typename TO>
cudaError_t read_launch(const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, void* k_out, void* v_out, cudaStream_t s) {
  const int sm = device_sm_count(), heads = 2 * pl.Hkv;
  int tb = kStoreReach;
  while (tb > 1 && (pb.total_new + tb - 1) / tb < 4 * sm) tb /= 2;
  const int blocks = (pb.total_new + tb - 1) / tb, items = tb * heads * (pl.d / 16);
  int ys = 1;
  if (blocks < 4 * sm) {
    ys = (items + kStoreThreads - 1) / kStoreThreads;
    if (ys > heads) ys = heads;
  }
  const int per_y = (heads + ys - 1) / ys;
  auto kern = pl.d == 128 ? read_kernel<TC, TO, 128> : read_kernel<TC, TO, 64>;
  return launch_ex(kern, dim3(blocks, (heads + per_y - 1) / per_y), dim3(kStoreThreads), 0, s, 0, true, pb, pl, (const TC*)pages.k, (const TC*)pages.v,
                   (const unsigned char*)pages.k_scales, (const unsigned char*)pages.v_scales, (TO*)k_out, (TO*)v_out, tb, per_y);
}

}  // namespace

cudaError_t launch_store(const RopeTable* rope, const StoreGroups& g, const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, cudaStream_t s) {
  RopeTable none = {};
  none.dim = pl.d;
  const RopeTable& rt = rope ? *rope : none;
  StoreLaunch r = {};
  r.q = g.q; r.k = g.k; r.v = g.v; r.q_out = g.q_out;
  r.q_stride = g.q_stride; r.k_stride = g.k_stride; r.v_stride = g.v_stride; r.q_out_stride = g.q_out_stride;
  r.q_weight = g.q_weight; r.k_weight = g.k_weight;
  r.eps = g.eps;
  r.positions = g.positions;
  r.pb = pb;
  r.pl = pl;
  r.k_pages = pages.k; r.v_pages = pages.v;
  r.k_scales = pages.k_scales; r.v_scales = pages.v_scales;
  r.turn = rope != nullptr;
  const bool e8 = pages.type == kPagesE4m3;
  // one launch per element type (queries may have another than a cache of 16 or 32 bits)
  cudaError_t e = cudaSuccess;
  for (int f32 = 0; f32 < 2 && e == cudaSuccess; ++f32) {
    const int size = f32 ? 4 : 2;
    r.n_q = g.q && g.q_f32 == f32 ? pl.Hq : 0;
    r.n_kv = g.kv_f32 == f32 ? pl.Hkv : 0;
    if (r.n_q + r.n_kv == 0) continue;
    bool wide = wide_rotation(rt, size);
    if (r.n_q) wide = wide && wide_strides(r.q, size, r.q_stride, 0, 0) && wide_strides(r.q_out, size, r.q_out_stride, 0, 0);
    if (r.n_kv) wide = wide && wide_strides(r.k, size, r.k_stride, 0, 0) && wide_strides(r.v, size, r.v_stride, 0, 0);
    e = f32 ? store_type<float>(r, rt, e8, wide, s) : store_type<__nv_bfloat16>(r, rt, e8, wide, s);
  }
  return e;
}

cudaError_t launch_read(const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, void* k_out, void* v_out, int out_f32, cudaStream_t s) {
  if (pages.type == kPagesE4m3)
    return out_f32 ? read_launch<unsigned char, float>(pb, pl, pages, k_out, v_out, s) : read_launch<unsigned char, __nv_bfloat16>(pb, pl, pages, k_out, v_out, s);
  if (pages.type == kPagesF32)
    return out_f32 ? read_launch<float, float>(pb, pl, pages, k_out, v_out, s) : read_launch<float, __nv_bfloat16>(pb, pl, pages, k_out, v_out, s);
  return out_f32 ? read_launch<__nv_bfloat16, float>(pb, pl, pages, k_out, v_out, s) : read_launch<__nv_bfloat16, __nv_bfloat16>(pb, pl, pages, k_out, v_out, s);
}

}  // namespace spla
