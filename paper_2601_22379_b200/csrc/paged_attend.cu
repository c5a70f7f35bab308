// Attention of new tokens over a paged cache, in fp32 arithmetic for every type (fp32 caches or queries, addresses that TMA does not
// take), and the kernel that joins the partial results of units cut between CTAs, whichever kernel made them.
//
//   s_ij = scale q_i.k_j;  s <- cap tanh(s / cap);  s <- s - slope |p_i - j|;  o_i = sum_j softmax(s)_ij v_j;  lse_i = ln sum_j exp(s_ij)
//
// One pass over the keys with the running maximum and sum of the softmax in base 2.  A CTA walks tiles of TK keys for R query
// rows: scores from row pieces in shared memory (four rows x KT keys per thread, packed FMAs over two channels), then the
// product with V (four rows x CW channels per thread, the tile's tokens shared by TS threads).  K of the next tile is on its way from
// when the scores are done, V from when the product is done (asynchronous copies where the cache is fp32), the page table one tile ahead of that.
// R = 4, 16 and 64 by the rows that a unit has at most; a row tile's products cost the same however few of its rows are real.
// 4 rows are bound by reading K and V (8 sequences of 32000, 8 heads of 128: 2.1 GB in 493 us, 4.3 TB/s; bf16 caches, which are not copied
// asynchronously, 1.05 GB in 1.20 ms), 16 by shared memory's reads for the scores (G = 8, the same cache: 523 us), 64 by the FMA pipe, in use half
// of the time: the phases of a tile alternate with barriers (300 tokens on 3000 x 4, 32 heads of 128: 1.54 ms, 36 TFLOP/s; tiles of 32
// keys with P beside K are 9 % slower, row tiles of 128 in one CTA of 512 threads, or with eight rows per thread, within 7 %).
#include "paged.h"

namespace spla {

namespace {

template <int R, int D>
struct PgShape {
  static constexpr int THREADS = 256;
  static constexpr int TK = 64;
  static constexpr bool OVER = R == 64;                            // P takes the place of K (two CTAs per SM; the copies of K and V start together then)
  static constexpr int KT = R == 64 ? 4 : 1;       // keys per thread
  static constexpr int RG = R / 4;                                 // groups of four rows
  static constexpr int CS = THREADS / (RG * (TK / KT));            // threads that share the channels of a score
  static constexpr int CW = R == 64 ? D / 16 : 4;                  // channels per thread in the product with V
  static constexpr int TS = THREADS / (RG * (D / CW));             // threads that share a tile's tokens there
  static constexpr int LD = D + 4, LP = TK + 4;
  static constexpr int kQ = 0, kK = kQ + R * LD * 4, kV = kK + TK * LD * 4, kP = OVER ? kK : kV + TK * D * 4, kFac = kV + TK * D * 4 + (OVER ? 0 : R * LP * 4), kLo = kFac + R * 4,
                       kHi = kLo + R * 4, kSum = kHi + R * 4, kMax = kSum + R * 4, kTop = kMax + R * 4, kRows = (kTop + R * 8 * 4 + 15) / 16 * 16,
                       kSeqs = kRows + 2 * (TK / 16) * 8, kBytes = kSeqs + (int)sizeof(PagedSeqs);
  static_assert(CS >= 1 && TS >= 1 && D % (4 * CS) == 0, "shape");
  static_assert(!OVER || LP <= LD, "P in the place of K");
  static_assert((TS - 1) * R * D * 4 <= TK * (LD + D) * 4, "the partial products of a unit fit the K and V tiles");
  static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs per SM (with one, 300 tokens on 3000 x 4 take 1.93 ms in place of 1.54)");
};

__device__ __forceinline__ void copy16(void* dst, const void* src, bool there) {   // asynchronous; zeros where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T>
__device__ __forceinline__ float4 load4(const T* p) {
  float v[4];
  load_vec<4>(p, v);
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)); }

template <typename TQ, typename TKV, int R, int D>
__global__ void __launch_bounds__((PgShape<R, D>::THREADS), 2)
    paged_general_kernel(const PagedAttend a, const TKV* __restrict__ k_pages, const TKV* __restrict__ v_pages) {
  using S = PgShape<R, D>;
  constexpr int THREADS = S::THREADS, TK = S::TK, KT = S::KT, CS = S::CS, CW = S::CW, TS = S::TS, LD = S::LD, LP = S::LP, D4 = D / 4;
  extern __shared__ __align__(16) unsigned char smem[];
  float* qs = reinterpret_cast<float*>(smem + S::kQ);
  float* ks = reinterpret_cast<float*>(smem + S::kK);
  float* vs = reinterpret_cast<float*>(smem + S::kV);
  float* ps = reinterpret_cast<float*>(smem + S::kP);
  float* fac = reinterpret_cast<float*>(smem + S::kFac);
  int* lo_s = reinterpret_cast<int*>(smem + S::kLo);
  int* hi_s = reinterpret_cast<int*>(smem + S::kHi);
  float* sum_s = reinterpret_cast<float*>(smem + S::kSum);
  float* max_s = reinterpret_cast<float*>(smem + S::kMax);
  float* top_s = reinterpret_cast<float*>(smem + S::kTop);        // [R][warps of a row group]
  long long* rows_s = reinterpret_cast<long long*>(smem + S::kRows);   // [2][TK / 16]: first row of every 16 tokens of a tile, -1: none
  PagedSeqs& seqs = *reinterpret_cast<PagedSeqs*>(smem + S::kSeqs);
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, G = a.pl.G;
  const long long share = paged_share(a.w, paged_fill_seqs(a, seqs, tid, THREADS));
  PagedWalk wk;
  const bool any = wk.seek(a, seqs, blockIdx.x * share, share);
  if (a.w.cuts && tid < 32) {
    const int4 cut = wk.cut_here(a, any, share);
    if (tid == 0) a.w.cuts[blockIdx.x] = cut;
  }
  if (!any) return;
  // scores: thread = (channel share, key, row group); product: (channel group, token share, row group)
  const int cs = tid % CS, kg = tid / CS % (TK / KT), rg = tid / (CS * (TK / KT));
  const int cg = tid % (D / CW), ts = tid / (D / CW) % TS, rp = tid / (D / CW * TS);
  const float sc = a.sm_scale, inv_cap = a.softcap > 0.f ? 1.f / a.softcap : 0.f;
  while (wk.next(a, seqs)) {
    const int i0 = wk.first_pos(a.w), rows = min(wk.n - i0, wk.n_pos(a.w)) * G;
    const int pos0 = wk.L - wk.n + i0;
    auto find_rows = [&](int t) {                                  // a few threads: where tile t lies
      if (tid < TK / 16 && t < wk.t1) {
        const int tok = t * TK + tid * 16;
        long long row = -1;
        if (tok < wk.L) {
          row = paged_row(a.pb, a.pl, wk.b, wk.h, tok >> a.pl.log_p);
          if (row >= 0) row += tok & (a.pl.P - 1);
        }
        rows_s[(t & 1) * (TK / 16) + tid] = row;
      }
    };
    auto fetch = [&](const TKV* pages, float* to, int ld, int t) { // one tile of K or V
#pragma unroll
      for (int x0 = 0; x0 < TK * D4; x0 += THREADS) {
        const int x = x0 + tid, j = x / D4, c = x % D4;
        const long long row = rows_s[(t & 1) * (TK / 16) + j / 16];
        const bool there = row >= 0 && t * TK + j < wk.L;
        const TKV* from = pages + (there ? (row + j % 16) * D + c * 4 : 0);
        if constexpr (sizeof(TKV) == 4) copy16(to + j * ld + c * 4, from, there);
        else *reinterpret_cast<float4*>(to + j * ld + c * 4) = there ? load4(from) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      copies_close();
    };
    __syncthreads();                                               // the segment before is done with shared memory
    find_rows(wk.t0);
    for (int x = tid; x < R * D4; x += THREADS) {
      const int r = x / D4, c = x % D4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) {
        const TQ* q = reinterpret_cast<const TQ*>(a.q) + (wk.row0 + i0 + r / G) * a.q_stride + (long long)(wk.h * G + r % G) * D + c * 4;
        if (((uintptr_t)a.q | (uintptr_t)(a.q_stride * sizeof(TQ))) % (4 * sizeof(TQ)) == 0) v = load4(q);
        else v = make_float4(to_float(q[0]), to_float(q[1]), to_float(q[2]), to_float(q[3]));
      }
      *reinterpret_cast<float4*>(qs + r * LD + c * 4) = v;
    }
    bool sees_any = false;
    if (tid < R) {
      PagedSees s{0, 0};
      if (tid < rows) s = paged_sees(a, wk.row0, wk.n, wk.L, wk.prefix, i0 + tid / G);
      lo_s[tid] = s.lo;
      hi_s[tid] = s.hi;
      sees_any = s.lo < s.hi;
    }
    // a warp whose rows are all behind the unit's last has nothing to compute (its rows of scores and of the product are the same)
    const bool idle = tid / 32 * 32 / (CS * (TK / KT)) * 4 >= rows;
    float slope[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) slope[i] = a.slopes && rg * 4 + i < rows ? __ldg(a.slopes + wk.h * G + (rg * 4 + i) % G) : 0.f;
    float m[4], l[4], o[4][CW];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int x = 0; x < CW; ++x) o[i][x] = 0.f;
    }
    sees_any = __syncthreads_or(sees_any);                         // (rows' bounds; where the first tile lies)
    // the tiles that some row sees (of a segment's, those before all documents' starts and behind all rows' ends are passed over), and
    // the keys that all rows see
    int t_from = wk.t0, t_to = sees_any ? wk.t1 : wk.t0, all_lo, all_hi;
    {
      int lo = lo_s[0], hi = hi_s[rows - 1];                       // (both grow with the position, but for documents)
      all_lo = lo_s[rows - 1];
      all_hi = hi_s[0];
      if (a.first_key) {
        lo = 0x7fffffff;
        for (int r = 0; r < rows; r += G) {
          if (lo_s[r] < hi_s[r]) lo = min(lo, lo_s[r]);
          all_lo = max(all_lo, lo_s[r]);
        }
      }
      if (sees_any) {
        t_from = max(t_from, lo / TK);
        t_to = min(t_to, (hi + TK - 1) / TK);
      }
    }
    if (t_from < t_to) {
      if (t_from != wk.t0) {
        find_rows(t_from);
        __syncthreads();
      }
      fetch(k_pages, ks, LD, t_from);
      fetch(v_pages, vs, D, t_from);
    }
#pragma unroll 1
    for (int t = t_from; t < t_to; ++t) {
      const int tok0 = t * TK;
      const bool part = tok0 < all_lo || tok0 + TK > all_hi;       // some row does not see all of it
      find_rows(t + 1);
      copies_wait<1>();                                            // K is here
      __syncthreads();
      float s[4][KT], mt[4];
      constexpr int kRowThreads = CS * (TK / KT);                  // 16 (R = 64: half a warp), 64 (two warps) or 256
      constexpr int W = kRowThreads > 32 ? kRowThreads / 32 : 1;   // warps of a row group: their maxima meet in shared memory
      if (!idle) {
        // ---- scores of four rows x KT keys, this thread's share of the channels
        float2 acc[4][KT];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int y = 0; y < KT; ++y) acc[i][y] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = cs * 4; c < D; c += 4 * CS) {
          float4 kx[KT];
#pragma unroll
          for (int y = 0; y < KT; ++y) kx[y] = *reinterpret_cast<const float4*>(ks + (kg + y * (TK / KT)) * LD + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 qx = *reinterpret_cast<const float4*>(qs + (rg * 4 + i) * LD + c);
#pragma unroll
            for (int y = 0; y < KT; ++y) {
              acc[i][y] = __ffma2_rn(make_float2(qx.x, qx.y), make_float2(kx[y].x, kx[y].y), acc[i][y]);
              acc[i][y] = __ffma2_rn(make_float2(qx.z, qx.w), make_float2(kx[y].z, kx[y].w), acc[i][y]);
            }
          }
        }
        // ---- running maximum and sum; every row belongs to CS x TK / KT neighbouring threads
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = rg * 4 + i, pos = pos0 + r / G;
          mt[i] = -INFINITY;
#pragma unroll
          for (int y = 0; y < KT; ++y) {
            float v = acc[i][y].x + acc[i][y].y;
#pragma unroll
            for (int w = 1; w < CS; w <<= 1) v += __shfl_xor_sync(0xffffffffu, v, w);
            v *= sc;
            if (a.softcap > 0.f) v = a.softcap * tanhf(v * inv_cap);
            const int j = tok0 + kg + y * (TK / KT);
            if (slope[i] != 0.f) v -= slope[i] * (float)abs(pos - j);
            s[i][y] = !part || (j >= lo_s[r] && j < hi_s[r]) ? v * kLog2e : -INFINITY;
            mt[i] = fmaxf(mt[i], s[i][y]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int w = kRowThreads < 32 ? kRowThreads / 2 : 16; w >= CS; w >>= 1) mt[i] = fmaxf(mt[i], __shfl_xor_sync(0xffffffffu, mt[i], w));
        if constexpr (W > 1) {
          if (tid % 32 == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) top_s[(rg * 4 + i) * 8 + tid / 32 % W] = mt[i];
        }
      }
      __syncthreads();                                             // (K is used up; the maxima; where the next tile lies)
      if constexpr (!S::OVER) {
        if (t + 1 < t_to) fetch(k_pages, ks, LD, t + 1); else copies_close();
      }
      if (!idle) {
        if constexpr (W > 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < W; ++x) mt[i] = fmaxf(mt[i], top_s[(rg * 4 + i) * 8 + x]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float mn = fmaxf(m[i], mt[i]), f = m[i] == mn ? 1.f : ex2(m[i] - mn), nm = mn == -INFINITY ? 0.f : -mn;
          m[i] = mn;
          l[i] *= f;
          if (tid % kRowThreads == 0) fac[rg * 4 + i] = f;
#pragma unroll
          for (int y = 0; y < KT; ++y) {
            const float p = ex2(s[i][y] + nm);
            l[i] += p;                                               // (this thread's keys only, until the segment's end)
            if (cs == 0) ps[(rg * 4 + i) * LP + kg + y * (TK / KT)] = p;
          }
        }
      }
      copies_wait<S::OVER ? 0 : 1>();                              // V is here
      bool bad = false;                                            // a value that is not finite, in a tile that some row does not see all of
      if (part) {
#pragma unroll
        for (int x0 = 0; x0 < TK * D4; x0 += THREADS) {            // (what this thread has brought)
          const float4 v = *reinterpret_cast<const float4*>(vs + (x0 + tid) * 4);
          bad |= !(fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY && fabsf(v.z) < INFINITY && fabsf(v.w) < INFINITY);
        }
      }
      bad = __syncthreads_or(bad);
      // ---- product with V: four rows x CW channels, every TS-th group of four tokens
      if (!idle) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = fac[rp * 4 + i];
#pragma unroll
          for (int x = 0; x < CW; ++x) o[i][x] *= f;
        }
        if (!bad) {
#pragma unroll 2
          for (int j = ts * 4; j < TK; j += 4 * TS) {
            float4 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(ps + (rp * 4 + i) * LP + j);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              float4 v[CW / 4];
#pragma unroll
              for (int x = 0; x < CW / 4; ++x) v[x] = *reinterpret_cast<const float4*>(vs + (j + y) * D + x * (D * 4 / CW) + cg * 4);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float w = y == 0 ? p[i].x : y == 1 ? p[i].y : y == 2 ? p[i].z : p[i].w;
#pragma unroll
                for (int x = 0; x < CW / 4; ++x) {
                  float2* d = reinterpret_cast<float2*>(&o[i][x * 4]);
                  d[0] = __ffma2_rn(make_float2(w, w), make_float2(v[x].x, v[x].y), d[0]);
                  d[1] = __ffma2_rn(make_float2(w, w), make_float2(v[x].z, v[x].w), d[1]);
                }
              }
            }
          }
        } else {                                                     // 0 x infinity is no 0: hidden keys stay out
#pragma unroll 1
          for (int j = ts; j < TK; j += TS)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = rp * 4 + i;
              if (tok0 + j < lo_s[r] || tok0 + j >= hi_s[r]) continue;
#pragma unroll
              for (int x = 0; x < CW; ++x) o[i][x] = fmaf(ps[r * LP + j], vs[j * D + x / 4 * (D * 4 / CW) + cg * 4 + x % 4], o[i][x]);
            }
        }
      }
      __syncthreads();                                             // (V and P are used up)
      if (t + 1 < t_to) {
        if constexpr (S::OVER) fetch(k_pages, ks, LD, t + 1);
        fetch(v_pages, vs, D, t + 1);
      } else {
        copies_close();
      }
    }
    copies_wait<0>();
    // ---- end of the segment: sums over the threads of a row, then over the token shares
    constexpr int kRowThreads = CS * (TK / KT);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int w = kRowThreads < 32 ? kRowThreads / 2 : 16; w >= CS; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    __syncthreads();
    if constexpr (kRowThreads > 32) {
      constexpr int W = kRowThreads / 32;
      if (tid % 32 == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) ps[(rg * 4 + i) * LP + tid / 32 % W] = l[i];
      __syncthreads();
      if (tid < R) {
        float sum = 0.f;
        for (int x = 0; x < W; ++x) sum += ps[tid * LP + x];
        sum_s[tid] = sum;
      }
    } else if (tid % kRowThreads == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sum_s[rg * 4 + i] = l[i];
    }
    if (tid % kRowThreads == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) max_s[rg * 4 + i] = m[i];
    if constexpr (TS > 1) {
      float* part = ks;                                            // (K and V are used up)
      if (ts > 0)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < CW; x += 4)
            *reinterpret_cast<float4*>(part + ((ts - 1) * R + rp * 4 + i) * D + x / 4 * (D * 4 / CW) + cg * 4) =
                make_float4(o[i][x], o[i][x + 1], o[i][x + 2], o[i][x + 3]);
      __syncthreads();
      if (ts == 0)
        for (int y = 0; y < TS - 1; ++y)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < CW; ++x) o[i][x] += part[(y * R + rp * 4 + i) * D + x / 4 * (D * 4 / CW) + cg * 4 + x % 4];
    } else {
      __syncthreads();
    }
    const bool whole = wk.head && wk.tail;
    const long long slot = 2LL * blockIdx.x + (wk.head ? 1 : 0);
    if (ts == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = rp * 4 + i;
        if (r >= rows) continue;
        const float sum = sum_s[r], mul = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
        const long long row = (long long)(wk.row0 + i0 + r / G) * a.pl.Hq + wk.h * G + r % G;
#pragma unroll
        for (int x = 0; x < CW; x += 4) {
          const int c = x / 4 * (D * 4 / CW) + cg * 4;
          float4 v = make_float4(o[i][x] * mul, o[i][x + 1] * mul, o[i][x + 2] * mul, o[i][x + 3] * mul);
          if (whole) {
            if (sum == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
            store4(reinterpret_cast<TQ*>(a.out) + row * D + c, v);
          } else {
            *reinterpret_cast<float4*>(a.w.part_o + (slot * a.w.rows + r) * D + c) = v;
          }
        }
        if (cg == 0) {
          if (!whole) a.w.part_ml[slot * a.w.rows + r] = make_float2(max_s[r], sum);
          else if (a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (max_s[r] + log2f(sum)) * kLn2;
        }
      }
  }
}

// Joins the partial results of a cut unit: the share before its first cut holds its head, the shares after hold the rest.
// A few CTAs per cut, which find nothing to do unless it is the first of its unit.  32 rows and more (two or three parts, mostly): a thread
// takes four channels of a row.  Fewer rows (many parts): a warp or several per row, each sums a run of the parts, the runs' sums
// meet in shared memory, in order.
constexpr int kJoinThreads = 256;
template <typename TO, int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const PagedAttend a) {
  __shared__ float run_o[kJoinThreads / 32][D];
  __shared__ float run_sum[kJoinThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.pl.G;
  const int cut = blockIdx.x + 1;                                  // the border between shares cut - 1 and cut
  const int4 c = a.w.cuts[cut];
  const int rows = c.x, parts = c.y;
  if (rows == 0) return;
  auto slot_of = [&](int x) { return x == 0 ? 2LL * (cut - 1) + 1 : 2LL * (cut + x - 1); };
  auto out_row = [&](int r) { return (long long)(c.z + r / G) * a.pl.Hq + c.w * G + r % G; };
  if (rows >= 32) {
    for (int x = blockIdx.y * kJoinThreads + tid; x < rows * (D / 4); x += gridDim.y * kJoinThreads) {
      const int r = x / (D / 4), ch = x % (D / 4) * 4;
      float M = -INFINITY, sum = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int y = 0; y < parts; ++y) {                            // (the running maximum: one pass)
        const long long at = slot_of(y) * a.w.rows + r;
        const float2 ml = a.w.part_ml[at];
        const float4 v = *reinterpret_cast<const float4*>(a.w.part_o + at * D + ch);
        if (ml.y == 0.f) continue;                                 // (a part that has seen no key takes no part)
        const float top = fmaxf(M, ml.x), f = M == top ? 1.f : ex2(M - top), w = ex2(ml.x - top);
        M = top;
        sum = fmaf(ml.y, w, sum * f);
        o.x = fmaf(v.x, w, o.x * f); o.y = fmaf(v.y, w, o.y * f); o.z = fmaf(v.z, w, o.z * f); o.w = fmaf(v.w, w, o.w * f);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const long long row = out_row(r);
      store4(reinterpret_cast<TO*>(a.out) + row * D + ch, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (ch == 0 && a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
    }
    return;
  }
  constexpr int V = D / 32;
  const int per_row = rows >= 8 ? 1 : rows >= 4 ? 2 : rows >= 2 ? 4 : 8, at_once = 8 / per_row;   // warps per row, rows at a time
  const int run = warp % per_row, x0 = parts * run / per_row, x1 = parts * (run + 1) / per_row;
  for (int r0 = blockIdx.y * at_once; r0 < rows; r0 += gridDim.y * at_once) {
    const int r = r0 + warp / per_row;
    float o[V], sum = 0.f, M = -INFINITY;
#pragma unroll
    for (int x = 0; x < V; ++x) o[x] = 0.f;
    if (r < rows) {
      for (int x = lane; x < parts; x += 32) M = fmaxf(M, a.w.part_ml[slot_of(x) * a.w.rows + r].x);
      M = warp_max(M);
#pragma unroll 8
      for (int x = x0; x < x1; ++x) {
        const long long at = slot_of(x) * a.w.rows + r;
        const float2 ml = a.w.part_ml[at];
        float v[V];
        load_vec<V>(a.w.part_o + at * D + lane * V, v);
        if (ml.y != 0.f) {
          const float w = ex2(ml.x - M);
          sum = fmaf(ml.y, w, sum);
#pragma unroll
          for (int y = 0; y < V; ++y) o[y] = fmaf(v[y], w, o[y]);
        }
      }
    }
    if (per_row > 1) {
      __syncthreads();                                             // (the rows before have been read)
#pragma unroll
      for (int y = 0; y < V; ++y) run_o[warp][lane * V + y] = o[y];
      if (lane == 0) run_sum[warp] = sum;
      __syncthreads();
      if (run > 0) continue;
      for (int x = 1; x < per_row; ++x) {
        sum += run_sum[warp + x];
#pragma unroll
        for (int y = 0; y < V; ++y) o[y] += run_o[warp + x][lane * V + y];
      }
    }
    if (r >= rows) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const long long row = out_row(r);
#pragma unroll
    for (int y = 0; y < V; ++y) o[y] *= inv;
    TO* out = reinterpret_cast<TO*>(a.out) + row * D + lane * V;
    if constexpr (sizeof(TO) == 4) {
#pragma unroll
      for (int y = 0; y < V; y += 2) *reinterpret_cast<float2*>(out + y) = make_float2(o[y], o[y + 1]);
    } else {
#pragma unroll
      for (int y = 0; y < V; y += 2) *reinterpret_cast<uint32_t*>(out + y) = pack_bf16(o[y], o[y + 1]);
    }
    if (lane == 0 && a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
  }
}

template <typename TQ, typename TKV, int R, int D>
cudaError_t general_launch(const PagedAttend& a, const void* k, const void* v, cudaStream_t s) {
  auto kern = paged_general_kernel<TQ, TKV, R, D>;
  static unsigned long long allowed = 0;
  cudaError_t e = allow_smem_once(kern, PgShape<R, D>::kBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(a.w.n_cta), dim3(PgShape<R, D>::THREADS), PgShape<R, D>::kBytes, s, 0, true, a, reinterpret_cast<const TKV*>(k), reinterpret_cast<const TKV*>(v));
}
template <typename TQ, typename TKV, int D>
cudaError_t general_rows(const PagedAttend& a, const void* k, const void* v, cudaStream_t s) {
  const int r = a.w.ppos * a.pl.G;
  return r <= 4 ? general_launch<TQ, TKV, 4, D>(a, k, v, s) : r <= 16 ? general_launch<TQ, TKV, 16, D>(a, k, v, s) : general_launch<TQ, TKV, 64, D>(a, k, v, s);
}
template <typename TQ, typename TKV>
cudaError_t general_dim(const PagedAttend& a, const void* k, const void* v, cudaStream_t s) {
  return a.pl.d == 128 ? general_rows<TQ, TKV, 128>(a, k, v, s) : general_rows<TQ, TKV, 64>(a, k, v, s);
}

}  // namespace

void paged_plan_general(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count) {
  const int most = pb.max_new * pl.G;                              // rows that a sequence has for one KV head, at most
  const int R = most <= 4 ? 4 : most <= 16 ? 16 : 64;
  w->ppos = w->upos = R / pl.G;
  w->log_tk = 6;
  const long long tiles = (pb.max_len + (1 << w->log_tk) - 1) >> w->log_tk, units = (long long)pb.batch * pl.Hkv * paged_units(*w, pb.max_new);
  constexpr int per_sm = 2;
  w->by_unit = tiles <= (R == 64 ? 2 : 4);   // (prompts of 100 tokens x 4, 32 heads: whole 42 us, cut 49; of 200: whole 48, cut 32)
  w->min_tiles = w->by_unit || R == 64 ? 1 : 2;               // (the same prompt with shares of two tiles at least: 51 us)
  w->extra = 0;
  const long long most_ctas = w->by_unit ? units : (units * tiles + w->min_tiles - 1) / w->min_tiles;
  w->n_cta = (int)(most_ctas < (long long)per_sm * sm_count ? most_ctas : (long long)per_sm * sm_count);
  w->narrow = paged_narrow(*w, pb, pl);
  w->rows = (pb.max_new < w->upos ? pb.max_new : w->upos) * pl.G;
}

cudaError_t launch_paged_general(const PagedAttend& a, const void* k, const void* v, int q_bf16, int kv_bf16, cudaStream_t s) {
  if (q_bf16) return kv_bf16 ? general_dim<__nv_bfloat16, __nv_bfloat16>(a, k, v, s) : general_dim<__nv_bfloat16, float>(a, k, v, s);
  return kv_bf16 ? general_dim<float, __nv_bfloat16>(a, k, v, s) : general_dim<float, float>(a, k, v, s);
}

cudaError_t launch_paged_join(const PagedAttend& a, int out_bf16, cudaStream_t s) {
  if (!a.w.cuts) return cudaSuccess;
  auto kern = a.pl.d == 128 ? (out_bf16 ? paged_join_kernel<__nv_bfloat16, 128> : paged_join_kernel<float, 128>)
                            : (out_bf16 ? paged_join_kernel<__nv_bfloat16, 64> : paged_join_kernel<float, 64>);
  const int ys = a.w.rows >= 32 ? (a.w.rows * (a.pl.d / 4) + 2 * kJoinThreads - 1) / (2 * kJoinThreads) : (a.w.rows + 7) / 8;   // two items a thread at most, or a row a warp
  return launch_ex(kern, dim3(a.w.n_cta - 1, ys < 16 ? ys : 16), dim3(kJoinThreads), 0, s, 0, true, a);
}

}  // namespace spla
