// Attention over 8-bit pages for few query rows (single tokens, and a few of them: at most 16 rows of positions x the G heads of a KV head).
//
//   s_j = 2^a 2^ek(j) (q' . k8_j),  x_j = s_j scale log2 e (cap, distance),  y_j = x_j + ev(j),
//   w_j = 2^(y_j - m),  O += sum w_j v8_j,  l += sum w_j 2^-ev(j);  out = O / l,  lse = ln 2 (m + log2 l)
//
// The pages are read once and 8 bits at a time: that is what bounds such calls, so nothing else may take longer.  A tile of 128 tokens comes by TMA;
// every one of eight warps takes the 16 tokens of it that share a scale, from shared memory straight into the fragments of mma.m16n8k16
// (e4m3 is exact in fp16), rows of queries against tokens, and keeps its own running maximum, sum and output, which meet at the end of a
// segment.  (tcgen05 would want the values widened in shared memory: four times the traffic there, and 128 rows for 16.)  Which channel is which of a
// product's k, and which of its columns, is free: a lane takes 32 neighbouring bytes of a token of K, 16 of a token of V.
// The scales never touch the values: K's multiply a warp's 16 scores, V's are exponents and go into that of the weights, so that the
// weights of a row are at most 2^15, the largest at least 2^14, whatever the blocks' scales are, and fp16 holds them to 2^-11 of themselves and 2^-39 of the largest.  Queries are
// scaled by a power of two to below 2^15: fp16 holds bf16's eight bits down to 2^-28 of a row's largest channel.  Products are exact, sums fp32: each
// tile's are started anew and added to O in fp32 (the tensor core truncates when it adds into an accumulator).
//
// Warps: 8 or 16 as above; then one that brings tiles, scales and queries, one that plans the segments ahead (paged.h), one that looks up where their tiles lie.  Waits are bounded as in the other kernels.  No multicast.
//
// What bounds it: reading the pages.  32 heads in 8 groups of 128, graphs: one token on 32768 x8 115 us (82 at a copy's rate; bf16 pages 189), x8 heads of 64 75 (41), 17000 x64 375 (340; bf16 660), of
// 2000 to 32000 x64 under a cap, 40 heads, 393 to 400 (299; bf16 656), 300 x64 31 (6: segments of three tiles, each with its merge), four new tokens on 32768 x8 123.  About 8 us of each are the launch, 12 the ramp and
// the join.  Inside, of a small case (16384 x8): issue slots 46 %, tensor pipe 16 %, conversions the longest pipe (32 words of a warp's block, 8 cycles each).
// fp32 queries (two parts, twice the products): one token on 32768 x8 180 us, 300 x64 41, ragged under a cap 895 (the fp32 kernel: 1266, 123, 5235; heads of 128
// spill 37 to 45 registers a thread).
// Steps (32768 x8, which takes 117 now): eight warps of 16 rows each 133, places and scales looked up eight tiles ahead and the rows as columns (R8) 117; capped scores two at a time
// with the far form only where a score needs it 459 -> 400 (ragged).  Not kept: handing a stage back once its values are in registers (ragged 459 -> 490: the warps fall out of step and
// the stage waits for the last of them anyway), rings of K and V apart and the merge in halves (459 -> 543), four warps that widen to shared memory.
#include "paged_tiles.cuh"

namespace spla {

namespace {

constexpr int kPfBlocks = 8;                       // blocks of a tile, each a warp's
template <bool R8> constexpr int kPfWarps = R8 ? 2 * kPfBlocks : kPfBlocks;   // that compute
template <bool R8> constexpr int kPfThreads = 32 * (kPfWarps<R8> + 4);        // (whole groups of four warps, which share registers out: one of the last is idle)
constexpr int kPfKeys = 128;                       // tokens of a tile: 16 for each warp
constexpr int kPfRows = 16;
constexpr int kPfSegs = 4;                         // segments planned ahead
constexpr int kPfGroups = 4;                       // groups of 8 tiles whose places are looked up ahead
static_assert(kPfKeys == 16 * kPfBlocks, "a block of a scale for each warp");

struct PfSeg {
  int b, h, row0, n, L, prefix;
  int t0, t1, ns, skip;                            // key tiles
  bool head, tail, end;
};

template <int D>
struct PfSmem {
  // (An even number of stages: with R8 two sets of warps take the tiles in turn, and a stage has to be one set's alone.  A set that is ahead would take the
  // phase before, which is the other's, for the one that it waits for.)
  static constexpr int kTile = kPfKeys * D, NS = D == 128 ? 4 : 8;   // K and V of a stage: 2 kTile
  static_assert(NS % 2 == 0, "a stage is one set's");
  static constexpr int kRing = 0, kMerge = NS * 2 * kTile;           // float [8 warps][16 rows][D], or of 16 warps 8 rows
  static constexpr int kQ = kMerge + kPfBlocks * kPfRows * D * 4;    // bf16 [kPfSegs][16][D]
  static constexpr int kScales = kQ + kPfSegs * kPfRows * D * 2;     // int [NS][16]: exponents of K's blocks, of V's
  static constexpr int kMl = kScales + NS * 64;                      // float2 [8][16], [16][8]
  static constexpr int kWhere = kMl + kPfBlocks * kPfRows * 8;       // int [kPfGroups][8 tiles][24]: cache rows of the blocks, exponents of K's, of V's
  static constexpr int kSegs = kWhere + kPfGroups * 8 * 24 * 4;
  static constexpr int kSeqs = kSegs + (kPfSegs * (int)sizeof(PfSeg) + 15) / 16 * 16;
  static constexpr int kBars = kSeqs + ((int)sizeof(PagedSeqs) + 15) / 16 * 16;
  static constexpr int kMisc = kBars + (2 * NS + 3 * kPfSegs + 2 + 2 * kPfGroups) * 8;
  static constexpr int kBytes = kMisc + 16;
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t has_nan8(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t nan8_to_zero(uint32_t w) {
  const uint32_t m = has_nan8(w) >> 7;             // 1 in the bytes that are NaN
  return w & ~(m * 0xffu);
}
// 16-byte piece `c` of row `row` of a tile, as TMA's swizzle lays it.
template <int D>
__device__ __forceinline__ int piece_at(int row, int c) { return row * D + ((D == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4); }

// Two fp32 values as fp16 and what that leaves, as fp16 again (of an infinity nothing).
__device__ __forceinline__ void two_parts(float x, float y, uint32_t& first, uint32_t& rest) {
  first = pack_f16(x, y);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&first));
  rest = pack_f16(fabsf(x) < INFINITY ? x - f.x : 0.f, fabsf(y) < INFINITY ? y - f.y : 0.f);
}

// 8 x 8 values of 16 bits, two neighbours of a row in each lane: its transpose.
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(v));
  return y;
}

// R8: at most 8 rows.  Tokens and channels are the products' 16 rows then, the queries their 8 columns: half the products and half the registers, so
// that sixteen warps work, eight on a tile and eight on the next.
// F32: fp32 queries and outputs.  Queries and weights are two parts of fp16, 22 bits, each times the same fragments: channels are off by 2^-23 of a row's largest at most (its second part
// is up to 8 where the largest is 2^14, rounded to steps of 2^-8), weights by 2^-22 of themselves, or 2^-25 where the row's largest is 2^14 at least.
template <int D, bool MODS, bool R8, bool F32>
__global__ void __launch_bounds__(kPfThreads<R8>, 1)
    paged_few_kernel(const __grid_constant__ PagedAttend a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using SM = PfSmem<D>;
  constexpr int NS = SM::NS, WARPS = kPfWarps<R8>, THREADS = kPfThreads<R8>, ROWS = R8 ? 8 : kPfRows;
  constexpr int NT = R8 ? D / 16 : D / 8;          // tiles of the output: 16 channels x 8 rows, or 16 rows x 8 channels
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + SM::kBars);
  uint64_t *full = bars, *empty = full + NS, *seg_full = empty + NS, *seg_empty = seg_full + kPfSegs, *q_full = seg_empty + kPfSegs,
           *merge_full = q_full + kPfSegs, *merge_free = merge_full + 1, *where_full = merge_free + 1, *where_free = where_full + kPfGroups;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::kMisc);
  PfSeg* segs = reinterpret_cast<PfSeg*>(smem + SM::kSegs);
  PagedSeqs& seqs = *reinterpret_cast<PagedSeqs*>(smem + SM::kSeqs);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1);  mbar_init(&empty[s], kPfBlocks); }
    for (int s = 0; s < kPfSegs; ++s) { mbar_init(&seg_full[s], 1);  mbar_init(&seg_empty[s], WARPS + 2);  mbar_init(&q_full[s], 1); }
    for (int s = 0; s < kPfGroups; ++s) { mbar_init(&where_full[s], 1);  mbar_init(&where_free[s], 1); }
    mbar_init(merge_full, WARPS);
    mbar_init(merge_free, WARPS);
    mbar_init_done();
    *abort_flag = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  const long long share = paged_share(a.w, paged_fill_seqs(a, seqs, tid, THREADS));   // (ends with a barrier)
  const int lim = a.wait_limit, G = a.pl.G;
  bool ok = true;

  if (warp >= WARPS) {
  warpgroup_reg_dec<R8 ? 64 : 88>();               // (88 + 2 x 208 = 3 x 168, 64 + 4 x 104 = 5 x 96: what the CTA is launched with)
  if (warp == WARPS + 1) {
    // -------------------------------------------------------------- the share's segments, ahead of their use ----------------
    PagedWalk wk;
    bool more = wk.seek(a, seqs, blockIdx.x * share, share);
    const int4 cut = a.w.cuts ? wk.cut_here(a, more, share) : make_int4(0, 0, 0, 0);
#pragma unroll 1
    for (int i = 0;; ++i) {
      more = more && wk.next(a, seqs);
      PfSeg sg;
      if (more) {
        sg.t0 = wk.t0; sg.t1 = wk.t1; sg.ns = wk.ns; sg.skip = wk.skip;
        if (a.first_key) {                         // documents: from the first that a token sees on
          int least = 0x7fffffff;
          if (lane < wk.n) least = paged_sees(a, wk.row0, wk.n, wk.L, wk.prefix, lane).lo;
          sg.t0 = min(sg.t1, max(sg.t0, __reduce_min_sync(0xffffffffu, least) / kPfKeys));
        }
      }
      if (i >= kPfSegs && !pm_wait(&seg_empty[i % kPfSegs], (i / kPfSegs - 1) & 1, lim, abort_flag)) { ok = false; break; }
      if (lane == 0) {
        sg.end = !more;
        if (more) {
          sg.b = wk.b; sg.h = wk.h; sg.row0 = wk.row0; sg.n = wk.n; sg.L = wk.L; sg.prefix = wk.prefix;
          sg.head = wk.head; sg.tail = wk.tail;
        }
        segs[i % kPfSegs] = sg;
        mbar_arrive1(&seg_full[i % kPfSegs]);
      }
      __syncwarp();
      if (!more) break;
    }
    if (a.w.cuts && lane == 0) a.w.cuts[blockIdx.x] = cut;
  } else if (warp == WARPS) {
    // -------------------------------------------------------------- tiles, scales, queries ----------------------------------
    // Lane 16 v + i: K's (v = 0) or V's (v = 1) block i of a tile: its scale, and where it is the first of a page, the page's box.
    const int i8 = lane & 15, is_v = lane >> 4, P = a.pl.P;
    const bool mine = i8 < kPfBlocks, boxes = mine && (16 * i8 & (P - 1)) == 0;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    const uint32_t dst = smem_u32(smem) + SM::kRing + is_v * SM::kTile + 16 * i8 * D;
    const int n_rows = (int)((long long)a.pl.n_pages * a.pl.page_stride);          // (a box there reads zeros)
    const int* where = reinterpret_cast<const int*>(smem + SM::kWhere);
    int* sc_s = reinterpret_cast<int*>(smem + SM::kScales);
    int kt = 0, i = 0, group = 0;
    for (; ok; ++i) {
      const int slot = i % kPfSegs;
      if (!pm_wait(&seg_full[slot], (i / kPfSegs) & 1, lim, abort_flag)) { ok = false; break; }
      const PfSeg sg = segs[slot];
      if (sg.end) break;
      if (!F32 && lane == 0) mbar_expect_tx(&q_full[slot], sg.n * G * D * 2 + (uint32_t)a.dbg_tx_extra);
      __syncwarp();
      if (!F32 && lane < sg.n)                       // (fp32 queries: straight from memory, there is no place for them)
        bulk_g2s(smem + SM::kQ + (slot * kPfRows + lane * G) * D * 2,
                 reinterpret_cast<const __nv_bfloat16*>(a.q) + (sg.row0 + lane) * a.q_stride + (long long)sg.h * G * D, G * D * 2, &q_full[slot]);
#pragma unroll 1
      for (int t = sg.t0; t < sg.t1 && ok; t += 8, ++group) {
        if (!pm_wait(&where_full[group % kPfGroups], (group / kPfGroups) & 1, lim, abort_flag)) { ok = false; break; }
#pragma unroll 1
        for (int u = 0; u < min(8, sg.t1 - t); ++u, ++kt) {
          const int* at = where + ((group % kPfGroups) * 8 + u) * 24;
          const int row = mine ? at[i8] : 0, e = mine ? at[8 + is_v * 8 + i8] : 0, st = kt % NS;
          if (kt >= NS && !pm_wait(&empty[st], ((kt / NS) - 1) & 1, lim, abort_flag)) { ok = false; break; }
          if (mine) sc_s[st * 16 + is_v * 8 + i8] = e;
          __syncwarp();
          if (lane == 0) mbar_expect_tx(&full[st], 2 * SM::kTile + (uint32_t)a.dbg_tx_extra);
          __syncwarp();
          if (boxes) tma_load_box(dst + st * 2 * SM::kTile, map, 0, row < 0 ? n_rows : row, &full[st]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive1(&where_free[group % kPfGroups]);
      }
      if (!ok) { ++i; break; }                     // (its queries are on their way)
      __syncwarp();
      if (lane == 0) mbar_arrive1(&seg_empty[slot]);
    }
    if (!ok) *abort_flag = 1;
    // every copy has landed before the CTA leaves, whatever the other roles do
    for (int x = max(0, kt - NS); x < kt; ++x) warp_waits(&full[x % NS], (x / NS) & 1, lim);
    for (int x = max(0, i - kPfSegs); x < i && !F32; ++x) warp_waits(&q_full[x % kPfSegs], (x / kPfSegs) & 1, lim);
  } else if (warp == WARPS + 2) {
    // -------------------------------------------------------------- where tiles lie, and their scales: eight tiles at a time --------
    // (a byte of a scale comes from memory like anything else, behind the page's number: a microsecond, which one tile would not hide)
    const int i8 = lane & 7;
    int* where = reinterpret_cast<int*>(smem + SM::kWhere);
    int group = 0;
    for (int i = 0; ok; ++i) {
      const int slot = i % kPfSegs;
      if (!pm_wait(&seg_full[slot], (i / kPfSegs) & 1, lim, abort_flag)) { ok = false; break; }
      const PfSeg sg = segs[slot];
      if (sg.end) break;
      auto find = [&](int t) {                     // cache row of this lane's block, -1: none
        const int tok = (t < sg.ns ? t : t + sg.skip) * kPfKeys + 16 * i8;
        if (t >= sg.t1 || tok >= sg.L) return -1;
        const long long r = paged_row(a.pb, a.pl, sg.b, sg.h, tok >> a.pl.log_p);
        return r < 0 ? -1 : (int)(r + (tok & (a.pl.P - 1)));
      };
#pragma unroll 1
      for (int t = sg.t0; t < sg.t1; t += 8, ++group) {
        int row[2], ek[2], ev[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) row[x] = find(t + 4 * x + (lane >> 3));
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          ek[x] = row[x] < 0 ? 0 : paged_exponent(a.k_scales + (row[x] >> 4));
          ev[x] = row[x] < 0 ? 0 : paged_exponent(a.v_scales + (row[x] >> 4));
        }
        if (group >= kPfGroups && !pm_wait(&where_free[group % kPfGroups], ((group / kPfGroups) - 1) & 1, lim, abort_flag)) { ok = false; break; }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          int* at = where + ((group % kPfGroups) * 8 + 4 * x + (lane >> 3)) * 24 + i8;
          at[0] = row[x];
          at[8] = ek[x];
          at[16] = ev[x];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive1(&where_full[group % kPfGroups]);
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive1(&seg_empty[slot]);
    }
  }
  } else {
    // -------------------------------------------------------------- scores, weights, output ----------------------------------
    warpgroup_reg_inc<R8 ? 104 : 208>();
    // g: a row of the products' left operand (and + 8), a column of the right one; t4: four channels of a k-step, two columns of the result
    const int g = lane >> 2, t4 = lane & 3, block = warp & (kPfBlocks - 1);
    const float sc2 = a.sm_scale * kLog2e;
    const float cap = a.softcap, to_u = MODS && cap > 0.f ? 1.f / (cap * kLog2e) : 0.f;
    const int* sc_s = reinterpret_cast<const int*>(smem + SM::kScales);
    float2* ml_s = reinterpret_cast<float2*>(smem + SM::kMl);
    float* merge = reinterpret_cast<float*>(smem + SM::kMerge);
    // rows of this lane's scores: row(0), row(1); tokens of them in a block: token(0), ... (two of R8, four)
    constexpr int TOKENS = R8 ? 2 : 4;
    auto row_of = [&](int x) { return R8 ? 2 * t4 + x : g + 8 * x; };
    auto token_of = [&](int y) { return R8 ? g + 8 * y : 2 * t4 + (y & 1) + 4 * (y & 2); };
    int kt = 0;
#pragma unroll 1
    for (int i = 0; ok; ++i) {
      const int slot = i % kPfSegs;
      if (!pm_wait(&seg_full[slot], (i / kPfSegs) & 1, lim, abort_flag)) { ok = false; break; }
      const PfSeg& sg = segs[slot];
      if (sg.end) break;
      const int rows = sg.n * G;
      // what the rows see
      PagedSees see[2];
      float slope2[2];
      int pos[2];
      int lo_least = 0x7fffffff, lo_most = 0, hi_least = 0x7fffffff, hi_most = 0;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = row_of(x), pi = r / G;
        see[x] = PagedSees{0x7fffffff, 0};
        slope2[x] = 0.f;
        pos[x] = sg.L - sg.n + pi;
        if (r < rows) {
          see[x] = paged_sees(a, sg.row0, sg.n, sg.L, sg.prefix, pi);
          if (MODS && a.slopes) slope2[x] = __ldg(a.slopes + sg.h * G + r - pi * G) * kLog2e;
          lo_least = min(lo_least, see[x].lo);
          lo_most = max(lo_most, see[x].lo);
          hi_least = min(hi_least, see[x].hi);
          hi_most = max(hi_most, see[x].hi);
        }
      }
      lo_least = __reduce_min_sync(0xffffffffu, lo_least);
      lo_most = __reduce_max_sync(0xffffffffu, lo_most);
      hi_least = __reduce_min_sync(0xffffffffu, hi_least);
      hi_most = __reduce_max_sync(0xffffffffu, hi_most);
      // queries as fragments: k-step j takes bytes 4 j .. of the lane's 32 (16) channels; rows g (and g + 8)
      uint32_t qf[D / 16][R8 ? 2 : 4], ql[F32 ? D / 16 : 1][4];
      int qe[2];
      if (!F32 && !pm_wait(&q_full[slot], (i / kPfSegs) & 1, lim, abort_flag)) { ok = false; break; }
#pragma unroll
      for (int x = 0; x < (R8 ? 1 : 2); ++x) {
        const int r = g + 8 * x;
        if constexpr (F32) {
          float w[D / 4];
          const float4* from = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + (sg.row0 + r / G) * a.q_stride + ((long long)sg.h * G + r % G) * D + t4 * (D / 4));
#pragma unroll
          for (int y = 0; y < D / 16; ++y) {
            const float4 v = r < rows ? from[y] : make_float4(0.f, 0.f, 0.f, 0.f);
            w[4 * y] = v.x; w[4 * y + 1] = v.y; w[4 * y + 2] = v.z; w[4 * y + 3] = v.w;
          }
          float top = 0.f;
#pragma unroll
          for (int y = 0; y < D / 4; ++y)
            if (fabsf(w[y]) < INFINITY) top = fmaxf(top, fabsf(w[y]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          qe[x] = top > 0.f ? max((__float_as_int(top) >> 23) - 127 - 14, -100) : 0;
          const float mul = power_of_two(-qe[x]);
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int y = 0; y < 2; ++y) two_parts(w[4 * j + 2 * y] * mul, w[4 * j + 2 * y + 1] * mul, qf[j][2 * y + x], ql[j][2 * y + x]);
          continue;
        }
        uint32_t w[D / 8];
        if (r < rows) {
          const uint4* from = reinterpret_cast<const uint4*>(smem + SM::kQ + (slot * kPfRows + r) * D * 2 + t4 * (D / 2));
#pragma unroll
          for (int y = 0; y < D / 32; ++y) {
            const uint4 v = from[y];
            w[4 * y] = v.x; w[4 * y + 1] = v.y; w[4 * y + 2] = v.z; w[4 * y + 3] = v.w;
          }
        } else {
#pragma unroll
          for (int y = 0; y < D / 8; ++y) w[y] = 0u;
        }
        float top = 0.f;
#pragma unroll
        for (int y = 0; y < D / 8; ++y) {
          const float lo = fabsf(bf16_lo(w[y])), hi = fabsf(bf16_hi(w[y]));
          if (lo < INFINITY) top = fmaxf(top, lo);
          if (hi < INFINITY) top = fmaxf(top, hi);
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        qe[x] = top > 0.f ? max((__float_as_int(top) >> 23) - 127 - 14, -100) : 0;
        const float mul = power_of_two(-qe[x]);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          qf[j][x] = pack_f16(bf16_lo(w[2 * j]) * mul, bf16_hi(w[2 * j]) * mul);
          qf[j][(R8 ? 1 : 2) + x] = pack_f16(bf16_lo(w[2 * j + 1]) * mul, bf16_hi(w[2 * j + 1]) * mul);
        }
      }
      if constexpr (R8) {                          // (of the rows that the lane's scores are of)
        const int e = qe[0];
        qe[0] = __shfl_sync(0xffffffffu, e, 8 * t4);
        qe[1] = __shfl_sync(0xffffffffu, e, 8 * t4 + 4);
      }
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float o[NT][4];
#pragma unroll
      for (int x = 0; x < NT; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
#pragma unroll 1
      for (int t = sg.t0, t1 = sg.t1; t < t1; ++t, ++kt) {
        if (R8 && (kt & 1) != warp / kPfBlocks) continue;
        const int st = kt % NS, key0 = (t < sg.ns ? t : t + sg.skip) * kPfKeys + 16 * block;
        if (!pm_wait(&full[st], (kt / NS) & 1, lim, abort_flag)) { ok = false; break; }
        if (key0 < hi_most && (key0 + 16 > lo_least || key0 < a.sinks)) {
          const bool part = key0 < lo_most || key0 + 16 > hi_least;
          const unsigned char *kt_s = smem + SM::kRing + st * 2 * SM::kTile, *vt_s = kt_s + SM::kTile;
          const int ek = sc_s[st * 16 + block], ev = sc_s[st * 16 + 8 + block];
          // ---- scores: tokens g and g + 8 of the block are the lane's
          uint32_t kw[2][D / 16];
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
              const uint4 v = *reinterpret_cast<const uint4*>(kt_s + piece_at<D>(16 * block + 8 * nt + g, t4 * (D / 64) + x));
              kw[nt][4 * x] = v.x; kw[nt][4 * x + 1] = v.y; kw[nt][4 * x + 2] = v.z; kw[nt][4 * x + 3] = v.w;
            }
          float p[2][TOKENS];                      // of a row: its scores, then weights
          {
            float s[2][2][4];                      // the channels' sums in two parts
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int y = 0; y < 2; ++y) s[x][y][0] = s[x][y][1] = s[x][y][2] = s[x][y][3] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
              uint32_t b[2][2];
              widen(kw[0][j], b[0][0], b[0][1]);
              widen(kw[1][j], b[1][0], b[1][1]);
              if constexpr (R8) {
                const uint32_t left[4] = {b[0][0], b[1][0], b[0][1], b[1][1]};
                mma_f16(s[0][j & 1], left, qf[j][0], qf[j][1]);
              } else {
                mma_f16(s[0][j & 1], qf[j], b[0][0], b[0][1]);
                mma_f16(s[1][j & 1], qf[j], b[1][0], b[1][1]);
                if constexpr (F32) {
                  mma_f16(s[0][j & 1], ql[j], b[0][0], b[0][1]);
                  mma_f16(s[1][j & 1], ql[j], b[1][0], b[1][1]);
                }
              }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int y = 0; y < TOKENS; ++y) {
                const int at = R8 ? 2 * y + x : 2 * x + (y & 1), nt = R8 ? 0 : y >> 1;
                p[x][y] = s[nt][0][at] + s[nt][1][at];
              }
          }
          // values on their way: tokens 2 t4, + 1, + 8, + 9; channels D / 8 g ..
          uint32_t v[4][D / 32];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int row = 16 * block + 2 * t4 + (x & 1) + 4 * (x & 2);
            if constexpr (D == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(vt_s + piece_at<D>(row, g));
              v[x][0] = y.x; v[x][1] = y.y; v[x][2] = y.z; v[x][3] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(vt_s + piece_at<D>(row, g >> 1) + (g & 1) * 8);
              v[x][0] = y.x; v[x][1] = y.y;
            }
          }
          // ---- weights
          float f[2], top[2], up[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) up[x] = power_of_two(min(max(qe[x] + ek, -126), 127));
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < TOKENS; ++y) p[x][y] = p[x][y] * up[x] * sc2;
          if constexpr (MODS) {
            if (cap > 0.f) {                       // cap tanh(z / cap), in base 2 (see paged_mma.cuh)
              float most = 0.f;
#pragma unroll
              for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < TOKENS; ++y) most = fmaxf(most, fabsf(p[x][y]));
              const bool far = __any_sync(0xffffffffu, most * to_u >= kCapNear);
#pragma unroll
              for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < TOKENS; y += 2) {
                  const float2 z = make_float2(p[x][y], p[x][y + 1]), u = __fmul2_rn(z, make_float2(to_u, to_u)), u2 = __fmul2_rn(u, u);
                  float2 c = __ffma2_rn(u2, make_float2(kTanh3, kTanh3), make_float2(kTanh2, kTanh2));
                  c = __ffma2_rn(u2, c, make_float2(kTanh1, kTanh1));
                  c = __fmul2_rn(z, __ffma2_rn(u2, c, make_float2(kTanh0, kTanh0)));
                  p[x][y] = c.x;
                  p[x][y + 1] = c.y;
                  if (far) {
                    auto other = [&](float& to, float v) {
                      if (fabsf(v) >= kCapNear) to = copysignf(fmaf(-2.f, rcp_approx(1.f + ex2(fabsf(v) * (2.f * kLog2e))), 1.f), v) * (cap * kLog2e);
                    };
                    other(p[x][y], u.x);
                    other(p[x][y + 1], u.y);
                  }
                }
            }
            if (a.slopes)
#pragma unroll
              for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < TOKENS; ++y) p[x][y] = fmaf(-slope2[x], fabsf((float)(key0 - pos[x] + token_of(y))), p[x][y]);
          }
          if (part)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int y = 0; y < TOKENS; ++y) {
                const int j = key0 + token_of(y);
                if (!((j >= see[x].lo || j < a.sinks) && j < see[x].hi)) p[x][y] = -INFINITY;
              }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            top[x] = -INFINITY;
#pragma unroll
            for (int y = 0; y < TOKENS; ++y) top[x] = fmaxf(top[x], p[x][y]);
            top[x] += (float)(ev - 15);
            f[x] = 1.f;
          }
          // The first tokens that a row sees set its maximum, one above what their weights need; later ones only move it when a weight would exceed 2^15.
          // (From scores of 2^24 on fp32 counts in steps of 2 and more, and the largest weight may come out up to a step above 2^15, which fp16 would not hold, or below 2^14,
          // but never below 1: the weights are held to 2^15, for O and l alike, which is less than the score's own rounding does.)
          if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
              for (int w = R8 ? 4 : 1; w < (R8 ? 32 : 4); w <<= 1) top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], w));
              if (top[x] > m[x]) {
                f[x] = ex2(m[x] - (top[x] + 1.f));
                m[x] = top[x] + 1.f;
              }
            }
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float mn = m[x];
            const float nm = mn == -INFINITY ? 0.f : (float)ev - mn;
            float sum = 0.f;
#pragma unroll
            for (int y = 0; y < TOKENS; ++y) {
              p[x][y] = ex2(min_or_nan(p[x][y] + nm, 15.f));
              sum += p[x][y];
            }
            l[x] = fmaf(l[x], f[x], sum * power_of_two(-ev));
          }
          uint32_t pf[R8 ? 2 : 4], pl[4];
          if constexpr (R8) {
            pf[0] = transposed(pack_f16(p[0][0], p[1][0]));
            pf[1] = transposed(pack_f16(p[0][1], p[1][1]));
          } else if constexpr (F32) {
            two_parts(p[0][0], p[0][1], pf[0], pl[0]);
            two_parts(p[1][0], p[1][1], pf[1], pl[1]);
            two_parts(p[0][2], p[0][3], pf[2], pl[2]);
            two_parts(p[1][2], p[1][3], pf[3], pl[3]);
          } else {
            pf[0] = pack_f16(p[0][0], p[0][1]);
            pf[1] = pack_f16(p[1][0], p[1][1]);
            pf[2] = pack_f16(p[0][2], p[0][3]);
            pf[3] = pack_f16(p[1][2], p[1][3]);
          }
          bool bad = false;
          if (part) {                              // values that no row sees are zeroed (0 x NaN is no 0)
            const bool alike = sg.n == 1;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int j = key0 + 2 * t4 + (x & 1) + 4 * (x & 2);
              const bool seen = j < hi_most && (j >= lo_least || j < a.sinks);
#pragma unroll
              for (int y = 0; y < D / 32; ++y) {
                if (!seen) v[x][y] = 0u;
                if (!alike && has_nan8(v[x][y])) {
                  bad = true;
                  v[x][y] = nan8_to_zero(v[x][y]);
                }
              }
            }
            bad = __any_sync(0xffffffffu, bad);
          }
          // ---- output.  Tile x holds channels D / 8 column + x of two rows; of R8, channels D / 8 g + 2 x (and + 1) of two rows
          const float2 f0 = R8 ? make_float2(f[0], f[1]) : make_float2(f[0], f[0]), f1 = R8 ? f0 : make_float2(f[1], f[1]);
          auto add = [&](float (&d)[4], const float (&c)[4]) {
            const float2 d0 = __ffma2_rn(make_float2(d[0], d[1]), f0, make_float2(c[0], c[1]));
            const float2 d1 = __ffma2_rn(make_float2(d[2], d[3]), f1, make_float2(c[2], c[3]));
            d[0] = d0.x; d[1] = d0.y; d[2] = d1.x; d[3] = d1.y;
          };
#pragma unroll
          for (int y = 0; y < D / 32; ++y) {
            uint32_t b[2][4];                      // of tokens (2 t4, + 1) and (+ 8, + 9): four channels
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              widen(__byte_perm(v[2 * x][y], v[2 * x + 1][y], 0x5140), b[x][0], b[x][1]);
              widen(__byte_perm(v[2 * x][y], v[2 * x + 1][y], 0x7362), b[x][2], b[x][3]);
            }
            if constexpr (R8) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                const uint32_t left[4] = {b[0][2 * x], b[0][2 * x + 1], b[1][2 * x], b[1][2 * x + 1]};
                mma_f16(c, left, pf[0], pf[1]);
                add(o[2 * y + x], c);
              }
            } else {
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(c, pf, b[0][x], b[1][x]);
                if constexpr (F32) mma_f16(c, pl, b[0][x], b[1][x]);
                add(o[4 * y + x], c);
              }
            }
          }
          if (bad) {                               // rows that see a token with such a value: its channels are NaN
#pragma unroll 1
            for (int j = 0; j < 16; ++j) {
              const int key = key0 + j;
              const bool sees0 = (key >= see[0].lo || key < a.sinks) && key < see[0].hi, sees1 = (key >= see[1].lo || key < a.sinks) && key < see[1].hi;
              if (!sees0 && !sees1) continue;
              const float nan = __int_as_float(0x7fffffff);
              constexpr int HAS = R8 ? D / 8 : D / 4;   // neighbouring channels of the lane
#pragma unroll
              for (int x = 0; x < HAS; x += 4) {
                const int c = (R8 ? g : t4) * HAS + x;
                const uint32_t w = *reinterpret_cast<const uint32_t*>(vt_s + piece_at<D>(16 * block + j, c >> 4) + (c & 15)), which = has_nan8(w);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                  constexpr int half = D / 8;
                  const int tile = R8 ? (x + y) / 2 : (x + y) % half, at0 = R8 ? 2 * ((x + y) & 1) : (x + y) / half, at1 = R8 ? at0 + 1 : 2 + at0;
                  if (which & (0x80u << (8 * y))) {
                    if (sees0) o[tile][at0] = nan;
                    if (sees1) o[tile][at1] = nan;
                  }
                }
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive1(&empty[st]);
      }
      if (!ok) break;
      // ---- the warps' results meet: 16 bytes of a row at a time, laid so that neither side meets itself on a bank
      if (i > 0 && !pm_wait(merge_free, (i - 1) & 1, lim, abort_flag)) { ok = false; break; }
      constexpr int Q4 = R8 ? D / 32 : D / 16;     // 16-byte pieces that a lane has of a row
      auto turn_of_row = [](int r, int tt) { return R8 ? (D == 128 ? r >> 1 & 3 : (r >> 1 & 1) | (r & 4)) : D == 128 ? (2 * tt) ^ (r & 1) : (tt >> 1) | ((r & 1) << 1); };
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int w = R8 ? 4 : 1; w < (R8 ? 32 : 4); w <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], w);
        const int r = row_of(x), mine = R8 ? g : t4;
        if (r >= rows) continue;
        if ((R8 ? g : t4) == 0) ml_s[warp * ROWS + r] = make_float2(m[x], l[x]);
        float4* to = reinterpret_cast<float4*>(merge + (warp * ROWS + r) * D);
        const int turn = turn_of_row(r, t4);
#pragma unroll
        for (int y = 0; y < Q4; ++y) {
          float4 w;
          if constexpr (R8) {
            w = make_float4(o[2 * y][x], o[2 * y][2 + x], o[2 * y + 1][x], o[2 * y + 1][2 + x]);
          } else {
            constexpr int half = D / 8;
            const int c = 4 * y, col = 2 * x + c / half, tile = c % half;
            w = make_float4(o[tile][col], o[tile + 1][col], o[tile + 2][col], o[tile + 3][col]);
          }
          to[mine * Q4 + y ^ turn] = w;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive1(merge_full);
      if (!pm_wait(merge_full, i & 1, lim, abort_flag)) { ok = false; break; }
      const bool whole = sg.head && sg.tail;
      const long long part0 = (2LL * blockIdx.x + (sg.head ? 1 : 0)) * a.w.rows;
#pragma unroll 1
      for (int x = tid; x < rows * (D / 4); x += 32 * WARPS) {
        const int r = x / (D / 4), q4 = x % (D / 4), at = q4 ^ turn_of_row(r & 7, q4 / Q4);
        float M = -INFINITY, sum = 0.f;
#pragma unroll
        for (int y = 0; y < WARPS; ++y) {
          const float2 ml = ml_s[y * ROWS + r];
          if (ml.y != 0.f) M = fmaxf(M, ml.x);
        }
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int y = 0; y < WARPS; ++y) {
          const float2 ml = ml_s[y * ROWS + r];
          if (ml.y == 0.f) continue;               // (no token seen)
          const float w = ex2(ml.x - M);
          const float4 z = *(reinterpret_cast<const float4*>(merge + (y * ROWS + r) * D) + at);
          sum = fmaf(ml.y, w, sum);
          v.x = fmaf(z.x, w, v.x); v.y = fmaf(z.y, w, v.y); v.z = fmaf(z.z, w, v.z); v.w = fmaf(z.w, w, v.w);
        }
        const int pi = r / G;
        const long long out_row = (long long)(sg.row0 + pi) * a.pl.Hq + sg.h * G + r - pi * G;
        if (whole) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          if constexpr (F32)
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + out_row * D + 4 * q4) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
          else
            *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + out_row * D + 4 * q4) =
                make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
          if (q4 == 0 && a.lse) a.lse[out_row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
        } else {
          *reinterpret_cast<float4*>(a.w.part_o + (part0 + r) * D + 4 * q4) = v;
          if (q4 == 0) a.w.part_ml[part0 + r] = make_float2(M, sum);
        }
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive1(merge_free);
        mbar_arrive1(&seg_empty[slot]);
      }
    }
  }
  if (!ok) *abort_flag = 1;
  __syncwarp();
  __syncthreads();
  if (*abort_flag && tid == 0) atomicExch(a.pl.status, kStatusTimeout);
}

template <int D, bool MODS, bool R8, bool F32>
cudaError_t few_launch(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) {
  auto kern = paged_few_kernel<D, MODS, R8, F32>;
  static unsigned long long allowed = 0;
  cudaError_t e = allow_smem_once(kern, PfSmem<D>::kBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(a.w.n_cta), dim3(kPfThreads<R8>), PfSmem<D>::kBytes, s, 0, true, a, *reinterpret_cast<const CUtensorMap*>(maps.k),
                   *reinterpret_cast<const CUtensorMap*>(maps.v));
}
template <int D>
cudaError_t few_dim(const PagedAttend& a, const PagedMaps& maps, int f32, cudaStream_t s) {
  const bool mods = a.softcap > 0.f || a.slopes;
  if (f32) return mods ? few_launch<D, true, false, true>(a, maps, s) : few_launch<D, false, false, true>(a, maps, s);   // (two parts fill the registers of eight warps)
  if (a.w.rows <= 8) return mods ? few_launch<D, true, true, false>(a, maps, s) : few_launch<D, false, true, false>(a, maps, s);
  return mods ? few_launch<D, true, false, false>(a, maps, s) : few_launch<D, false, false, false>(a, maps, s);
}

}  // namespace

// (32768 x8, 32 heads in 8 groups of 128, graphs: 16 rows take 123 us here, and the 20 to 32 of the tensor-core kernel 166, which would take fewer no less.)
int paged_few_positions(const PagedLayout& pl) { return kPfRows / pl.G; }

void paged_plan_few(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count) {
  w->ppos = w->upos = paged_few_positions(pl);
  w->log_tk = 7;
  static_assert(kPfKeys == 1 << 7, "tokens per tile");
  const long long tiles = (pb.max_len + kPfKeys - 1) / kPfKeys, units = (long long)pb.batch * pl.Hkv;
  w->by_unit = tiles <= 4 || (tiles <= 12 && units <= sm_count && 4 * units >= sm_count);   // (as in paged_mma.cu)
  w->min_tiles = w->by_unit ? 1 : 2;
  w->extra = 1;
  const long long most = w->by_unit ? units : (units * tiles + w->min_tiles - 1) / w->min_tiles;
  w->n_cta = (int)(most < sm_count ? most : sm_count);
  w->narrow = paged_narrow(*w, pb, pl);
  w->rows = (pb.max_new < w->upos ? pb.max_new : w->upos) * pl.G;
}

cudaError_t launch_paged_few(const PagedAttend& a, const PagedMaps& maps, int f32, cudaStream_t s) {
  return a.pl.d == 128 ? few_dim<128>(a, maps, f32, s) : few_dim<64>(a, maps, f32, s);
}

}  // namespace spla
