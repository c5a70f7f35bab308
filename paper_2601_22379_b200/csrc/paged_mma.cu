// Attention of new tokens over a paged cache on the 5th-generation tensor cores: bf16 cache and queries.
//
//   S = Q K^T,  P = 2^(S scale log2 e - m),  O += P V,  l += sum P    over tiles of 128 keys; lse = ln 2 (m + log2 l), out = O / l
//
// One CTA per SM, persistent, on an equal share of all key tiles (paged.h).  Two row tiles of 128 query rows (positions x the G heads
// of one KV head) are in work at a time, each with its own softmax warps and its own S and O in tensor memory, so that the tensor cores
// work on one while the other is in its exponentials:
//   - a unit of more than one row tile: two row tiles against the same key tile, K and V are read once for both;
//   - a unit of one row tile (short chunks): the same rows against key tiles in turn, the two halves merged at the end.
// Launches whose units have at most 32 rows (single tokens, FEW) hold the rows four times, a copy for each softmax warp, which takes 32
// of the tile's 128 keys: its row of P has zeros elsewhere, its rows of O and l are sums over its keys, and the four are merged at the
// end.  (One warp with all 128 keys of the rows was the whole chain: capped scores of 64 ragged sequences 978 us, 618 so on the same box.)
// P takes the place of S in tensor memory, as the left operand of O += P V, rounded to bf16, half a step of 2^-8, as the outputs are
// (error of out against float64, 2-norm: 2.3e-3 for single tokens, 2.1e-3 for prompts, of which the rounding of out is 1.7e-3; a second part of P
// would take 24 products in place of 16, and their issue is what bounds prompts).  Its sum l is of the unrounded values, so that lse is as
// exact as the scores.  The maximum is a stale one: O is rescaled only when it
// grows by more than 2^8.  The tensor core truncates when it adds into an accumulator: every kPmDrain tiles the softmax warps take O into fp32
// sums of their own in the workspace (sums of a million keys came out 0.4 % low without, of four million 2.3 %).
//
// Warps: 0 and 2 TMA (pages of K and the query rows as boxes of G heads x positions; pages of V), 1 the MMA issuer, 3 plans the
// segments ahead of the others, 4 to 7 and 8 to 11 softmax and epilogue of either row tile, one row per thread.
//
// What bounds it.  Single tokens: reading K and V (8 sequences of 32768, 8 KV heads: 5.7 to 6.0 TB/s by box, 0.87 to 0.92 of a copy's
// rate).  Prompts: products issue at about 82 cycles each (64 would be the tensor pipe's own time: S reads both operands from shared
// memory, at its full rate), 16 per row tile and key tile, and each row tile's chain of scores, softmax (about 1900 cycles), P and product is
// not quite hidden behind the other's: 8192 tokens, 32 heads of 128: 0.59 to 0.62 ms by box, 0.89 to 0.93 PFLOP/s.  Slower, on a box where
// this took 533 us: scores in halves of 64 keys with two buffers (623 us: twice the instructions at the same 82 cycles); P handed over in
// halves (561); a quarter of the exponentials by polynomial on the FMA pipe (565); loading S twice instead of holding a row in registers.
//
// Keys outside a row's mask: their scores are replaced before the maximum, whatever they are.  Values are looked over in tiles that
// some row sees only in part: behind the sequence's end they are zeroed, and where one that is not finite is inside, the tile's product
// with V is formed by the softmax warps, visible keys only (0 x infinity is no 0).
//
// Every wait is bounded; on expiry the CTA's roles leave their loops, copies and products in flight are waited for, tensor memory is
// released and the time-out status latched.  No multicast.
#include <type_traits>

#include "paged.h"
#include "umma.cuh"

namespace spla {

namespace {

constexpr int kPmThreads = 384;
constexpr int kPmKeys = 128;                       // keys per tile
constexpr int kPmDrain = 128;                      // tiles that are added up in O before it is drained: 1024 truncations, each of less than 2^-23: 2^-13 at most
constexpr uint32_t kPmTmemCols = 512;              // S0, S1, O0, O1: 128 columns each

template <int D, bool FEW>
struct PmSmem {
  static constexpr int H = D / 64;                               // arrays of 128-byte rows per operand
  static constexpr int kHalf = kPmKeys * 128;
  static constexpr int kTile = H * kHalf;                        // one K or V tile, or the queries of a row tile
  // stages: V is held until its softmax is through, K only until the scores; one row tile leaves room for another of V
  static constexpr int NK = D == 128 ? 2 : 4, NV = (D == 128 ? 2 : 4) + (FEW ? (D == 128 ? 1 : 2) : 0);
  static constexpr int kQ = 0, kK = kQ + (FEW ? 1 : 2) * kTile, kV = kK + NK * kTile, kSeqs = kV + NV * kTile;
  static constexpr int kMl = kSeqs + (int)((sizeof(PagedSeqs) + 15) / 16 * 16);   // float2 [128]: maximum and sum of the second half, of a quarter
  static constexpr int kSegs = kMl + 128 * 8;                     // PmSeg [4]: the segments that come next
  static constexpr int kStage = kSegs + 4 * 96;                   // [8 warps][32 rows][64 + 16 bytes], FEW [4 warps][8 rows][512 + 16] or fewer columns of more rows: rows on their way out
  static constexpr int kStageRow = 80;
  static constexpr int kBars = kStage + 8 * 32 * 80;
  static constexpr int kNumBars = 2 * NK + 2 * NV + 15 + 8;
  static constexpr int kMisc = kBars + kNumBars * 8;             // tensor-memory base, abort flag, skip flags [2], look-over marks [2][2]
  static constexpr int kBytes = kMisc + 48;
  static_assert(4 * 32 * 144 <= 8 * 32 * 80 && 4 * 16 * 272 <= 8 * 32 * 80 && 4 * 8 * 528 <= 8 * 32 * 80, "rows on their way out");
  static_assert(kBytes <= 227 * 1024, "shared memory of the paged attention kernel");
  static_assert(kPmKeys >= 128, "positions of a row tile (see PmPlan)");
};

// What the roles agree on for one segment: which key tiles either row tile walks, and which of them every row sees whole.
// No tile between A and E is walked by neither: row tile 1 has at most 128 positions, as many as a tile has keys, right behind those of row
// tile 0, so that the first key that one of its rows sees lies at most 127 behind the last that row tile 0 sees: a1 <= e0 (and e1 >= e0 > a0),
// whatever the documents, the window and the prefix.
struct PmPlan {
  bool single;                                     // one row tile, key tiles in turn
  int a0, e0, a1, e1;                              // key tiles of row tile 0, of row tile 1
  int A, E;                                        // of either
  int la0, le0, la1, le1;                          // seen whole by all rows (the values of the others are looked over)
  template <int S>
  __device__ __forceinline__ bool act(int t) const { return single ? ((t - A) & 1) == S : S == 0 ? t >= a0 && t < e0 : t >= a1 && t < e1; }
  template <int S>
  __device__ __forceinline__ bool look(int t) const { return single || S == 0 ? t < la0 || t >= le0 : t < la1 || t >= le1; }
  __device__ __forceinline__ int items(int s) const { return single ? (E - A + 1 - s) >> 1 : s == 0 ? e0 - a0 : e1 - a1; }
};

// (whole warps)
__device__ __forceinline__ void pm_row_tile(const PagedAttend& a, const PagedWalk& wk, int lane, int ia, int ib, int& ta, int& te, int& la, int& le) {
  ta = te = la = le = 0;
  if (ib < ia) return;
  const int first = wk.L - wk.n;
  int lo = a.window > 0 ? max(0, first + ia - a.window + 1) : 0;
  int all_lo = a.window > 0 ? max(0, first + ib - a.window + 1) : 0;
  const int hi = min(wk.L, max(first + ib + 1, wk.prefix)), all_hi = min(wk.L, max(first + ia + 1, wk.prefix));
  if (a.first_key) {
    int least = 0x7fffffff, most = 0;
    for (int i = ia + lane; i <= ib; i += 32) {
      const PagedSees v = paged_sees(a, wk.row0, wk.n, wk.L, wk.prefix, i);
      if (v.lo < v.hi) least = min(least, v.lo);
      most = max(most, v.lo);
    }
    lo = __reduce_min_sync(0xffffffffu, least);
    all_lo = __reduce_max_sync(0xffffffffu, most);
  }
  if (lo >= hi) return;
  ta = max(wk.t0, lo / kPmKeys);
  te = max(ta, min(wk.t1, (hi + kPmKeys - 1) / kPmKeys));
  la = all_lo / kPmKeys + (all_lo % kPmKeys != 0);
  le = all_hi / kPmKeys;
}
__device__ __forceinline__ PmPlan pm_plan(const PagedAttend& a, const PagedWalk& wk, int lane) {
  PmPlan p;
  p.single = wk.n <= a.w.ppos;
  const int i0 = wk.first_pos(a.w), end = min(wk.n, i0 + wk.n_pos(a.w));
  pm_row_tile(a, wk, lane, i0, min(end, i0 + a.w.ppos) - 1, p.a0, p.e0, p.la0, p.le0);
  pm_row_tile(a, wk, lane, i0 + a.w.ppos, (p.single ? 0 : min(end, i0 + 2 * a.w.ppos)) - 1, p.a1, p.e1, p.la1, p.le1);
  const bool h0 = p.e0 > p.a0, h1 = p.e1 > p.a1;
  p.A = h0 && h1 ? min(p.a0, p.a1) : h0 ? p.a0 : p.a1;
  p.E = h0 && h1 ? max(p.e0, p.e1) : h0 ? p.e0 : p.e1;
  return p;
}

// One segment as the scheduling warp hands it to the other roles.
struct PmSeg {
  PmPlan pl;
  int b, h, row0, n, L, prefix, first;             // first: its first new token, in the sequence
  bool head, tail, end;                            // end: none is left
};
constexpr int kPmSegs = 4;
static_assert(sizeof(PmSeg) <= 96, "a segment's place");

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

constexpr float kCapNear = 0.375f;                 // up to here tanh goes by a polynomial
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, int half, int head, int tok, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(map), "r"(0), "r"(half), "r"(head), "r"(tok), "r"(smem_u32(bar))
               : "memory");
}
// 128 consecutive columns of this thread's tensor-memory lane.
__device__ __forceinline__ void tmem_ld128(uint32_t addr, uint32_t (&r)[128]) {
#pragma unroll
  for (int x = 0; x < 4; ++x) tmem_ld32_async(addr + 32 * x, reinterpret_cast<uint32_t(&)[32]>(r[32 * x]));
#pragma unroll
  for (int x = 0; x < 4; ++x) tmem_ld_wait32(reinterpret_cast<uint32_t(&)[32]>(r[32 * x]));
}
// bits a .. e - 1 of a word (a, e in any range)
__device__ __forceinline__ uint32_t bits_between(int a, int e) {
  const uint32_t below_e = e >= 32 ? 0xffffffffu : e <= 0 ? 0u : (1u << e) - 1u;
  const uint32_t below_a = a >= 32 ? 0xffffffffu : a <= 0 ? 0u : (1u << a) - 1u;
  return below_e & ~below_a;
}
__device__ __forceinline__ uint32_t pair_not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// A thread's row of O into its sums, [slot of a CTA][D / 4][128 threads] 16 bytes each and then [128] of l: sums = sums f + O, or O where there
// are none yet.  And back, for the end of a segment: O = sums f + O; returns l.
__device__ __forceinline__ float* pm_sums(float* drain, int slot, int d) { return drain + (2LL * blockIdx.x + slot) * (128 * (d + 1)); }
template <int D>
__device__ __forceinline__ void pm_drain(uint32_t tO, float* drain, int slot, int thr, float f, bool fresh, float l) {
  float *place = pm_sums(drain, slot, D) + 4 * thr, *place_l = pm_sums(drain, slot, D) + 128 * D + thr;
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t o[16];
    tmem_ld16_async(tO + c, o);
    tmem_ld_wait16(o);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float4* at = reinterpret_cast<float4*>(place) + (c / 4 + x) * 128;
      float4 v = make_float4(__uint_as_float(o[4 * x]), __uint_as_float(o[4 * x + 1]), __uint_as_float(o[4 * x + 2]), __uint_as_float(o[4 * x + 3]));
      if (!fresh) {
        const float4 s = *at;
        v.x = fmaf(s.x, f, v.x); v.y = fmaf(s.y, f, v.y); v.z = fmaf(s.z, f, v.z); v.w = fmaf(s.w, f, v.w);
      }
      *at = v;
    }
  }
  *place_l = fresh ? l : fmaf(*place_l, f, l);
}
template <int D>
__device__ __forceinline__ float pm_undrain(uint32_t tO, float* drain, int slot, int thr, float f, float l) {
  const float *place = pm_sums(drain, slot, D) + 4 * thr, *place_l = pm_sums(drain, slot, D) + 128 * D + thr;
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t o[16];
    tmem_ld16_async(tO + c, o);
    tmem_ld_wait16(o);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float4 s = *(reinterpret_cast<const float4*>(place) + (c / 4 + x) * 128);
      const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int y = 0; y < 4; ++y) o[4 * x + y] = __float_as_uint(fmaf(v[y], f, __uint_as_float(o[4 * x + y])));
    }
    tmem_st16(tO + c, o);
  }
  tmem_st_wait();
  return fmaf(*place_l, f, l);
}

// LONG: caches of more than kPmDrain tiles (the others go without what drains O: 106 us for a mixed batch in place of 108).
template <int D, bool MODS, bool FEW, bool LONG>
__global__ void __launch_bounds__(kPmThreads, 1)
    paged_mma_kernel(const PagedAttend a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_q) {
  using SM = PmSmem<D, FEW>;
  constexpr int H = SM::H, NK = SM::NK, NV = SM::NV;
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + SM::kBars);
  uint64_t *k_full = bars, *k_empty = k_full + NK, *v_full = k_empty + NK, *v_empty = v_full + NV, *q_full = v_empty + NV, *q_empty = q_full + 1,
           *s_full = q_empty + 1, *p_ready = s_full + 2, *pv_done = p_ready + 2, *o_free = pv_done + 2, *scanned = o_free + 2, *halves = scanned + 2,
           *quarters = halves + 1, *done = quarters + 1, *seg_full = done + 1, *seg_empty = seg_full + kPmSegs;
  uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(smem + SM::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::kMisc + 4);
  volatile int* skip_pv = reinterpret_cast<volatile int*>(smem + SM::kMisc + 8);    // [2]: this product with V has been formed by the softmax warps
  volatile int* found_bad = reinterpret_cast<volatile int*>(smem + SM::kMisc + 16); // [2][2]: the last look-over (of even, of odd number) that found such a value
  float2* ml_s = reinterpret_cast<float2*>(smem + SM::kMl);
  PagedSeqs& seqs = *reinterpret_cast<PagedSeqs*>(smem + SM::kSeqs);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wg = warp >> 2;

  if (tid == 0) {
    for (int s = 0; s < NK; ++s) { mbar_init(&k_full[s], 1);  mbar_init(&k_empty[s], 1); }
    for (int s = 0; s < NV; ++s) { mbar_init(&v_full[s], 1);  mbar_init(&v_empty[s], 1); }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);  mbar_init(&p_ready[s], 4);
      mbar_init(&pv_done[s], 1);  mbar_init(&o_free[s], 4);
      mbar_init(&scanned[s], 4);
      skip_pv[s] = 0;
      found_bad[2 * s] = found_bad[2 * s + 1] = 0;
    }
    mbar_init(halves, 4);
    mbar_init(quarters, 4);
    mbar_init(done, 1);
    for (int s = 0; s < kPmSegs; ++s) { mbar_init(&seg_full[s], 1);  mbar_init(&seg_empty[s], 11); }   // K, V, MMA and eight softmax warps
    mbar_init_done();
    *abort_flag = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
  }
  if (warp == 1) tmem_alloc(tmem_base_s, kPmTmemCols);
  pdl_wait();
  pdl_launch_dependents();
  tc_fence_before();
  const long long share = paged_share(a.w, paged_fill_seqs(a, seqs, tid, kPmThreads));   // (ends with a barrier)
  tc_fence_after();
  const uint32_t tmem = *tmem_base_s;
  const uint32_t sbase = smem_u32(smem);
  const int lim = a.wait_limit;
  const int ppos = a.w.ppos, G = a.pl.G;
  PmSeg* segs = reinterpret_cast<PmSeg*>(smem + SM::kSegs);
  // The CTA's segments, one after the other: the body returns false to give up.
  auto each_segment = [&](bool& ok, auto body) {
#pragma unroll 1
    for (int i = 0; ok; ++i) {
      if (!pm_wait(&seg_full[i % kPmSegs], (i / kPmSegs) & 1, lim, abort_flag)) { ok = false; break; }
      const PmSeg& sg = segs[i % kPmSegs];
      if (sg.end) break;
      if (!body(sg)) { ok = false; break; }
      __syncwarp();
      if (lane == 0) mbar_arrive1(&seg_empty[i % kPmSegs]);
    }
  };

  if (wg == 0) {
    warpgroup_reg_dec<120>();                                     // (120 + 2 x 192 = 3 x 168, what the CTA is launched with)
    if (warp == 0 || warp == 2) {
      // ------------------------------------------------------------ TMA: queries and K, or V ----------------------------
      const bool is_k = warp == 0;
      const int NS = is_k ? NK : NV;
      const int P = a.pl.P, npg = kPmKeys / P, boxes = npg * H, pg = lane / H, hh = lane % H;
      const uint32_t dst = sbase + (is_k ? SM::kK : SM::kV) + hh * SM::kHalf + pg * P * 128;
      const CUtensorMap* map = is_k ? &map_k : &map_v;
      uint64_t *full = is_k ? k_full : v_full, *empty = is_k ? k_empty : v_empty;
      const int n_rows = (int)((a.pl.n_pages - 1) * a.pl.page_stride + (a.pl.Hkv - 1) * a.pl.head_stride + P);   // (a box there reads zeros)
      int kt = 0, seg = 0;
      bool ok = true;
      each_segment(ok, [&](const PmSeg& sg) {
        const PmPlan pl = sg.pl;
        if (pl.A >= pl.E) return true;
        const int L = sg.L, b = sg.b, h = sg.h;
        // row of this lane's box in tile t; loaded a tile ahead
        auto box_row = [&](int t) {
          const int index = t * npg + pg;
          long long r = -1;
          if (lane < boxes && t < pl.E && index * P < L) r = paged_row(a.pb, a.pl, b, h, index);
          return r < 0 ? n_rows : (int)r;
        };
        int row = box_row(pl.A);
        if (is_k) {
          if (seg > 0 && !pm_wait(q_empty, (seg - 1) & 1, lim, abort_flag)) return false;
          if (lane == 0) {
            const bool two = !pl.single && pl.items(1) > 0;
            const int boxes_q = FEW ? 4 : two ? 2 : 1;             // (four copies of the same rows, or the row tiles)
            mbar_expect_tx(q_full, boxes_q * H * ppos * G * 128 + (uint32_t)a.dbg_tx_extra);
            for (int s = 0; s < boxes_q; ++s)
              for (int x = 0; x < H; ++x)
                tma_load_q(sbase + SM::kQ + s * (FEW ? 32 * 128 : SM::kTile) + x * SM::kHalf, &map_q, x, h * G,
                           sg.row0 + sg.first + (FEW ? 0 : s * ppos), q_full);
          }
        }
        ++seg;
        for (int t = pl.A; t < pl.E; ++t) {
          const int row_next = box_row(t + 1);
          const int st = kt % NS;
          if (kt >= NS && !pm_wait(&empty[st], ((kt / NS) - 1) & 1, lim, abort_flag)) return false;
          if (lane == 0) mbar_expect_tx(&full[st], SM::kTile + (uint32_t)a.dbg_tx_extra);
          __syncwarp();
          if (lane < boxes) tma_load_box(dst + st * SM::kTile, map, hh * 64, row, &full[st]);
          ++kt;
          row = row_next;
        }
        return true;
      });
      if (!ok) *abort_flag = 1;
      // every copy has landed before the CTA leaves, whatever the other roles do
      for (int x = max(0, kt - NS); x < kt; ++x) warp_waits(&full[x % NS], (x / NS) & 1, lim);
      if (is_k && seg > 0) warp_waits(q_full, (seg - 1) & 1, lim);
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMA issuer -----------------------------------------
      constexpr uint32_t id_s = umma_idesc(true, false, false, 128, kPmKeys);
      constexpr uint32_t id_o = umma_idesc(true, false, true, 128, D);
      constexpr uint32_t kStep = 2048 / 16;                       // 16 keys of V
      const uint32_t one = elect_one();                           // (the whole warp runs this loop: see umma_ss_one)
      const uint32_t q_lo = umma_desc_lo(sbase + SM::kQ, 16), k_lo = umma_desc_lo(sbase + SM::kK, 16), v_lo = umma_desc_lo(sbase + SM::kV, SM::kHalf);
      bool ok = true;
      uint32_t kt = 0;
      int seg = 0;
      uint32_t n_p0 = 0, n_p1 = 0, n_o0 = 0, n_o1 = 0;            // items whose P was awaited, segments that used O
      // the item of either row tile whose product with V is to come: its stage and phase, whether it is the segment's first, its number
      // there, whether V is free after it, whether the softmax warps may have formed it
      bool pend0 = false, pend1 = false, first0 = true, first1 = true, free0 = false, free1 = false, look0 = false, look1 = false;
      int st0 = 0, st1 = 0, it0 = 0, it1 = 0;
      uint32_t ph0 = 0, ph1 = 0;
      auto product = [&](auto slot_c) {                           // O (+)= P V
        constexpr int S = decltype(slot_c)::value;
        bool &pend = S ? pend1 : pend0, &first = S ? first1 : first0;
        int& it = S ? it1 : it0;
        uint32_t &n_p = S ? n_p1 : n_p0, &n_o = S ? n_o1 : n_o0;
        const int st = S ? st1 : st0;
        pend = false;
        if (!pm_wait(&v_full[st], S ? ph1 : ph0, lim, abort_flag) || !pm_wait(&p_ready[S], n_p & 1, lim, abort_flag)) { ok = false; return; }
        ++n_p;
        if (first) {
          if (n_o > 0 && !pm_wait(&o_free[S], (n_o - 1) & 1, lim, abort_flag)) { ok = false; return; }
          ++n_o;
        }
        tc_fence_after();
        if (!((S ? look1 : look0) && skip_pv[S])) {
          const uint32_t pt = tmem + S * 128, o = tmem + 256 + S * 128, v = v_lo + st * (SM::kTile / 16);
          umma_ts4_one<8, kStep>(one, o, pt, v, id_o, first || (LONG && it % kPmDrain == 0) ? 0u : 1u);
          umma_ts4_one<8, kStep>(one, o, pt + 32, v + 4 * kStep, id_o, 1u);
        }
        first = false;
        if (LONG) ++it;
        umma_commit_one(one, &pv_done[S]);
        if (S ? free1 : free0) umma_commit_one(one, &v_empty[st]);
      };
      constexpr std::integral_constant<int, 0> s0{};
      constexpr std::integral_constant<int, 1> s1{};
      auto score = [&](auto slot_c, const PmPlan& pl, int t, bool last) {   // S = Q K^T
        constexpr int S = decltype(slot_c)::value;
        if (S ? pend1 : pend0) product(slot_c);                   // (S takes the place of the P before)
        const uint32_t q = q_lo + (FEW || pl.single ? 0 : S * (SM::kTile / 16)), k = k_lo + kt % NK * (SM::kTile / 16);
#pragma unroll
        for (int x = 0; x < H; ++x) umma_ss4_one<2, 2>(one, tmem + S * 128, q + x * (SM::kHalf / 16), k + x * (SM::kHalf / 16), id_s, x > 0);
        umma_commit_one(one, &s_full[S]);
        if (last) umma_commit_one(one, &k_empty[kt % NK]);
        (S ? pend1 : pend0) = true;
        (S ? st1 : st0) = kt % NV;
        (S ? ph1 : ph0) = (kt / NV) & 1;
        (S ? free1 : free0) = last;
        (S ? look1 : look0) = pl.template look<S>(t);
      };
      each_segment(ok, [&](const PmSeg& sg) {
        const PmPlan pl = sg.pl;
        if (pl.A >= pl.E) return true;
        if (!pm_wait(q_full, seg & 1, lim, abort_flag)) return false;
        ++seg;
        first0 = first1 = true;
        it0 = it1 = 0;
#pragma unroll 1
        for (int t = pl.A; t < pl.E; ++t) {
          const bool act0 = pl.act<0>(t), act1 = pl.act<1>(t);
          if (!pm_wait(&k_full[kt % NK], (kt / NK) & 1, lim, abort_flag)) return false;
          tc_fence_after();
          if (act0) {
            score(s0, pl, t, !act1);
            if (ok && pend1) product(s1);
          }
          if (ok && act1) {
            score(s1, pl, t, true);
            if (ok && pend0) product(s0);
          }
          if (!ok) return false;
          ++kt;
        }
        umma_commit_one(one, q_empty);
        if (pend0) product(s0);
        if (ok && pend1) product(s1);
        return ok;
      });
      umma_commit_one(one, done);
      if (!warp_waits(done, 0, lim)) ok = false;
      if (!ok) *abort_flag = 1;
    } else {
      // ------------------------------------------------------------ scheduling: the share's segments, ahead of their use ---
      PagedWalk wk;
      bool more = wk.seek(a, seqs, blockIdx.x * share, share);
      const int4 cut = a.w.cuts ? wk.cut_here(a, more, share) : make_int4(0, 0, 0, 0);
#pragma unroll 1
      for (int i = 0;; ++i) {
        more = more && wk.next(a, seqs);
        PmSeg sg;
        if (more) sg.pl = pm_plan(a, wk, lane);
        if (i >= kPmSegs && !pm_wait(&seg_empty[i % kPmSegs], (i / kPmSegs - 1) & 1, lim, abort_flag)) { *abort_flag = 1; break; }
        if (lane == 0) {
          sg.end = !more;
          if (more) {
            sg.b = wk.b; sg.h = wk.h; sg.row0 = wk.row0; sg.n = wk.n; sg.L = wk.L; sg.prefix = wk.prefix;
            sg.first = wk.first_pos(a.w);
            sg.head = wk.head; sg.tail = wk.tail;
          }
          segs[i % kPmSegs] = sg;
          mbar_arrive1(&seg_full[i % kPmSegs]);
        }
        __syncwarp();
        if (!more) break;
      }
      if (a.w.cuts && lane == 0) a.w.cuts[blockIdx.x] = cut;
    }
  } else {
    // -------------------------------------------------------------- softmax and epilogue: one row per thread -------------
    warpgroup_reg_inc<192>();
    const int slot = wg - 1, thr = tid - 128 * wg, row = FEW ? lane : thr, pi = row / G, g = row % G;
    constexpr int KEYS = FEW ? 32 : kPmKeys;                      // keys of a tile that a thread takes
    const int kb = FEW ? 32 * (warp & 3) : 0;                     // the first of them
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + slot * 128 + lane_off, tO = tmem + 256 + slot * 128 + lane_off;
    const float sc2 = a.sm_scale * kLog2e;
    const float to_u = MODS && a.softcap > 0.f ? a.sm_scale / a.softcap : 0.f, sq_u = to_u * to_u;
    const float cap0 = 0.99999994f * sc2, cap1 = -0.33331972f * sc2 * sq_u, cap2 = 0.13284431f * sc2 * sq_u * sq_u,
                cap3 = -0.048268907f * sc2 * sq_u * sq_u * sq_u;   // (a score of 1 is sc2 in base 2)
    bool ok = true;
    int kt = 0, n = 0, n_scan = 0, n_half = 0, n_quarter = 0, n_used = 0;   // tiles of the CTA, items of this slot, look-overs, merges, segments that used O
    each_segment(ok, [&](const PmSeg& sg) {
      int t, t_end, t_step, la, le, k_base, my;                   // this slot's tiles, those seen whole, the tile counter's offset
      bool single, second, alike;
      PagedSees see{0x7fffffff, 0};
      bool valid;
      int pos;
      float slope2 = 0.f;
      {
        const PmPlan pl = sg.pl;
        single = pl.single;
        second = single && pl.items(1) > 0;
        alike = sg.n == 1;
        my = pl.items(slot);
        t = single ? pl.A + slot : slot ? pl.a1 : pl.a0;
        t_end = single ? pl.E : slot ? pl.e1 : pl.e0;
        t_step = single ? 2 : 1;
        la = single || !slot ? pl.la0 : pl.la1;
        le = single || !slot ? pl.le0 : pl.le1;
        k_base = kt - pl.A;
        kt += pl.E - pl.A;
        const int i = sg.first + (single ? 0 : slot * ppos) + pi;
        valid = row < ppos * G && i < sg.n;
        if (valid || alike) see = paged_sees(a, sg.row0, sg.n, sg.L, sg.prefix, alike ? 0 : i);
        if (MODS && a.slopes && valid) slope2 = __ldg(a.slopes + sg.h * G + g) * kLog2e;
        pos = sg.L - sg.n + i;
      }
      const bool live = __any_sync(0xffffffffu, valid);
      const bool counts = valid || alike;
      const int lo_most = __reduce_max_sync(0xffffffffu, counts ? see.lo : 0), hi_least = __reduce_min_sync(0xffffffffu, counts ? see.hi : 0x7fffffff);
      float m = -INFINITY, l = 0.f, fd = 1.f;                      // fd: what the sums of drained tiles are behind the maximum
      int done_items = 0;
#pragma unroll 1
      for (; t < t_end; t += t_step) {
        const int tok0 = t * kPmKeys, st = (uint32_t)(k_base + t) % NV;
        const bool look = t < la || t >= le;
        bool simt = false;
        if (!pm_wait(&s_full[slot], n & 1, lim, abort_flag)) return false;
        if (LONG && done_items > 0 && done_items % kPmDrain == 0 && live) {
          if (!pm_wait(&pv_done[slot], (n - 1) & 1, lim, abort_flag)) return false;
          tc_fence_after();
          pm_drain<D>(tO, a.w.drain, slot, thr, fd, done_items == kPmDrain, l);   // (the next product starts O anew)
          l = 0.f;
          fd = 1.f;
        }
        if (look) {
          // (After the scores: they were issued behind the products of all tiles up to two before this one, each of which waited for its V, so
          // that the parity below can only mean this tile.)
          // Values of this tile.  Where all rows see the same keys (single tokens) the rows of the others are zeroed; otherwise they are
          // looked over: zeroed behind the end where they are not finite, and elsewhere such a value makes the tile special.
          if (!pm_wait(&v_full[st], ((uint32_t)(k_base + t) / NV) & 1, lim, abort_flag)) return false;
          unsigned char* vt = smem + SM::kV + st * SM::kTile;
          bool bad = false;
          if (alike) {
            const int from = lo_most - tok0, to = hi_least - tok0;
            for (int j = thr >> 3; j < kPmKeys; j += 16)           // a row of 128 bytes by eight threads
              if (j < from || j >= to) {
#pragma unroll
                for (int x = 0; x < H; ++x) *reinterpret_cast<uint4*>(vt + x * SM::kHalf + j * 128 + (thr & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
              }
          } else {
            vt += thr * 16;                                       // 16-byte pieces: rows thr / 8 + 16 x of either array
            __nv_bfloat162 most = __floats2bfloat162_rn(0.f, 0.f); // the largest magnitude, NaN above all
#pragma unroll 8
            for (int x = 0; x < SM::kTile / 2048; ++x) {
              const uint4 v = *reinterpret_cast<const uint4*>(vt + x * 2048);
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) most = __hmax2_nan(most, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[e])));
            }
            if (pair_not_finite(*reinterpret_cast<const uint32_t*>(&most))) {
              const int L = sg.L;
#pragma unroll 1
              for (int x = 0; x < SM::kTile / 2048; ++x) {
                const uint4 v = *reinterpret_cast<const uint4*>(vt + x * 2048);
                if (pair_not_finite(v.x) | pair_not_finite(v.y) | pair_not_finite(v.z) | pair_not_finite(v.w)) {
                  if (tok0 + (thr >> 3) + 16 * (x & 7) >= L) *reinterpret_cast<uint4*>(vt + x * 2048) = make_uint4(0u, 0u, 0u, 0u);
                  else bad = true;
                }
              }
            }
          }
          proxy_fence();                                          // (zeros written -> tensor core)
          const int mark = 2 * slot + (n_scan & 1);              // (a warp is at most one look-over ahead of another)
          if (__any_sync(0xffffffffu, bad) && lane == 0) found_bad[mark] = n_scan + 1;
          __syncwarp();
          if (lane == 0) mbar_arrive1(&scanned[slot]);
          if (!pm_wait(&scanned[slot], n_scan & 1, lim, abort_flag)) return false;
          simt = __any_sync(0xffffffffu, found_bad[mark] == n_scan + 1);
          ++n_scan;
        }
        tc_fence_after();
        if (live) {
          const int key0 = tok0 + kb;
          const bool part = key0 < lo_most || key0 + KEYS > hi_least;     // (warp-uniform)
          const float mul = MODS ? 1.f : sc2;
          uint32_t r[KEYS];
          if constexpr (FEW) {
            tmem_ld32_async(tS + kb, r);
            tmem_ld_wait32(r);
          } else {
            tmem_ld128(tS, r);
          }
          if constexpr (MODS) {
            if (a.softcap > 0.f) {
              // cap tanh(u), u = x / cap, in base 2.  Up to |u| = 3/8 an odd polynomial (interpolated at Chebyshev nodes, 6e-8 off), its coefficients
              // scaled to the raw scores; where a row of the warp has more, 1 - 2 / (1 + e^(2 |u|)) there, which alone would be off by
              // 2^-22 of the cap, however small the score, and takes two of the exponential unit's turns per key.
              float most = 0.f;
#pragma unroll
              for (int x = 0; x < KEYS; x += 2) most = max3(most, fabsf(__uint_as_float(r[x])), fabsf(__uint_as_float(r[x + 1])));
              auto near = [&](float2 v) {
                const float2 z = __fmul2_rn(v, v);
                float2 y = __ffma2_rn(z, make_float2(cap3, cap3), make_float2(cap2, cap2));
                y = __ffma2_rn(z, y, make_float2(cap1, cap1));
                return __fmul2_rn(__ffma2_rn(z, y, make_float2(cap0, cap0)), v);
              };
              if (!__any_sync(0xffffffffu, valid && most * to_u >= kCapNear)) {
#pragma unroll
                for (int x = 0; x < KEYS; x += 2) {
                  const float2 y = near(make_float2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])));
                  r[x] = __float_as_uint(y.x);
                  r[x + 1] = __float_as_uint(y.y);
                }
              } else {
                const float c2 = a.softcap * kLog2e, k2 = 2.f * kLog2e * to_u;
#pragma unroll
                for (int x = 0; x < KEYS; x += 2) {
                  const float2 v = make_float2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), y = near(v);
                  const float t0 = fmaf(-2.f, rcp_approx(1.f + ex2(fabsf(v.x) * k2)), 1.f), t1 = fmaf(-2.f, rcp_approx(1.f + ex2(fabsf(v.y) * k2)), 1.f);
                  r[x] = __float_as_uint(fabsf(v.x) * to_u >= kCapNear ? copysignf(t0 * c2, v.x) : y.x);
                  r[x + 1] = __float_as_uint(fabsf(v.y) * to_u >= kCapNear ? copysignf(t1 * c2, v.y) : y.y);
                }
              }
            } else {
#pragma unroll
              for (int x = 0; x < KEYS; ++x) r[x] = __float_as_uint(__uint_as_float(r[x]) * sc2);
            }
            if (a.slopes) {
              const float d0 = (float)(key0 - pos);
#pragma unroll
              for (int x = 0; x < KEYS; ++x) r[x] = __float_as_uint(fmaf(-slope2, fabsf(d0 + (float)x), __uint_as_float(r[x])));
            }
          }
          if (part) {
#pragma unroll
            for (int c = 0; c < KEYS / 32; ++c) {
              const uint32_t bits = bits_between(see.lo - key0 - 32 * c, see.hi - key0 - 32 * c);
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!(bits & (1u << x))) r[32 * c + x] = 0xff800000u;
            }
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int x = 0; x < KEYS; x += 2) mx[x / 2 & 3] = fmaxf(mx[x / 2 & 3], fmaxf(__uint_as_float(r[x]), __uint_as_float(r[x + 1])));
          const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * mul;
          // The first visible keys of a row set its maximum (its row of O is zero so far); later ones only move it when it would
          // let a probability exceed 2^8.
          const bool grow = mt > m + 8.f && m > -INFINITY;
          if (m == -INFINITY) m = mt;
          if (__any_sync(0xffffffffu, grow)) {
            if (!pm_wait(&pv_done[slot], (n - 1) & 1, lim, abort_flag)) return false;   // every product with P so far
            tc_fence_after();
            const float m_new = grow ? mt : m, f = grow ? ex2(m - m_new) : 1.f;
            m = m_new;
            l *= f;
            if (LONG) fd *= f;
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_ld16_async(tO + c, o);
              tmem_ld_wait16(o);
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              tmem_st16(tO + c, o);
            }
          }
          const float nm = m == -INFINITY ? 0.f : -m;
          float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
#pragma unroll
          for (int c = 0; c < KEYS / 32; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const float2 v = __ffma2_rn(make_float2(__uint_as_float(r[32 * c + 2 * x]), __uint_as_float(r[32 * c + 2 * x + 1])), make_float2(mul, mul), make_float2(nm, nm));
              const float2 p = make_float2(ex2(v.x), ex2(v.y));
              if (x & 1) sum1 = __fadd2_rn(sum1, p); else sum0 = __fadd2_rn(sum0, p);
              pk[x] = pack_bf16(p.x, p.y);
            }
            tmem_st16(tS + kb / 2 + 16 * c, pk);
          }
          if constexpr (FEW) {                                    // the keys of the other warps
            uint32_t zero[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) zero[x] = 0u;
#pragma unroll
            for (int c = 1; c < 4; ++c) tmem_st16(tS + (((warp & 3) + c) & 3) * 16, zero);
          }
          l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
          tmem_st_wait();
        }
        if (simt) {
          const bool begun = LONG ? done_items % kPmDrain != 0 : done_items > 0;          // O holds products already
          // the product with V here: O += sum over the row's visible keys of p v
          if (done_items > 0 && !pm_wait(&pv_done[slot], (n - 1) & 1, lim, abort_flag)) return false;
          if (done_items == 0 && n_used > 0 && !pm_wait(&o_free[slot], (n_used - 1) & 1, lim, abort_flag)) return false;
          tc_fence_after();
          const unsigned char* vt = smem + SM::kV + st * SM::kTile;
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            float acc[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[x] = 0.f;
#pragma unroll 1
            for (int w = FEW ? kb / 32 : 0; w < (FEW ? kb / 32 + 1 : 4); ++w) {
              uint32_t pw[16];
              tmem_ld16_async(tS + 16 * w, pw);
              tmem_ld_wait16(pw);
              const uint32_t bits = valid ? bits_between(see.lo - tok0 - 32 * w, see.hi - tok0 - 32 * w) : 0u;
#pragma unroll
              for (int y = 0; y < 32; ++y) {
                if (!(bits & (1u << y))) continue;
                const float p = (y & 1) ? bf16_hi(pw[y >> 1]) : bf16_lo(pw[y >> 1]);
                const int j = 32 * w + y;
                const unsigned char* vr = vt + (c >> 6) * SM::kHalf + j * 128;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  const uint4 v = *reinterpret_cast<const uint4*>(vr + (((((c & 63) >> 3) + x) ^ (j & 7)) << 4));
                  const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                  for (int z = 0; z < 4; ++z) {
                    acc[8 * x + 2 * z] = fmaf(p, bf16_lo(q[z]), acc[8 * x + 2 * z]);
                    acc[8 * x + 2 * z + 1] = fmaf(p, bf16_hi(q[z]), acc[8 * x + 2 * z + 1]);
                  }
                }
              }
              __syncwarp();
            }
            uint32_t o[16];
            if (begun) {
              tmem_ld16_async(tO + c, o);
              tmem_ld_wait16(o);
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(begun ? __uint_as_float(o[x]) + acc[x] : acc[x]);
            tmem_st16(tO + c, o);
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (look && lane == 0 && (warp & 3) == 0) skip_pv[slot] = simt;
        if (lane == 0) mbar_arrive1(&p_ready[slot]);
        ++n;
        ++done_items;
      }
      // ------------------------------------------------------------ end of the segment ----------------------------------
      const bool whole = sg.head && sg.tail;
      if (my > 0) {
        if (!pm_wait(&pv_done[slot], (n - 1) & 1, lim, abort_flag)) return false;
        tc_fence_after();
        ++n_used;
      }
      if (LONG && my > kPmDrain && live) l = pm_undrain<D>(tO, a.w.drain, slot, thr, fd, l);
      float m1 = -INFINITY, l1 = 0.f;
      if (second) {
        if (slot == 1) {                                          // the second half's maxima and sums go to the first's warps, O stays where it is
          ml_s[thr] = make_float2(m, l);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive1(halves);
        } else {
          if (!pm_wait(halves, n_half & 1, lim, abort_flag)) return false;
          tc_fence_after();
          const float2 o = ml_s[thr];
          m1 = o.x;
          l1 = o.y;
        }
        ++n_half;
      }
      if (single && slot == 1) return true;
      // O of both halves relative to the larger maximum; an empty half (no key seen) takes no part
      float M = fmaxf(m, m1);
      float f0 = l == 0.f ? 0.f : ex2(m - M), f1 = l1 == 0.f ? 0.f : ex2(m1 - M);
      float sum = (l == 0.f ? 0.f : l * f0) + (l1 == 0.f ? 0.f : l1 * f1);
      if constexpr (FEW) {                                        // ... and of the four warps' keys
        ml_s[thr] = make_float2(M, sum);
        __syncwarp();
        if (lane == 0) mbar_arrive1(quarters);
        if (!pm_wait(quarters, n_quarter & 1, lim, abort_flag)) return false;
        ++n_quarter;
        float top = -INFINITY, all = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) top = fmaxf(top, ml_s[32 * x + lane].x);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float2 o = ml_s[32 * x + lane];
          if (o.y != 0.f) all = fmaf(o.y, ex2(o.x - top), all);
        }
        const float f = sum == 0.f ? 0.f : ex2(M - top);
        f0 *= f;
        f1 *= f;
        M = top;
        sum = all;
      }
      const float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
      const float w0 = f0 * inv, w1 = f1 * inv;
      const int i0 = sg.first + (single ? 0 : slot * ppos);
      const long long out_row = (long long)(sg.row0 + i0 + pi) * a.pl.Hq + sg.h * G + g;
      const long long part_row = (2LL * blockIdx.x + (sg.head ? 1 : 0)) * a.w.rows + (single ? 0 : slot * ppos * G) + row;
      if constexpr (FEW) {
        // The four warps' rows meet in shared memory, as many columns at a time as fit; a thread adds and writes 8 columns of a row.
        const int n_rows = min(ppos, sg.n - i0) * G, cols = n_rows <= 8 ? (D < 128 ? D : 128) : n_rows <= 16 ? 64 : 32;
        const int r_cap = n_rows <= 8 ? 8 : n_rows <= 16 ? 16 : 32, r_bytes = cols * 4 + 16, pieces = cols >> 3;
        unsigned char* stage = smem + SM::kStage;
        const int r = thr / pieces, piece = thr - r * pieces, ri = r / G;
        const long long o_row = (long long)(sg.row0 + i0 + ri) * a.pl.Hq + sg.h * G + (r - ri * G);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += cols) {
          if (c0 > 0) {                                           // (the columns before are out of the way)
            __syncwarp();
            if (lane == 0) mbar_arrive1(quarters);
            if (!pm_wait(quarters, n_quarter & 1, lim, abort_flag)) return false;
            ++n_quarter;
          }
#pragma unroll 1
          for (int c = 0; c < cols; c += 32) {
            float o[32], o1[32];
            if (my > 0) tmem_ld32(tO + c0 + c, o);
            if (second) tmem_ld32(tO + 128 + c0 + c, o1);
            if (valid) {
#pragma unroll
              for (int x = 0; x < 32; ++x) {
                const float y = my > 0 && l != 0.f ? o[x] * w0 : 0.f;
                o[x] = second && l1 != 0.f ? fmaf(o1[x], w1, y) : y;
              }
              unsigned char* to = stage + ((warp & 3) * r_cap + lane) * r_bytes + c * 4;
#pragma unroll
              for (int x = 0; x < 8; ++x) *reinterpret_cast<float4*>(to + x * 16) = make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive1(quarters);
          if (!pm_wait(quarters, n_quarter & 1, lim, abort_flag)) return false;
          ++n_quarter;
          if (r < n_rows) {
            float4 v0 = make_float4(0.f, 0.f, 0.f, 0.f), v1 = v0;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float4* from = reinterpret_cast<const float4*>(stage + (x * r_cap + r) * r_bytes + piece * 32);
              const float4 a0 = from[0], a1 = from[1];
              v0.x += a0.x; v0.y += a0.y; v0.z += a0.z; v0.w += a0.w;
              v1.x += a1.x; v1.y += a1.y; v1.z += a1.z; v1.w += a1.w;
            }
            if (whole) {
              *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + o_row * D + c0 + piece * 8) =
                  make_uint4(pack_bf16(v0.x, v0.y), pack_bf16(v0.z, v0.w), pack_bf16(v1.x, v1.y), pack_bf16(v1.z, v1.w));
            } else {
              float4* dst = reinterpret_cast<float4*>(a.w.part_o + (part_row + (r - row)) * D + c0 + piece * 8);
              dst[0] = v0;
              dst[1] = v1;
            }
          }
        }
        if (valid && (warp & 3) == 0) {
          if (!whole) a.w.part_ml[part_row] = make_float2(M, sum);
          else if (a.lse) a.lse[out_row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
        }
      } else if (live) {
        // A thread holds a row; written as it is, every store would touch 32 rows.  64 bytes of each row go through shared memory: four
        // lanes a row, whole sectors (8192-token prompt: 691 -> 653 us).
        unsigned char* stage = smem + SM::kStage + (warp - 4) * 32 * SM::kStageRow;
        unsigned char* mine = stage + lane * SM::kStageRow;
        const int r_first = (warp & 3) * 32 + (lane >> 2), piece = lane & 3;    // rows r_first + 8 k of the row tile
        unsigned char* dst[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = r_first + 8 * k, ri = r / G;
          const bool there = r < ppos * G && i0 + ri < sg.n;
          if (!there) dst[k] = nullptr;
          else if (whole)
            dst[k] = reinterpret_cast<unsigned char*>(a.out) + ((long long)(sg.row0 + i0 + ri) * a.pl.Hq + sg.h * G + (r - ri * G)) * (D * 2) + piece * 16;
          else
            dst[k] = reinterpret_cast<unsigned char*>(a.w.part_o) + (part_row + (r - row)) * (D * 4) + piece * 16;
        }
        auto send = [&](int at) {                                 // 64 bytes of every row, `at` bytes into it
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4 v = *reinterpret_cast<const uint4*>(stage + ((lane >> 2) + 8 * k) * SM::kStageRow + piece * 16);
            if (dst[k]) *reinterpret_cast<uint4*>(dst[k] + at) = v;
          }
          __syncwarp();
        };
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          if (my > 0) {
            tmem_ld32(tO + c, o);
#pragma unroll
            for (int x = 0; x < 32; ++x) o[x] = l == 0.f ? 0.f : o[x] * w0;
          } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) o[x] = 0.f;
          }
          if (second) {
            float o1[32];
            tmem_ld32(tO + 128 + c, o1);
            if (l1 != 0.f)
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] = fmaf(o1[x], w1, o[x]);
          }
          if (whole) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
              *reinterpret_cast<uint4*>(mine + x * 16) = make_uint4(pack_bf16(o[8 * x], o[8 * x + 1]), pack_bf16(o[8 * x + 2], o[8 * x + 3]),
                                                                    pack_bf16(o[8 * x + 4], o[8 * x + 5]), pack_bf16(o[8 * x + 6], o[8 * x + 7]));
            send(c * 2);
          } else {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
              for (int x = 0; x < 4; ++x)
                *reinterpret_cast<float4*>(mine + x * 16) = make_float4(o[16 * y + 4 * x], o[16 * y + 4 * x + 1], o[16 * y + 4 * x + 2], o[16 * y + 4 * x + 3]);
              send(c * 4 + y * 64);
            }
          }
        }
        if (valid && !whole) a.w.part_ml[part_row] = make_float2(M, sum);
        if (valid && whole && a.lse) a.lse[out_row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (my > 0) mbar_arrive1(&o_free[slot]);
        if (second) mbar_arrive1(&o_free[1]);
      }
      return true;
    });
    if (!ok) *abort_flag = 1;
  }

  // ---------------------------------------------------------------- end: tensor memory back -----------------------------
  __syncwarp();
  __syncthreads();
  if (*abort_flag && tid == 0) atomicExch(a.pl.status, kStatusTimeout);
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_free(tmem, kPmTmemCols);
  }
}

template <int D, bool MODS, bool FEW, bool LONG>
cudaError_t mma_variant(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) {
  auto kern = paged_mma_kernel<D, MODS, FEW, LONG>;
  constexpr int bytes = PmSmem<D, FEW>::kBytes;
  static unsigned long long allowed = 0;
  cudaError_t e = allow_smem_once(kern, bytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(a.w.n_cta), dim3(kPmThreads), bytes, s, 0, true, a, *reinterpret_cast<const CUtensorMap*>(maps.k),
                   *reinterpret_cast<const CUtensorMap*>(maps.v), *reinterpret_cast<const CUtensorMap*>(maps.q));
}
template <int D, bool MODS, bool FEW>
cudaError_t mma_launch(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) {
  return a.w.drain ? mma_variant<D, MODS, FEW, true>(a, maps, s) : mma_variant<D, MODS, FEW, false>(a, maps, s);
}
template <int D>
cudaError_t mma_d(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) {
  const bool mods = a.softcap > 0.f || a.slopes, few = a.w.ppos * a.pl.G <= 32;
  if (few) return mods ? mma_launch<D, true, true>(a, maps, s) : mma_launch<D, false, true>(a, maps, s);
  return mods ? mma_launch<D, true, false>(a, maps, s) : mma_launch<D, false, false>(a, maps, s);
}

}  // namespace

size_t paged_mma_drain_bytes(const PagedWork& w, const PagedBatch& pb, const PagedLayout& pl) {
  return pb.max_len > kPmDrain * kPmKeys ? (size_t)w.n_cta * 2 * 128 * (pl.d + 1) * 4 : 0;
}

int paged_mma_positions(const PagedBatch& pb, const PagedLayout& pl) { return (pb.max_new * pl.G <= 32 ? 32 : 128) / pl.G; }

void paged_plan_mma(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count) {
  w->ppos = paged_mma_positions(pb, pl);
  const bool few = w->ppos * pl.G <= 32;
  w->upos = (few ? 1 : 2) * w->ppos;
  w->log_tk = 7;
  static_assert(kPmKeys == 1 << 7, "keys per tile");
  const long long tiles = (pb.max_len + kPmKeys - 1) / kPmKeys, units = (long long)pb.batch * pl.Hkv * paged_units(*w, pb.max_new);
  // Whole units where none is long (one head's 500 tokens in us: whole 11.3, cut 15.3; 64 sequences of them 35.1 and 49.7), and up to
  // 12 tiles where there is about a CTA for each (16 sequences of 1000 tokens 16.8 and 23.9, of 1500 21.8 and 29.3, a prompt of 1000 28.1 and 38.5; with
  // fewer units, 8 of 1000 tokens: 14.7 and 14.1; with more, ragged prompts of up to 1000 x 16: 165 and 146).
  w->by_unit = tiles <= 4 || (tiles <= 12 && units <= sm_count && 4 * units >= sm_count);
  w->min_tiles = w->by_unit ? 1 : 2;
  w->extra = few ? 1 : 2;                // (a prompt of 8192 tokens with 0, 1, 2, 3, 4: 656, 616, 577, 582, 588 us; single tokens: no difference within 2 %)
  const long long most = w->by_unit ? units : (units * tiles + w->min_tiles - 1) / w->min_tiles;
  w->n_cta = (int)(most < sm_count ? most : sm_count);
  w->narrow = paged_narrow(*w, pb, pl);
  w->rows = (pb.max_new < w->upos ? pb.max_new : w->upos) * pl.G;
}

cudaError_t launch_paged_mma(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) {
  return a.pl.d == 128 ? mma_d<128>(a, maps, s) : mma_d<64>(a, maps, s);
}

}  // namespace spla
