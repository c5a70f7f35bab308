// The paged cache and the rotary positions: parameters of their kernels and the division of the attention's work, shared by
// the translation units (not part of the public ABI).
#pragma once

#include "spla_internal.h"

namespace spla {

constexpr int kRopeMaxPairs = 128;
constexpr int kRopeMaxHeads = 4096;     // of one tensor

// Frequencies as 64-bit fractions of a turn: position x frequency wraps at whole turns by itself, so that what is left for
// the sine and cosine is the exact angle modulo a turn, at any position.
struct RopeTable {
  unsigned long long freq[kRopeMaxPairs];
  int dim, rot, interleaved;            // head channels, rotated ones (0: copy only), pairing
  float amplitude;
};

// A group of heads that one launch rotates or copies.
struct RopeGroup {
  const void* in;
  void* out;                            // null: the group goes to pages
  int n_heads, rotate;
  long long in_batch, in_token, in_head, out_batch, out_token, out_head;   // elements
  int elem_f32;                         // element type: 1 = fp32, 0 = bf16
};

// One tensor of launch_norm: x -> out, and in the backward pass the gradient dy of y.  Strides in elements.
struct NormGroup {
  const void *x, *dy;
  void* out;
  const float* weight;                  // [dim]
  int n_heads;                          // 0: not there
  long long x_batch, x_token, x_head, dy_batch, dy_token, dy_head, out_batch, out_token, out_head;
};

// The new tokens of launch_store; strides in elements between tokens.
struct StoreGroups {
  const void *q, *k, *v;
  void* q_out;
  long long q_stride, k_stride, v_stride, q_out_stride;
  int q_f32, kv_f32;
  const float *q_weight, *k_weight;     // null: not normed
  float eps;
  const int* positions;
};

// What the pages hold.  8-bit pages: e4m3 values, and for every 16 rows (tokens of a head) the scale 2^(byte - 127).
enum { kPagesBf16 = 0, kPagesF32 = 1, kPagesE4m3 = 2 };
struct PagedPages {
  void *k, *v;
  unsigned char *k_scales, *v_scales;
  int type;
};

struct PagedBatch {
  const int* cu;                        // [batch + 1] rows of the new tokens
  const int* lens;                      // [batch] cached tokens, the new ones included
  const int* table;                     // [batch][table_stride]
  int batch, total_new, max_new, max_len, table_stride;
  int first;                            // sequences of the call before these (earlier launches')
};

struct PagedLayout {
  int Hq, Hkv, G, d, P, log_p, n_pages;
  long long page_stride, head_stride;   // rows
  int* status;
};

// One sequence's new tokens: first row, count, cached tokens; n = 0 where there is nothing to do or the numbers do not fit together.
// Besides, a sequence is served only if no earlier prefix sum inside [0, total_new] is above its first row, so that a row has one owner
// whatever the prefix sums are.  That takes a look at them all only where some sequence's own numbers do not fit (prefix sums that
// do not ascend belong to one whose do not).
struct PagedSeq {
  int row0, n, L;
  bool fits;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& pb, int* status, int b) {
  const int r0 = __ldg(pb.cu + b), r1 = __ldg(pb.cu + b + 1), L = __ldg(pb.lens + b);
  PagedSeq s{r0, r1 - r0, L, false};
  s.fits = r0 >= 0 && r1 >= r0 && r1 <= pb.total_new && r1 - r0 <= pb.max_new && L >= r1 - r0 && L <= pb.max_len;
  if (!s.fits) {
    atomicExch(status, kStatusBounds);
    s.n = 0;
  }
  return s;
}

// A prefix sum for comparisons of order: those outside [0, total_new] take no part.
__device__ __forceinline__ int paged_order(const PagedBatch& pb, int c) { return c >= 0 && c <= pb.total_new ? c : -1; }
// The largest of a warp's values up to each lane, and `before`.
__device__ __forceinline__ int paged_max_scan(int v, int before, int lane) {
  v = max(v, before);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) v = max(v, __shfl_up_sync(0xffffffffu, v, o));   // (lanes below o get their own)
  return v;
}
// The sequence that may own a row of the new tokens, -1: none.  Lane k < K of a warp asks for row + k step.  (Its own numbers are the caller's to check.)
// The last one that starts at or before the row, as long as the prefix sums ascend.  Where they do not, the one before the first prefix sum above
// the row, if no earlier one is above its own.
template <int K>
__device__ __forceinline__ int paged_owner(const PagedBatch& pb, int row, int step, int lane) {
  int at = -1;
  bool ascend = true;
  for (int b0 = 0; b0 < pb.batch; b0 += 32) {
    const int b = b0 + lane, c = b < pb.batch ? __ldg(pb.cu + b) : 0x7fffffff;
    if (b > 0 && b < pb.batch) ascend &= c >= __ldg(pb.cu + b - 1);
    bool more = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const unsigned in = __ballot_sync(0xffffffffu, c <= row + k * step);
      if (lane == k) at += __popc(in);
      more |= in == 0xffffffffu;
    }
    if (!more) break;
  }
  if (__all_sync(0xffffffffu, ascend)) return at;
  at = -1;
  int top = -1;
  bool open = true;
#pragma unroll 1
  for (int b0 = 0; b0 < pb.batch; b0 += 32) {
    const int c = b0 + lane < pb.batch ? paged_order(pb, __ldg(pb.cu + b0 + lane)) : 0x7fffffff, upto = paged_max_scan(c, top, lane);
    const unsigned sound = __ballot_sync(0xffffffffu, c == upto);
    top = __shfl_sync(0xffffffffu, upto, 31);
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
      const unsigned in = __ballot_sync(0xffffffffu, c <= row + k * step);
      if (lane != k || !open) continue;
      open = in == 0xffffffffu;
      const int last = open ? 31 : __ffs(~in) - 2;
      if (last >= 0) at = (sound >> last) & 1 ? b0 + last : -1;
    }
  }
  return at;
}

// ---- division of the attention's work --------------------------------------------------------------------------------
// A unit is one KV head's query rows of neighbouring new tokens (`upos` positions x G heads; a sequence of at most `ppos` new tokens
// is one unit of one row tile).  It walks the key tiles of TK tokens that any of its positions sees.  The tiles of all units, in the
// order sequence, head, unit, are dealt out in equal contiguous shares to the CTAs of one resident wave: every CTA carries the
// same number of tiles however ragged the lengths are.  A unit that a share's border cuts leaves partial results (maximum, sum,
// unnormalised output per row) that a second kernel joins, in the order of the shares: no atomics, the same bits every time.
// Short caches are dealt out by whole units instead, which needs no second kernel.
constexpr int kPagedMaxBatch = 384;    // sequences per launch (the host cuts larger batches)

struct PagedWork {
  int ppos, upos, log_tk;               // TK = 2^log_tk
  int by_unit;                          // dealt out by units instead of tiles
  int n_cta, min_tiles;
  int narrow;                           // all tiles together are below 2^31, by the host's bounds
  int extra;                            // what starting and ending a unit costs, in tiles: counted before its first tile when the work is dealt out
  int rows;                             // rows that a partial result holds
  float* part_o;                        // [2 n_cta][rows][d]
  float2* part_ml;                      // [2 n_cta][rows]  maximum (base 2), sum
  float* drain;                         // [2 n_cta][128 (d + 1)]  what the tensor cores' sums so far have been taken into (null: no walk is that long)
  int4* cuts;                           // [n_cta] of the unit whose first cut is the start of a share: rows (0: no such unit), parts, first row of its tokens, KV head
};

struct PagedAttend {
  PagedBatch pb;
  PagedLayout pl;
  PagedWork w;
  const void* q;
  long long q_stride;
  void* out;
  float* lse;
  float sm_scale, softcap;
  int window;
  const float* slopes;
  const int* first_key;
  const int* prefix;
  int wait_limit, dbg_tx_extra;         // as in Params
  int sinks;                            // so many first tokens are visible besides the window
  int from_new, to_new;                 // sequences of so many new tokens are this launch's (0, 0: all of them); the others are passed over
  const unsigned char *k_scales, *v_scales;   // of 8-bit pages
  const signed char* q_exp;             // exponents of the queries' rows, where paged_split.cu has scaled them
};

// Sequence table of a CTA, in shared memory.
struct PagedSeqs {
  long long pre[kPagedMaxBatch + 1];    // tiles (units) before a sequence, all heads (2^31 in one head: 40000 new tokens behind 2^24 cached ones, G = 16)
  int row0[kPagedMaxBatch], n[kPagedMaxBatch], L[kPagedMaxBatch], prefix[kPagedMaxBatch];
};

__host__ __device__ __forceinline__ int paged_units(const PagedWork& w, int n) { return n <= w.ppos ? (n > 0) : (n + w.upos - 1) / w.upos; }

// New tokens of a sequence as far as they are this launch's.
__device__ __forceinline__ int paged_mine(const PagedAttend& a, int n) { return a.to_new > 0 && (n < a.from_new || n > a.to_new) ? 0 : n; }

// Key tiles [t0, t1) that unit u of a sequence may walk.  With a window and sinks the tiles are numbered without those between the sinks' and the
// window's: the first `ns` are tiles 0 .. ns - 1, the others lie `skip` tiles further on.  Never empty: a position sees itself.  From e0 on they count when the work is
// dealt out: the tiles before are behind the start of its first token's document, where there is nothing to walk as long as
// documents follow one another (what is walked goes by every token's own start).
struct PagedSpan {
  int t0, t1, e0;
  int ns, skip;
};
__device__ __forceinline__ PagedSpan paged_span(const PagedAttend& a, int row0, int n, int L, int prefix, int u) {
  const PagedWork& w = a.w;
  const int p0 = L - n + u * w.upos, p1 = L - n + min(n, (u + 1) * w.upos) - 1;
  const int lo = a.window > 0 ? max(0, p0 - a.window + 1) : 0, hi = min(L, max(p1 + 1, prefix));
  PagedSpan s{lo >> w.log_tk, (hi + (1 << w.log_tk) - 1) >> w.log_tk, 0, 0, 0};
  if (a.sinks > 0 && s.t0 > 0) {
    s.ns = min(s.t0, (min(a.sinks, hi) + (1 << w.log_tk) - 1) >> w.log_tk);
    s.skip = s.t0 - s.ns;
    s.t0 = 0;
    s.t1 -= s.skip;
  }
  s.e0 = s.t0;
  if (a.first_key && !w.by_unit) s.e0 = min(max(s.t0, __ldg(a.first_key + row0 + u * w.upos) >> w.log_tk), s.t1 - 1);
  return s;
}
// What a unit counts for: its tiles and `extra` (one, where whole units are dealt out).
__device__ __forceinline__ int paged_unit_tiles(const PagedAttend& a, int row0, int n, int L, int prefix, int u) {
  if (a.w.by_unit) return 1;
  const PagedSpan s = paged_span(a, row0, n, L, prefix, u);
  return s.t1 - s.e0 + a.w.extra;
}

// What one sequence counts for, per head.  Whole warps: sequences of many units are counted by the warp together.
__device__ __forceinline__ long long paged_seq_tiles(const PagedAttend& a, int row0, int n, int L, int prefix, int lane) {
  const int nu = paged_units(a.w, n);
  int few = 0;
  if (nu <= 4)
    for (int u = 0; u < nu; ++u) few += paged_unit_tiles(a, row0, n, L, prefix, u);
  long long sum = few;
  for (unsigned many = __ballot_sync(0xffffffffu, nu > 4); many; many &= many - 1) {
    const int who = __ffs(many) - 1;
    const int n_ = __shfl_sync(0xffffffffu, n, who), L_ = __shfl_sync(0xffffffffu, L, who), p_ = __shfl_sync(0xffffffffu, prefix, who),
              nu_ = __shfl_sync(0xffffffffu, nu, who), r_ = __shfl_sync(0xffffffffu, row0, who);
    long long part = 0;
    for (int u = lane; u < nu_; u += 32) part += paged_unit_tiles(a, r_, n_, L_, p_, u);
    if (a.w.narrow) {
      part = __reduce_add_sync(0xffffffffu, (int)part);
    } else {
#pragma unroll 1
      for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    }
    if (lane == who) sum = part;
  }
  return sum;
}
template <typename N>
__device__ __forceinline__ N paged_scan(N v, int lane) {                   // inclusive, over a warp
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// Fills the table; all threads of the CTA (whole warps), ends with a barrier.  Returns the total.
__device__ __forceinline__ long long paged_fill_seqs(const PagedAttend& a, PagedSeqs& t, int tid, int threads) {
  const int batch = a.pb.batch, lane = tid & 31;
  if (batch <= 32 && a.pb.first == 0) { // every warp for itself, all of them the same values: one barrier, which is the caller's anyway
    int row0 = 0, n = 0, L = 0, pre = 0;
    bool fits = true;
    if (lane < batch) {
      pre = a.prefix ? __ldg(a.prefix + lane) : 0;
      const PagedSeq s = paged_seq(a.pb, a.pl.status, lane);
      row0 = s.row0; n = paged_mine(a, s.n); L = s.L; fits = s.fits;
    }
    if (!__all_sync(0xffffffffu, fits)) {
      const int c = paged_order(a.pb, row0);
      if (c != paged_max_scan(lane < batch ? c : -1, -1, lane)) n = 0;
    }
    if (lane < batch) {
      t.row0[lane] = row0; t.n[lane] = n; t.L[lane] = L; t.prefix[lane] = pre;
    }
    const long long per_head = paged_seq_tiles(a, row0, n, L, pre, lane);
    const long long v = a.w.narrow ? paged_scan((int)per_head * a.pl.Hkv, lane) : paged_scan(per_head * a.pl.Hkv, lane);
    if (lane < batch) t.pre[lane + 1] = v;
    if (lane == 0) t.pre[0] = 0;
    __syncthreads();
    return t.pre[batch];
  }
  bool fits = true;
  for (int b = tid - a.pb.first; b < 0; b += threads) {              // (sequences of earlier launches: their prefix sums)
    const int c = __ldg(a.pb.cu + b);
    fits &= c >= 0 && c <= __ldg(a.pb.cu + b + 1) && c <= a.pb.total_new;
  }
  for (int b0 = tid - lane; b0 < batch; b0 += threads) {
    const int b = b0 + lane;
    int row0 = 0, n = 0, L = 0, pre = 0;
    if (b < batch) {
      pre = a.prefix ? __ldg(a.prefix + b) : 0;
      const PagedSeq s = paged_seq(a.pb, a.pl.status, b);
      row0 = s.row0; n = paged_mine(a, s.n); L = s.L; fits &= s.fits;
      t.row0[b] = row0; t.n[b] = n; t.L[b] = L; t.prefix[b] = pre;
    }
    const long long per_head = paged_seq_tiles(a, row0, n, L, pre, lane);
    if (b < batch) t.pre[b + 1] = per_head * a.pl.Hkv;
  }
  const bool look = __syncthreads_or(!fits);
  if (tid < 32) {
    int top = -1;
    if (look) {
      for (int b = tid - a.pb.first; b < 0; b += 32) top = max(top, paged_order(a.pb, __ldg(a.pb.cu + b)));
      top = __reduce_max_sync(0xffffffffu, top);
    }
    long long carry = 0;
    for (int b0 = 0; b0 < batch; b0 += 32) {
      const int b = b0 + tid;
      if (look) {
        const int c = b < batch ? paged_order(a.pb, t.row0[b]) : -1, upto = paged_max_scan(c, top, tid);
        top = __shfl_sync(0xffffffffu, upto, 31);
        if (b < batch && c != upto) { t.n[b] = 0; t.pre[b + 1] = 0; }
      }
      const long long v = paged_scan(b < batch ? t.pre[b + 1] : 0ll, tid) + carry;
      carry = __shfl_sync(0xffffffffu, v, 31);
      if (b < batch) t.pre[b + 1] = v;
    }
    if (tid == 0) t.pre[0] = 0;
  }
  __syncthreads();
  return t.pre[batch];
}

// Tiles (units) per CTA.
__device__ __forceinline__ long long paged_share(const PagedWork& w, long long total) {
  const long long up = total + w.n_cta - 1;
  const long long per = w.narrow ? (long long)((unsigned)up / (unsigned)w.n_cta) : up / w.n_cta;
  return per < w.min_tiles ? w.min_tiles : per;
}

// A CTA's walk over its share: one segment (a run of key tiles of one unit) after the other.  Every role keeps its own copy.
struct PagedWalk {
  long long left;                       // tiles (units) still to walk
  int b, h, u, off, units;              // off: tiles of the unit that earlier segments (other CTAs) have; units of a head
  int row0, n, L, prefix;
  // the current segment
  int t0, t1;                           // key tiles
  int ns, skip;                         // see PagedSpan
  bool head, tail;                      // it starts / ends the unit

  __device__ __forceinline__ void load(const PagedWork& w, const PagedSeqs& t) { row0 = t.row0[b]; n = t.n[b]; L = t.L[b]; prefix = t.prefix[b]; units = paged_units(w, n); }
  // Goes to tile `at` of all; false if there is none.  Whole warps.
  __device__ __forceinline__ bool seek(const PagedAttend& a, const PagedSeqs& t, long long at, long long count) {
    const long long total = t.pre[a.pb.batch];
    left = min(count, total - at);
    if (left <= 0) { left = 0; return false; }
    const int lane = threadIdx.x & 31;
    b = -1;                             // the last b with pre[b] <= at
    for (int b0 = 0;; b0 += 32) {
      const unsigned in = __ballot_sync(0xffffffffu, b0 + lane < a.pb.batch && t.pre[b0 + lane] <= at);
      b += __popc(in);
      if (in != 0xffffffffu) break;
    }
    load(a.w, t);
    const long long rem = at - t.pre[b], all = t.pre[b + 1] - t.pre[b];
    const long long per_head = a.w.narrow ? (long long)((unsigned)all / (unsigned)a.pl.Hkv) : all / a.pl.Hkv;
    h = a.w.narrow ? (int)((unsigned)rem / (unsigned)per_head) : (int)(rem / per_head);
    long long in_head = rem - h * per_head;
    if (units == 1) {
      u = 0;
      off = (int)in_head;
      return true;
    }
    const int nu = units;
    for (u = 0;; u += 32) {             // 32 units at a time
      const int c = u + lane < nu ? paged_unit_tiles(a, row0, n, L, prefix, u + lane) : 0;
      int upto = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      const unsigned past = __ballot_sync(0xffffffffu, upto > in_head);
      if (past || u + 32 >= nu) {
        const int who = past ? __ffs(past) - 1 : 0;
        off = (int)in_head - __shfl_sync(0xffffffffu, upto - c, who);
        u += who;
        break;
      }
      in_head -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return true;
  }
  __device__ __forceinline__ bool next(const PagedAttend& a, const PagedSeqs& t) {
    do {
      if (left <= 0) return false;
      if (u >= units) {                              // the unit before was its head's last
        u = 0;
        if (++h == a.pl.Hkv) {
          h = 0;
          do ++b; while (b < a.pb.batch - 1 && t.pre[b + 1] == t.pre[b]);
          load(a.w, t);
        }
      }
      const PagedSpan s = paged_span(a, row0, n, L, prefix, u);
      ns = s.ns; skip = s.skip;
      if (a.w.by_unit) {
        t0 = s.t0; t1 = s.t1; head = tail = true;
        left -= 1;
      } else {                                       // the share holds off .. upto of the unit's extra and tiles
        const int upto = (int)min((long long)(s.t1 - s.e0 + a.w.extra), off + left);
        left -= upto - off;
        head = off <= a.w.extra;
        t0 = head ? s.t0 : s.e0 + off - a.w.extra;
        t1 = upto <= a.w.extra ? t0 : s.e0 + upto - a.w.extra;
        tail = t1 == s.t1;
      }
      off = 0;
      u_cur = u++;
    } while (t0 == t1);                              // (a share's last bit, too short for a tile: the next share starts the unit)
    return true;
  }
  // What the join has to know of the cut at the start of share `cut`, `mine` = seek(), before next().
  __device__ __forceinline__ int4 cut_here(const PagedAttend& a, bool mine, long long share) const {
    // (a border between two tiles of the unit, and its first: the share before holds the unit's head)
    if (!mine || off <= a.w.extra || off - a.w.extra > share) return make_int4(0, 0, 0, 0);
    const int tiles = paged_unit_tiles(a, row0, n, L, prefix, u), i0 = u * a.w.upos;
    const int parts = 1 + (int)((tiles - off + share - 1) / share);   // the share before (its second slot), then this one and those after (their first)
    return make_int4(min(n - i0, n <= a.w.ppos ? a.w.ppos : a.w.upos) * a.pl.G, parts, row0 + i0, h);
  }
  int u_cur;                            // unit of the current segment
  __device__ __forceinline__ int first_pos(const PagedWork& w) const { return u_cur * w.upos; }   // index of its first new token in the sequence
  __device__ __forceinline__ int n_pos(const PagedWork& w) const { return min(n - u_cur * w.upos, n <= w.ppos ? w.ppos : w.upos); }
};

// Keys [lo, hi) that the new token with index i of a sequence sees, besides those before both `hi` and a.sinks.
struct PagedSees {
  int lo, hi;
};
__device__ __forceinline__ PagedSees paged_sees(const PagedAttend& a, int row0, int n, int L, int prefix, int i) {
  const int pos = L - n + i;
  PagedSees s;
  s.lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  if (a.first_key) s.lo = max(s.lo, __ldg(a.first_key + row0 + i));
  s.hi = min(L, max(pos + 1, prefix));
  return s;
}

// First row of page `index` of a sequence's head; -1 where the page number is outside the pool.
__device__ __forceinline__ long long paged_row(const PagedBatch& pb, const PagedLayout& pl, int b, int h, int index) {
  const int page = __ldg(pb.table + (long long)b * pb.table_stride + index);
  if ((unsigned)page >= (unsigned)pl.n_pages) {
    atomicExch(pl.status, kStatusBounds);
    return -1;
  }
  return page * pl.page_stride + h * pl.head_stride;
}

// Whether all tiles (and extras) that a launch may have are below 2^31.
inline bool paged_narrow(const PagedWork& w, const PagedBatch& pb, const PagedLayout& pl) {
  const double units = (double)pl.Hkv * ((double)pb.total_new / w.upos + pb.batch), tiles = pb.max_len / (double)(1 << w.log_tk) + 1 + w.extra;
  return units * tiles + w.n_cta < 2147483647.0;
}

// Scales of 8-bit pages: exponents between -40 and 40 (others are read as the nearest).
constexpr int kExpMin = -40, kExpMax = 40;
__device__ __forceinline__ int paged_exponent(const unsigned char* p) { return min(max((int)__ldg(p) - 127, kExpMin), kExpMax); }
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((127 + e) << 23); }
__device__ __forceinline__ float paged_scale(const unsigned char* scales, long long row) { return power_of_two(paged_exponent(scales + (row >> 4))); }

struct PagedMaps {                      // TMA tensor maps (CUtensorMap), opaque to the host code
  alignas(64) unsigned char k[128];
  alignas(64) unsigned char v[128];
  alignas(64) unsigned char q[128];
};

// rope.cu: rotates / copies up to three groups; with `pages` the groups with out == null go to k_pages (group 1) and v_pages (group 2)
cudaError_t launch_rope(const RopeTable& rt, const int* positions, int batch, int tokens, const RopeGroup* groups, int n_groups,
                        const PagedBatch* pb, const PagedLayout* pl, void* k_pages, void* v_pages, int transpose, cudaStream_t s);
// store.cu: appends to pages of any type with norms, and to 8-bit pages; reads cached tokens back
cudaError_t launch_store(const RopeTable* rope, const StoreGroups& g, const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, cudaStream_t s);
cudaError_t launch_read(const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, void* k_out, void* v_out, int out_f32, cudaStream_t s);
// norm.cu
size_t norm_part_bytes(const RopeTable& rt, int batch, int tokens, int heads, int sm_count);
cudaError_t launch_norm(const RopeTable& rt, const int* positions, int batch, int tokens, const NormGroup& q, const NormGroup& k, float eps, int f32,
                        bool backward, float* dq_weight, float* dk_weight, void* workspace, cudaStream_t s);
// paged_attend.cu: fp32 kernels for every type, and the join of cut units
void paged_plan_general(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count);
cudaError_t launch_paged_general(const PagedAttend& a, const PagedPages& pages, int q_bf16, cudaStream_t s);
cudaError_t launch_paged_join(const PagedAttend& a, int out_bf16, cudaStream_t s);
// paged_few.cu: 8-bit pages, at most 16 rows per sequence and KV head
int paged_few_positions(const PagedLayout& pl);   // new tokens of a sequence that it takes, at most
void paged_plan_few(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count);
cudaError_t launch_paged_few(const PagedAttend& a, const PagedMaps& maps, int f32, cudaStream_t s);   // f32: queries and outputs
// paged_split.cu: bf16 queries as two parts of 8 bits, [token][head][part][d], and the exponents of the rows' scales [token][head]
size_t paged_split_bytes(const PagedLayout& pl, int total_new, size_t* exps);
cudaError_t launch_paged_split(const PagedLayout& pl, const void* q, long long q_stride, int total_new, unsigned char* parts, signed char* exps, cudaStream_t s);
// ... or the cached tokens as bf16 pages of kWidePage tokens: their layout, and the places of the values and of the page table behind the keys
constexpr int kWidePage = 128;
struct PagedWide {
  PagedLayout pl;
  int cols, slots, first;               // tiles of a sequence, pages it has (fewer with a window), those of the sinks
  size_t v_at, table_at, bytes;
  bool fits;                            // (rows that a TMA coordinate can name)
};
PagedWide paged_wide(const PagedLayout& pl, const PagedBatch& pb, int window, int sinks);
cudaError_t launch_paged_widen(const PagedBatch& pb, const PagedLayout& pl, const PagedPages& pages, const PagedWide& w, int window, void* to, cudaStream_t s);
// paged_mma.cu: bf16 on tcgen05
size_t paged_mma_drain_bytes(const PagedWork& w, const PagedBatch& pb, const PagedLayout& pl);
int paged_mma_positions(const PagedBatch& pb, const PagedLayout& pl);   // new tokens of a row tile: the query boxes' size
void paged_plan_mma(PagedWork* w, const PagedBatch& pb, const PagedLayout& pl, int sm_count);
cudaError_t launch_paged_mma(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s);
cudaError_t launch_paged_mma_bytes64(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s);    // ... and over 8-bit pages
cudaError_t launch_paged_mma_bytes128(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s);

}  // namespace spla
