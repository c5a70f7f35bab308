// Rotary positions, and the append to a paged cache that rotates on the way.
//
// A block takes TB tokens.  Its threads first form the tokens' sines and cosines, one (token, pair) each, in shared memory; then
// every thread keeps one piece of a head (VEC pairs: 16 bytes of either half, or 32 bytes of neighbouring pairs) and walks the
// (token, head) rows of the block, queries, keys and values as one list.  The angle is exact: the frequency is a 64-bit fraction of a
// turn, position x frequency wraps at whole turns in integer arithmetic, and only the remainder (its top 32 bits) becomes a float.
// Bound by memory: every channel is read and written once, 6 flops per pair.
#include "paged.h"

namespace spla {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTable = 512;          // (token, pair) entries of a block's table, at most
constexpr int kRopeTokens = 8;           // tokens of a block, at most

struct RopeLaunch {
  RopeGroup g[3];
  const int* positions;                  // null: the position in the sequence (pages only)
  int batch, tokens, tb;                 // tb: tokens per block
  int heads, rows_per_y;                 // (token, head) rows of a block are shared by the grid's y blocks
  int pieces;                            // pieces of a head = threads side by side
  int transpose;
  int paged;
  PagedBatch pb;
  PagedLayout pl;
  void *k_pages, *v_pages;
};

template <int VEC>
__device__ __forceinline__ void load_piece(const float* p, float (&x)[VEC]) {
  if constexpr (VEC == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = p[i];
  }
}
template <int VEC>
__device__ __forceinline__ void load_piece(const __nv_bfloat16* p, float (&x)[VEC]) {
  if constexpr (VEC == 8) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = __bfloat162float(p[i]);
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

// VEC pairs per piece; both element types may occur in one launch with VEC = 1 only.
template <typename T, int VEC>
__global__ void __launch_bounds__(kRopeThreads)
    rope_kernel(const RopeLaunch r, const __grid_constant__ RopeTable rt) {
  __shared__ __align__(16) float2 table[kRopeTable];      // [token][VEC pairs of piece 0, 1, ... two by two]
  __shared__ long long tok_row[kRopeTokens];              // page row of the token's position for head 0; -1: nothing to store
  __shared__ int tok_pos[kRopeTokens];
  __shared__ int tok_at[kRopeTokens];                     // sequence of the token; -1: none
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, pairs = rt.rot / 2;
  const long long tok0 = (long long)blockIdx.x * r.tb;
  const long long n_tok = (long long)r.batch * r.tokens;
  const int nt = (int)min((long long)r.tb, n_tok - tok0);
  if (tid < nt) {
    const long long tok = tok0 + tid;
    int pos = 0, at = 0;
    long long row = 0;
    if (r.paged) {
      int lo = 0, hi = r.pb.batch;                        // the last b with cu[b] <= tok
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(r.pb.cu + mid) <= tok) lo = mid; else hi = mid;
      }
      const PagedSeq s = paged_seq(r.pb, r.pl.status, lo);
      at = lo;
      row = -1;
      if (s.n > 0 && tok >= s.row0 && tok < s.row0 + s.n) {
        pos = s.L - s.n + (int)(tok - s.row0);
        const long long first = paged_row(r.pb, r.pl, lo, 0, pos >> r.pl.log_p);
        if (first >= 0) row = first + (pos & (r.pl.P - 1));
      } else {
        at = -1;
      }
    }
    if (r.positions && at >= 0) pos = __ldg(r.positions + tok);
    tok_pos[tid] = pos;
    tok_row[tid] = row;
    tok_at[tid] = at;
  }
  __syncthreads();
  // entry of (token, pair): the pairs of a piece lie two by two, the pieces side by side, so that a warp's loads are contiguous
  if (pairs > 0) {
    const int n_pieces = pairs / VEC;
    for (int x = tid; x < nt * pairs; x += kRopeThreads) {
      const int t = x / pairs, i = x - t * pairs;
      const float2 cs = turn_of(rt.freq[i], tok_pos[t], rt.amplitude, r.transpose != 0);
      const int piece = i / VEC, j = i % VEC;
      const int e = VEC == 1 ? i : ((j >> 1) * n_pieces + piece) * 2 + (j & 1);
      table[t * pairs + e] = cs;
    }
  }
  __syncthreads();
  const int by = kRopeThreads / r.pieces, piece = tid % r.pieces, ty = tid / r.pieces;
  if (ty >= by) return;
  const int rot_pieces = pairs / VEC;
  const bool turns_here = piece < rot_pieces;
  // channels of the piece: a and b of its pairs, or two runs of VEC channels to copy
  int ca, cb;
  if (!turns_here) { ca = rt.rot + (piece - rot_pieces) * 2 * VEC; cb = ca + VEC; }
  else if (rt.interleaved) { ca = piece * 2 * VEC; cb = ca + VEC; }
  else { ca = piece * VEC; cb = ca + pairs; }
  const int rows = nt * r.heads, end = min(rows, ((int)blockIdx.y + 1) * r.rows_per_y);

  struct Place {
    const T* in;
    T* out;
    int t;
    bool rot;
  };
  auto place = [&](int row) {
    Place pl;
    const int t = row / r.heads;
    int h = row - t * r.heads;
    pl.t = t;
    int gi = 0;
    if (h >= r.g[0].n_heads) { h -= r.g[0].n_heads; gi = 1; }
    if (gi == 1 && h >= r.g[1].n_heads) { h -= r.g[1].n_heads; gi = 2; }
    const RopeGroup& g = r.g[gi];
    const long long tok = tok0 + t;
    const long long b = r.batch == 1 ? 0 : tok / r.tokens, i = tok - b * r.tokens;
    pl.in = reinterpret_cast<const T*>(g.in) + b * g.in_batch + i * g.in_token + h * g.in_head;
    pl.rot = turns_here && g.rotate;
    if (g.out) pl.out = tok_at[t] < 0 ? nullptr : reinterpret_cast<T*>(g.out) + b * g.out_batch + i * g.out_token + h * g.out_head;
    else if (tok_row[t] < 0) pl.out = nullptr;
    else pl.out = reinterpret_cast<T*>(gi == 1 ? r.k_pages : r.v_pages) + (tok_row[t] + h * r.pl.head_stride) * rt.dim;
    return pl;
  };
  auto finish = [&](const Place& pl, float (&a)[VEC], float (&b)[VEC]) {
    if (pl.rot) {
      if constexpr (VEC == 1) {
        const float2 cs = table[pl.t * pairs + piece];
        const float x = a[0], y = b[0];
        a[0] = x * cs.x - y * cs.y;
        b[0] = y * cs.x + x * cs.y;
      } else {
        const float4* tab = reinterpret_cast<const float4*>(table + pl.t * pairs) + piece;
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
          const float4 cs = tab[j * rot_pieces];
          if (rt.interleaved) {                            // a then b hold neighbouring pairs (x, y), (x, y), ...
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
    }
    store_piece<VEC>(pl.out + ca, a);
    store_piece<VEC>(pl.out + cb, b);
  };
  for (int row = blockIdx.y * r.rows_per_y + ty; row < end; row += 2 * by) {       // two rows at a time, loads first
    const bool second = row + by < end;
    const Place p0 = place(row), p1 = place(second ? row + by : row);
    float a0[VEC], b0[VEC], a1[VEC], b1[VEC];
    if (p0.out) { load_piece<VEC>(p0.in + ca, a0); load_piece<VEC>(p0.in + cb, b0); }
    const bool do1 = second && p1.out;
    if (do1) { load_piece<VEC>(p1.in + ca, a1); load_piece<VEC>(p1.in + cb, b1); }
    if (p0.out) finish(p0, a0, b0);
    if (do1) finish(p1, a1, b1);
  }
}

bool wide(const RopeGroup& g, int e) {
  const long long v = 16 / e;
  auto ok = [&](long long s) { return s % v == 0; };
  return (uintptr_t)g.in % 16 == 0 && ok(g.in_batch) && ok(g.in_token) && ok(g.in_head) &&
         (!g.out || ((uintptr_t)g.out % 16 == 0 && ok(g.out_batch) && ok(g.out_token) && ok(g.out_head)));
}

template <typename T, int VEC>
cudaError_t rope_launch(RopeLaunch r, const RopeTable& rt, int sm_count, cudaStream_t s) {
  r.pieces = rt.dim / (2 * VEC);
  const int pairs = rt.rot / 2;
  // tokens per block: a full table's worth, so that every thread forms one or two sines; fewer where that would leave SMs idle
  const long long n_tok = (long long)r.batch * r.tokens;
  int tb = pairs > 0 ? kRopeThreads / pairs : kRopeTokens;
  if (tb < 1) tb = 1;
  if (tb > kRopeTokens) tb = kRopeTokens;
  while (tb > 1 && (n_tok + tb - 1) / tb < 2LL * sm_count) tb /= 2;
  r.tb = tb;
  const long long blocks = (n_tok + tb - 1) / tb;
  const int by = kRopeThreads / r.pieces, rows = tb * r.heads;
  int ys = 1;
  if (blocks < 2LL * sm_count) {
    ys = (rows + by - 1) / by;
    const long long most = (4LL * sm_count + blocks - 1) / blocks;
    if (ys > most) ys = (int)most;
  }
  r.rows_per_y = (rows + ys - 1) / ys;
  return launch_ex(rope_kernel<T, VEC>, dim3((unsigned)blocks, (rows + r.rows_per_y - 1) / r.rows_per_y), dim3(kRopeThreads), 0, s, 0, true, r, rt);
}

}  // namespace

cudaError_t launch_rope(const RopeTable& rt, const int* positions, int batch, int tokens, const RopeGroup* groups, int n_groups,
                        const PagedBatch* pb, const PagedLayout* pl, void* k_pages, void* v_pages, int transpose, cudaStream_t s) {
  RopeLaunch r = {};
  r.positions = positions;
  r.batch = batch;
  r.tokens = tokens;
  r.transpose = transpose;
  if (pb) { r.paged = 1; r.pb = *pb; r.pl = *pl; r.k_pages = k_pages; r.v_pages = v_pages; }
  const int sm = device_sm_count();
  // One launch per element type (queries may have another than the cache), wide pieces where every address allows them
  cudaError_t e = cudaSuccess;
  for (int f32 = 0; f32 < 2 && e == cudaSuccess; ++f32) {
    const int size = f32 ? 4 : 2, vec = 16 / size;
    bool fast = rt.dim % (2 * vec) == 0 && rt.rot % (2 * vec) == 0;
    r.heads = 0;
    for (int i = 0; i < 3; ++i) {
      r.g[i] = i < n_groups ? groups[i] : RopeGroup{};
      if (i >= n_groups || groups[i].elem_f32 != f32) r.g[i].n_heads = 0;
      if (r.g[i].n_heads > 0) fast = fast && wide(r.g[i], size);
      r.heads += r.g[i].n_heads;
    }
    if (r.heads == 0) continue;
    if (f32) e = fast ? rope_launch<float, 4>(r, rt, sm, s) : rope_launch<float, 1>(r, rt, sm, s);
    else e = fast ? rope_launch<__nv_bfloat16, 8>(r, rt, sm, s) : rope_launch<__nv_bfloat16, 1>(r, rt, sm, s);
  }
  return e;
}

}  // namespace spla
