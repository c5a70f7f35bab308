// Rotary positions, and the append to a paged cache that rotates on the way.
//
// A block takes TB tokens.  Its threads first form the tokens' sines and cosines, one (token, pair) each, in shared memory; then
// every thread keeps one piece of a head (VEC pairs: 16 bytes of either half, or 32 bytes of neighbouring pairs) and walks the
// (token, head) rows of the block, queries, keys and values as one list.  The angle is exact: the frequency is a 64-bit fraction of a
// turn, position x frequency wraps at whole turns in integer arithmetic, and only the remainder (its top 32 bits) becomes a float.
// Bound by memory: every channel is read and written once, 6 flops per pair (32768 tokens of 32 + 8 heads of 128: 111 us in a graph,
// 6.0 TB/s, 0.92 of a copy's rate, one channel at a time, VEC = 1, 369; small calls by a launch: 8 tokens 2.2 us).  The first rows' loads are
// issued before the tokens' places and the sines are known (175 -> 115 us with bases once per token, no 64-bit divisions; 115 -> 110 with
// the loads first).
#include "paged.h"

namespace spla {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTable = 2048;         // (token, pair) entries of a block's table, at most
constexpr int kRopeTokens = 32;          // tokens of a block, at most
constexpr int kRopePerWarp = kRopeTokens / (kRopeThreads / 32);

struct RopeLaunch {
  RopeGroup g[3];
  const int* positions;                  // null: the position in the sequence (pages only)
  int batch, tokens, tb;                 // tb: tokens per block
  int heads, rows_per_y;                 // (token, head) rows of a block are shared by the grid's y blocks
  int pieces;                            // pieces of a head = threads side by side
  unsigned head_magic;                   // ceil(2^32 / heads): row / heads = high word of row x magic (rows x heads is far below 2^32)
  int transpose;
  int paged;
  PagedBatch pb;
  PagedLayout pl;
  void *k_pages, *v_pages;
};

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

// VEC pairs per piece; both element types may occur in one launch with VEC = 1 only.
template <typename T, int VEC>
__global__ void __launch_bounds__(kRopeThreads, sizeof(T) == 4 ? 5 : 4)
    rope_kernel(const __grid_constant__ RopeLaunch r, const __grid_constant__ RopeTable rt) {
  constexpr int kWords = VEC == 1 ? 1 : 4;
  __shared__ __align__(16) float2 table[kRopeTable];      // [token][VEC pairs of piece 0, 1, ... two by two]
  __shared__ T* out_at[kRopeTokens][3];                   // pages: first head of the token, by group (null: nothing is written)
  __shared__ int tok_pos[kRopeTokens];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, pairs = rt.rot / 2;
  const int tok0 = blockIdx.x * r.tb, nt = min(r.tb, r.tokens - tok0), batch = blockIdx.z;
  const int by = kRopeThreads / r.pieces, piece = tid % r.pieces, ty = tid / r.pieces;
  const int rot_pieces = pairs / VEC;
  const bool turns_here = piece < rot_pieces;
  // channels of the piece: a and b of its pairs, or two runs of VEC channels to copy
  int ca, cb;
  if (!turns_here) { ca = rt.rot + (piece - rot_pieces) * 2 * VEC; cb = ca + VEC; }
  else if (rt.interleaved) { ca = piece * 2 * VEC; cb = ca + VEC; }
  else { ca = piece * VEC; cb = ca + pairs; }
  const int end = ty < by ? min(nt * r.heads, ((int)blockIdx.y + 1) * r.rows_per_y) : 0;
  const int n0 = r.g[0].n_heads, n01 = n0 + r.g[1].n_heads;

  struct Place {
    int t, h, gi;                                         // token of the block, head of the group, group
  };
  auto place = [&](int row) {
    Place pl;
    pl.t = r.heads == 1 ? row : (int)__umulhi((unsigned)row, r.head_magic);
    const int h = row - pl.t * r.heads;
    pl.gi = (h >= n0) + (h >= n01);
    pl.h = h - (pl.gi == 0 ? 0 : pl.gi == 1 ? n0 : n01);
    return pl;
  };
  // two rows at a time; the first are on their way before the tokens' places and the sines are known
  int row = blockIdx.y * r.rows_per_y + ty;
  Place p0, p1;
  uint32_t x0[kWords], y0[kWords], x1[kWords], y1[kWords];
  auto load = [&](const Place& pl, uint32_t (&x)[kWords], uint32_t (&y)[kWords]) {
    const RopeGroup& g = pl.gi == 0 ? r.g[0] : pl.gi == 1 ? r.g[1] : r.g[2];
    const T* in = reinterpret_cast<const T*>(g.in) + batch * g.in_batch + (long long)(tok0 + pl.t) * g.in_token + pl.h * g.in_head;
    load_raw(in + ca, x);
    load_raw(in + cb, y);
  };
  auto fetch = [&]() {
    if (row < end) p0 = place(row);
    if (row + by < end) p1 = place(row + by);
    if (row < end) load(p0, x0, y0);
    if (row + by < end) load(p1, x1, y1);
  };
  fetch();
  if (r.paged) {
    if (blockIdx.x == 0 && blockIdx.y == 0)               // every sequence's numbers are looked at once, those without tokens too
      for (int b = tid; b < r.pb.batch; b += kRopeThreads) paged_seq(r.pb, r.pl.status, b);
    // a warp's tokens: warp, warp + 8, ...; lane k ends up with the k-th
    const int tok = tok0 + warp + lane * (kRopeThreads / 32);
    const int at = paged_owner<kRopePerWarp>(r.pb, tok0 + warp, kRopeThreads / 32, lane);
    if (lane < kRopePerWarp && tok < tok0 + nt) {
      PagedSeq s{0, 0, 0, false};
      if (at >= 0) s = paged_seq(r.pb, r.pl.status, at);
      const bool there = s.n > 0 && tok >= s.row0 && tok < s.row0 + s.n;
      int pos = 0;
      long long page_row = -1;                            // of the token's position for head 0
      if (there) {
        pos = s.L - s.n + (tok - s.row0);
        page_row = paged_row(r.pb, r.pl, at, 0, pos >> r.pl.log_p);
        if (page_row >= 0) page_row += pos & (r.pl.P - 1);
      }
      const int t = tok - tok0;
      out_at[t][0] = r.g[0].out && there ? reinterpret_cast<T*>(r.g[0].out) + (long long)tok * r.g[0].out_token : nullptr;
      out_at[t][1] = page_row >= 0 ? reinterpret_cast<T*>(r.k_pages) + page_row * rt.dim : nullptr;
      out_at[t][2] = page_row >= 0 ? reinterpret_cast<T*>(r.v_pages) + page_row * rt.dim : nullptr;
      tok_pos[t] = r.positions && there ? __ldg(r.positions + tok) : pos;
    }
    __syncthreads();
  }
  // entry of (token, pair): the pairs of a piece lie two by two, the pieces side by side, so that a warp's loads are contiguous
  if (pairs > 0) {
    const unsigned long long* freq = rt.freq;
    asm("" : "+l"(freq));                                 // (an ordinary load: a constant one takes a turn per thread)
    for (int x = tid; x < nt * pairs; x += kRopeThreads) {
      const int t = x / pairs, i = x - t * pairs;
      const int pos = r.paged ? tok_pos[t] : __ldg(r.positions + (long long)batch * r.tokens + tok0 + t);
      const float2 cs = turn_of(freq[i], pos, rt.amplitude, r.transpose != 0);
      const int pc = i / VEC, j = i % VEC;
      const int e = VEC == 1 ? i : ((j >> 1) * rot_pieces + pc) * 2 + (j & 1);
      table[t * pairs + e] = cs;
    }
  }
  __syncthreads();
  auto finish = [&](const Place& pl, const uint32_t (&x)[kWords], const uint32_t (&y)[kWords]) {
    float a[VEC], b[VEC];
    unpack<T, VEC>(x, a);
    unpack<T, VEC>(y, b);
    const RopeGroup& g = pl.gi == 0 ? r.g[0] : pl.gi == 1 ? r.g[1] : r.g[2];
    T* out;
    if (r.paged) {
      out = out_at[pl.t][pl.gi];
      if (!out) return;
      out += pl.h * (g.out ? g.out_head : r.pl.head_stride * rt.dim);
    } else {
      out = reinterpret_cast<T*>(g.out) + batch * g.out_batch + (long long)(tok0 + pl.t) * g.out_token + pl.h * g.out_head;
    }
    if (turns_here && g.rotate) {
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
    store_piece<VEC>(out + ca, a);
    store_piece<VEC>(out + cb, b);
  };
  for (; row < end; row += 2 * by, fetch()) {
    finish(p0, x0, y0);
    if (row + by < end) finish(p1, x1, y1);
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
  r.head_magic = (unsigned)(((1ull << 32) + r.heads - 1) / r.heads);
  const int pairs = rt.rot / 2;
  // tokens per block: a sine for every thread (eight tokens at most: with 16 of 24 small fp32 heads 42 us in place of 37), and four rows for every
  // thread where heads are few, so that what comes before the first row pays (6 heads of 128, 80000 tokens: 22 tokens 69 us, 4 tokens 111);
  // fewer where that would leave SMs idle
  const int by = kRopeThreads / r.pieces;
  int tb = pairs > 0 && kRopeThreads / pairs < 8 ? kRopeThreads / pairs : 8;
  if (tb < (4 * by + r.heads - 1) / r.heads) tb = (4 * by + r.heads - 1) / r.heads;
  if (tb > kRopeTokens) tb = kRopeTokens;
  if (tb * pairs > kRopeTable) tb = kRopeTable / pairs;
  if (tb < 1) tb = 1;
  while (tb > 1 && (long long)tb * r.heads * r.heads >= (1ll << 32)) tb /= 2;   // (see head_magic)
  auto blocks = [&](int x) { return (long long)((r.tokens + x - 1) / x) * r.batch; };
  while (tb > 1 && blocks(tb) < 2LL * sm_count) tb /= 2;
  if (tb > r.tokens) tb = r.tokens;
  r.tb = tb;
  const int rows = tb * r.heads;
  int ys = 1;
  if (blocks(tb) < 2LL * sm_count) {
    ys = (rows + by - 1) / by;
    const long long most = (4LL * sm_count + blocks(tb) - 1) / blocks(tb);
    if (ys > most) ys = (int)most;
  }
  r.rows_per_y = (rows + ys - 1) / ys;
  // (the grid's third dimension ends at 65535)
  const int batch = r.batch;
  cudaError_t e = cudaSuccess;
  for (int b = 0; b < batch && e == cudaSuccess; b += 65535) {
    RopeLaunch part = r;
    part.batch = batch - b < 65535 ? batch - b : 65535;
    if (r.positions) part.positions = r.positions + (long long)b * r.tokens;
    for (RopeGroup& g : part.g) {
      if (g.in) g.in = (const char*)g.in + b * g.in_batch * (long long)sizeof(T);
      if (g.out) g.out = (char*)g.out + b * g.out_batch * (long long)sizeof(T);
    }
    e = launch_ex(rope_kernel<T, VEC>, dim3((r.tokens + tb - 1) / tb, (rows + r.rows_per_y - 1) / r.rows_per_y, part.batch), dim3(kRopeThreads), 0, s, 0,
                  true, part, rt);
  }
  return e;
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
    // a batch whose tokens follow one another, or of one token each, is one list of tokens
    r.batch = batch;
    r.tokens = tokens;
    bool list = batch > 1 && (long long)batch * tokens < (1ll << 31);
    for (int i = 0; i < 3 && list; ++i)
      if (r.g[i].n_heads > 0) list = tokens == 1 || (r.g[i].in_batch == tokens * r.g[i].in_token && r.g[i].out_batch == tokens * r.g[i].out_token);
    if (list) {
      for (RopeGroup& g : r.g)
        if (tokens == 1) { g.in_token = g.in_batch; g.out_token = g.out_batch; }
      r.tokens = batch * tokens;
      r.batch = 1;
    }
    if (f32) e = fast ? rope_launch<float, 4>(r, rt, sm, s) : rope_launch<float, 1>(r, rt, sm, s);
    else e = fast ? rope_launch<__nv_bfloat16, 8>(r, rt, sm, s) : rope_launch<__nv_bfloat16, 1>(r, rt, sm, s);
  }
  return e;
}

}  // namespace spla
