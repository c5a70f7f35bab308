// Norms of queries and keys, head by head, with the rotation to their positions in the same pass; and the gradients of that.
//
//   n_c = x_c r w_c,  r = (mean_c x_c^2 + eps)^(-1/2),  y = R n          (R: the rotation, an orthogonal map times its amplitude)
//   u = R^T dy,  dw_c = sum over tokens and heads of u_c x_c r,  dx_c = r (w_c u_c - x_c r^2 mean_c(w_c u_c x_c))
//
// A CTA takes a few tokens: their sines into shared memory, then all rows (one head of one token) of the queries, then of the keys.  A row
// belongs to a power of two of neighbouring lanes, 16 bytes of either half (or of neighbouring pairs) each, so that its sums are a few
// shuffles, its channels stay in registers, and every element is read and written once.  r is formed again in the backward
// pass: x has to be read anyway.
// Gradients of the weights: a thread adds its channels up in registers over all rows that its CTA takes (the grid is one wave then), the CTA's
// rows meet in shared memory, and a second kernel adds the CTAs' sums in their order: no atomics, the same bits every time.
// All arithmetic in fp32, one rounding at the end.
//
// What bounds it: memory, read and write once.  Forward, 4 x 8192 tokens of 32 + 8 heads of 128 in bf16: 125 us in a graph (102 at a copy's rate), in fp32 217 (204), 3 x 2731
// of 16 + 4 heads of 64 in fp32 22 (12.8).  Gradients 197 us (153), in fp32 357 (307), the smaller one 39 (19): two reads for a write, 128 registers, two CTAs an SM.  Few tokens: launches (eight tokens 8 us, what a graph of one
// small kernel takes here; the second kernel of the gradients takes 7 by itself when it is cold).  Steps: groups known to the compiler, four CTAs an SM and one row a thread 158 -> 135 us (two rows under way and three
// CTAs 156; five and six CTAs were slower too), the next row asked for as soon as this one's values are out of its registers 134 -> 125 (three CTAs 131, fp32 20.5 -> 24.6); gradients with tiles as large as the table allows and two values at a time 281 -> 197.
#include <type_traits>

#include "rope_device.cuh"

namespace spla {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormTable = 2048;         // (token, pair) entries of a CTA's table, at most
constexpr int kNormMaxDim = 2 * kRopeMaxPairs;

struct NormLaunch {
  NormGroup g[2];                        // queries, keys
  const int* positions;
  int tokens, tb, tiles_per_batch;       // of a batch entry; per tile
  int tiles;                             // of all batch entries
  int rows_per_y;
  unsigned head_magic[2];                // as in RopeLaunch
  float eps, per_channel;
  int width;                             // lanes of a row
  float* part;                           // [CTAs][2][dim]: sums for the weights' gradients
};

template <typename T, class ROW, bool BWD>
__global__ void __launch_bounds__(kNormThreads, BWD ? 2 : 4)
    norm_kernel(const __grid_constant__ NormLaunch r, const __grid_constant__ RopeTable rt) {
  constexpr int CH = ROW::CH, WORDS = ROW::WORDS;
  constexpr bool loose = sizeof(ROW) == sizeof(LooseRow<T, CH>);
  __shared__ __align__(16) float2 table[kNormTable];               // and the rows' sums for the weights, at the end
  __shared__ __align__(16) float w_s[2][kNormMaxDim];
  __shared__ float rows_s[loose ? kNormThreads / 32 : 1][loose ? kNormMaxDim : 1];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, pairs = rt.rot / 2, dim = rt.dim;
  const int width = r.width, by = kNormThreads / width, ty = tid / width;
  const ROW row(rt, tid % width);
  float* own_row = rows_s[loose ? tid / 32 : 0];
  const int n0 = r.g[0].n_heads, n_all = n0 + r.g[1].n_heads;
  auto weights = [&]() {
    for (int x = tid; x < 2 * dim; x += kNormThreads) {
      const int g = x >= dim;
      if (r.g[g].n_heads > 0) w_s[g][x - g * dim] = __ldg(r.g[g].weight + x - g * dim);
    }
  };
  constexpr std::integral_constant<int, 0> queries{};
  constexpr std::integral_constant<int, 1> keys{};
  // The rows of a tile that are this block's: of the queries, then of the keys.
  int b, tok0, nt, from[2], to[2];
  auto start = [&](int tile) {
    b = tile / r.tiles_per_batch;
    tok0 = (tile - b * r.tiles_per_batch) * r.tb;
    nt = min(r.tb, r.tokens - tok0);
    const int first = (int)blockIdx.y * r.rows_per_y, last = first + r.rows_per_y, rows0 = nt * n0, rows1 = nt * (n_all - n0);
    from[0] = min(first, rows0);
    to[0] = min(last, rows0);
    from[1] = max(first, rows0) - rows0;
    to[1] = min(last, rows0 + rows1) - rows0;
  };
  auto sines = [&]() {
    const int* pos = r.positions + (long long)b * r.tokens + tok0;
    fill_turns<ROW>(rt, table, nt, tid, kNormThreads, BWD, [&](int t) { return __ldg(pos + t); });
  };
  // A thread's row on its way: row x0 + ty of the group.  (Which group is known to the compiler: its strides are constants then.)
  int tk;                                                          // its token of the tile, -1: none
  T* out;
  uint32_t raw[WORDS] = {}, raw_g[BWD ? WORDS : 1] = {};
  auto fetch = [&](auto group_c, int x0) {
    constexpr int GI = decltype(group_c)::value;
    const NormGroup& g = r.g[GI];
    const int x = x0 + ty;
    tk = -1;
    if (x >= to[GI] || !row.here) return;
    const int t = g.n_heads == 1 ? x : (int)__umulhi((unsigned)x, r.head_magic[GI]), h = x - t * g.n_heads;
    const long long tok = tok0 + t;
    tk = t;
    out = reinterpret_cast<T*>(g.out) + b * g.out_batch + tok * g.out_token + h * g.out_head;
    row.load(reinterpret_cast<const T*>(g.x) + b * g.x_batch + tok * g.x_token + h * g.x_head, raw);
    if constexpr (BWD) row.load(reinterpret_cast<const T*>(g.dy) + b * g.dy_batch + tok * g.dy_token + h * g.dy_head, raw_g);
  };
  auto fetch_first = [&]() {
    if (from[0] < to[0]) fetch(queries, from[0]); else fetch(keys, from[1]);
  };
  // (what comes behind the rows from x0 on)
  auto fetch_next = [&](auto group_c, int x0) {
    constexpr int GI = decltype(group_c)::value;
    if (GI == 0 && x0 + by >= to[0]) fetch(keys, from[1]); else fetch(group_c, x0 + by);
  };
  float acc[2][BWD ? CH : 1];

  if constexpr (!BWD) {
    // one tile; the first rows are on their way before the sines are known
    start(blockIdx.x);
    fetch_first();
    weights();
    sines();
    __syncthreads();
    auto group = [&](auto group_c) {
      constexpr int GI = decltype(group_c)::value;
#pragma unroll 1
      for (int x0 = from[GI]; x0 < to[GI]; x0 += by) {             // (whole warps: a row's lanes meet in shuffles)
        float x[CH], w[CH];
        const int t = tk;
        T* const to_row = out;
        row.values(raw, x);                                     // (of no row: whatever, and not stored)
        fetch_next(group_c, x0);                                   // (its registers are free)
        if (!loose && !row.here)                                   // (lanes beside a row's: nothing to its sum)
#pragma unroll
          for (int i = 0; i < CH; ++i) x[i] = 0.f;
        const float rms = row_rms(x, width, r.per_channel, r.eps);
        row.weights(w_s[GI], w);
        row_scale(x, rms, w);
        row.turn(x, table + max(t, 0) * pairs, own_row);
        if (t >= 0) row.store(to_row, x);
      }
    };
    group(queries);
    group(keys);
  } else {
    // tiles one after the other; queries' rows, then keys', whose weights' gradients are sums of their own; the next row is on its way
    weights();
#pragma unroll
    for (int i = 0; i < CH; ++i) acc[0][i] = acc[1][i] = 0.f;
    auto group = [&](auto group_c) {
      constexpr int GI = decltype(group_c)::value;
      float (&sum)[CH] = acc[GI];
#pragma unroll 1
      for (int x0 = from[GI]; x0 < to[GI]; x0 += by) {
        float x[CH], u[CH];
        const int t = tk;
        T* const to_row = out;
        row.values(raw, x);
        row.values(raw_g, u);
        fetch_next(group_c, x0);                                   // (its registers are free)
        if (t < 0) {
#pragma unroll
          for (int i = 0; i < CH; ++i) x[i] = u[i] = 0.f;
        }
        float rms = row_rms(x, width, r.per_channel, r.eps);
        if (t < 0) rms = 0.f;                                      // (of no row: nothing to the sums, infinite or not)
        row.turn(u, table + max(t, 0) * pairs, own_row);
        float w[CH];
        row.weights(w_s[GI], w);
        float2 dot2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < CH; i += 2) {
          const float2 u2 = make_float2(u[i], u[i + 1]), x2 = make_float2(x[i], x[i + 1]);
          const float2 s2 = __ffma2_rn(__fmul2_rn(u2, x2), make_float2(rms, rms), make_float2(sum[i], sum[i + 1]));
          sum[i] = s2.x;
          sum[i + 1] = s2.y;
          const float2 g2 = __fmul2_rn(u2, make_float2(w[i], w[i + 1]));
          dot2 = __ffma2_rn(g2, x2, dot2);
          u[i] = g2.x;
          u[i + 1] = g2.y;
        }
        const float dot = -(row_sum(dot2.x + dot2.y, width) * r.per_channel * rms * rms);
#pragma unroll
        for (int i = 0; i < CH; i += 2) {
          const float2 y = __fmul2_rn(__ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(dot, dot), make_float2(u[i], u[i + 1])), make_float2(rms, rms));
          u[i] = y.x;
          u[i + 1] = y.y;
        }
        if (t >= 0) row.store(to_row, u);
      }
    };
    for (int tile = blockIdx.x; tile < r.tiles; tile += gridDim.x) {
      start(tile);
      fetch_first();
      if (tile != (int)blockIdx.x) __syncthreads();                // (the table before is used up)
      sines();
      __syncthreads();
      group(queries);
      group(keys);
    }
    float* red = reinterpret_cast<float*>(table);                  // [by][dim]
    for (int g = 0; g < 2; ++g) {
      if (r.g[g].n_heads == 0) continue;
      __syncthreads();
      if (row.here)
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (row.channel(i) < dim) red[ty * dim + row.channel(i)] = g ? acc[1][i] : acc[0][i];
      __syncthreads();
      for (int c = tid; c < dim; c += kNormThreads) {
        float s = 0.f;
        for (int y = 0; y < by; ++y) s += red[y * dim + c];
        r.part[((long long)(blockIdx.y * gridDim.x + blockIdx.x) * 2 + g) * dim + c] = s;
      }
    }
  }
}

// Sums of `n` CTAs for 32 channels of one weight, in their order: every warp a run of the CTAs, then the runs.
constexpr int kNormSumWarps = 32, kNormSumRows = 10;        // (two CTAs an SM: all rows of a warp under way at once)
__global__ void __launch_bounds__(32 * kNormSumWarps) norm_sum_kernel(const float* part, int n, int dim, float* dq, float* dk) {
  __shared__ float runs[kNormSumWarps][32];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, g = blockIdx.y;
  float* out = g ? dk : dq;
  if (!out) return;
  const int from = (int)((long long)n * warp / kNormSumWarps), to = (int)((long long)n * (warp + 1) / kNormSumWarps);
  float s = 0.f;
  if (c < dim)
    for (int x0 = from; x0 < to; x0 += kNormSumRows) {
      float v[kNormSumRows];
#pragma unroll
      for (int x = 0; x < kNormSumRows; ++x) v[x] = x0 + x < to ? part[((long long)(x0 + x) * 2 + g) * dim + c] : 0.f;
#pragma unroll
      for (int x = 0; x < kNormSumRows; ++x) s += v[x];
    }
  runs[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < dim) {
    float all = 0.f;
#pragma unroll
    for (int x = 0; x < kNormSumWarps; ++x) all += runs[x][lane];
    out[c] = all;
  }
}

struct NormPlan {
  int tb, tiles_per_batch, ys, rows_per_y, grid_x;
  long long tiles;
};
// (sizes alone decide it, not addresses: the workspace is asked for without them)
NormPlan plan_norm(const RopeTable& rt, int batch, int tokens, int heads, bool backward, int sm_count) {
  NormPlan p;
  const int pairs = rt.rot / 2;
  constexpr int by = 32;
  auto per_batch = [&](int x) { return (int)(((long long)tokens + x - 1) / x); };
  auto tiles = [&](int x) { return (long long)per_batch(x) * batch; };
  int tb, most = kNormTable / pairs < 64 ? kNormTable / pairs : 64;
  if (backward) {
    // two CTAs an SM, each as many tiles as the next, as large as the table of sines allows: what comes before a tile's first row is rarely paid
    const long long wave = 2LL * sm_count, rounds = (tiles(most) + wave - 1) / wave;
    for (tb = most; tb > 1 && tiles(tb - 1) <= rounds * wave;) --tb;
  } else {
    // two sines for every thread, rows for every thread where heads are few (as in rope.cu; with one sine 139 us for 4 x 8192, with four 137, in place of 135)
    tb = kNormThreads / pairs < 8 ? kNormThreads / pairs : 8;
    if (tb < (4 * by + heads - 1) / heads) tb = (4 * by + heads - 1) / heads;
    tb *= 2;
    if (tb > most) tb = most;
  }
  if (tb < 1) tb = 1;
  while (tb > 1 && (long long)tb * heads * heads >= (1ll << 32)) tb /= 2;      // (see head_magic)
  while (tb > 1 && tiles(tb) < (backward ? 1LL : 2LL) * sm_count) tb /= 2;
  if (tb > tokens) tb = tokens;
  p.tb = tb;
  p.tiles_per_batch = per_batch(tb);
  p.tiles = tiles(tb);
  const int rows = tb * heads;
  p.ys = 1;
  if (p.tiles < 2LL * sm_count) {
    p.ys = (rows + by - 1) / by;
    const long long many = ((backward ? 2LL : 4LL) * sm_count + p.tiles - 1) / p.tiles;
    if (p.ys > many) p.ys = (int)many;
  }
  p.rows_per_y = (rows + p.ys - 1) / p.ys;
  p.ys = (rows + p.rows_per_y - 1) / p.rows_per_y;
  const long long wave = (2LL * sm_count + p.ys - 1) / p.ys;
  p.grid_x = (int)(backward && wave < p.tiles ? wave : p.tiles);
  return p;
}

template <typename T, class ROW, bool BWD>
cudaError_t norm_launch(const NormLaunch& r, const NormPlan& p, const RopeTable& rt, cudaStream_t s) {
  return launch_ex(norm_kernel<T, ROW, BWD>, dim3(p.grid_x, p.ys), dim3(kNormThreads), 0, s, 0, true, r, rt);
}
template <typename T, bool BWD>
cudaError_t norm_rows(NormLaunch& r, const NormPlan& p, const RopeTable& rt, bool wide, cudaStream_t s) {
  constexpr int vec = 16 / (int)sizeof(T);
  if (!wide) {
    r.width = 32;
    return norm_launch<T, LooseRow<T, kNormMaxDim / 32>, BWD>(r, p, rt, s);
  }
  for (r.width = 1; r.width < rt.dim / (2 * vec);) r.width *= 2;
  return norm_launch<T, WideRow<T, vec>, BWD>(r, p, rt, s);
}

}  // namespace

size_t norm_part_bytes(const RopeTable& rt, int batch, int tokens, int heads, int sm_count) {
  const NormPlan p = plan_norm(rt, batch, tokens, heads, true, sm_count);
  return (size_t)p.grid_x * p.ys * 2 * rt.dim * 4;
}

cudaError_t launch_norm(const RopeTable& rt, const int* positions, int batch, int tokens, const NormGroup& q, const NormGroup& k, float eps, int f32,
                        bool backward, float* dq_weight, float* dk_weight, void* workspace, cudaStream_t s) {
  const int sm = device_sm_count(), heads = q.n_heads + k.n_heads;
  const NormPlan p = plan_norm(rt, batch, tokens, heads, backward, sm);
  if (p.tiles >= (1ll << 31)) return cudaErrorInvalidValue;
  NormLaunch r = {};
  r.g[0] = q;
  r.g[1] = k;
  r.positions = positions;
  r.tokens = tokens;
  r.tb = p.tb;
  r.tiles_per_batch = p.tiles_per_batch;
  r.tiles = (int)p.tiles;
  r.rows_per_y = p.rows_per_y;
  r.eps = eps;
  r.per_channel = 1.f / (float)rt.dim;
  r.part = reinterpret_cast<float*>(workspace);
  const int e = f32 ? 4 : 2;
  bool wide = wide_rotation(rt, e);
  for (int i = 0; i < 2; ++i) {
    const NormGroup& g = r.g[i];
    if (g.n_heads == 0) continue;
    r.head_magic[i] = (unsigned)(((1ull << 32) + g.n_heads - 1) / g.n_heads);
    wide = wide && wide_strides(g.x, e, g.x_batch, g.x_token, g.x_head) && wide_strides(g.out, e, g.out_batch, g.out_token, g.out_head) &&
           (!backward || wide_strides(g.dy, e, g.dy_batch, g.dy_token, g.dy_head));
  }
  cudaError_t err;
  if (backward) err = f32 ? norm_rows<float, true>(r, p, rt, wide, s) : norm_rows<__nv_bfloat16, true>(r, p, rt, wide, s);
  else err = f32 ? norm_rows<float, false>(r, p, rt, wide, s) : norm_rows<__nv_bfloat16, false>(r, p, rt, wide, s);
  if (err == cudaSuccess && backward)
    err = launch_ex(norm_sum_kernel, dim3((rt.dim + 31) / 32, 2), dim3(32 * kNormSumWarps), 0, s, 0, true, (const float*)workspace, p.grid_x * p.ys, rt.dim,
                    dq_weight, k.n_heads ? dk_weight : (float*)nullptr);
  return err;
}

}  // namespace spla
