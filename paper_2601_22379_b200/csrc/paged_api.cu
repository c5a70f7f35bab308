// C ABI of the rotary positions and of the paged cache: argument validation, plans and launches.  Host code only.
#include <math.h>
#include <new>
#include <string.h>

#include <cuda.h>

#include "../../include/spla.h"
#include "paged.h"

using namespace spla;

struct spla_rope {
  RopeTable t;
};

struct spla_paged {
  spla_paged_config_t cfg;
  PagedLayout pl;
  void *k_pages, *v_pages;
  PagedMaps maps;
  bool tensor;                          // bf16 cache and queries, tensor maps made: the tensor-core kernel serves it
  int sm_count;
  int wait_limit, dbg_tx_extra;
};

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
static bool is_dtype(int t) { return t == SPLA_F32 || t == SPLA_BF16; }
static int dtype_bytes(int t) { return t == SPLA_BF16 ? 2 : 4; }

// ---- rotary positions ------------------------------------------------------------------------------------------------
extern "C" int spla_rope_create(const spla_rope_config_t* c, spla_rope_t** rope_out) {
  if (!c || !rope_out) return SPLA_ERR_INVALID_ARG;
  const double base0 = c->base == 0.0 ? 10000.0 : c->base, factor = c->factor == 0.0 ? 1.0 : c->factor;
  const double amplitude = c->amplitude == 0.0 ? 1.0 : c->amplitude;
  const int rot = c->rot_dim == 0 ? c->head_dim : c->rot_dim;
  if (c->head_dim < 1 || rot < 2 || rot % 2 || rot > c->head_dim) return SPLA_ERR_INVALID_ARG;
  if (c->interleaved != 0 && c->interleaved != 1) return SPLA_ERR_INVALID_ARG;
  if (c->scaling < SPLA_ROPE_PLAIN || c->scaling > SPLA_ROPE_RAMP) return SPLA_ERR_INVALID_ARG;
  if (!(base0 > 0.0) || !isfinite(base0) || !(factor >= 1.0) || !isfinite(factor) || !isfinite(amplitude)) return SPLA_ERR_INVALID_ARG;
  if (c->scaling == SPLA_ROPE_BASE && rot == 2) return SPLA_ERR_INVALID_ARG;      // (the exponent R / (R - 2))
  if (c->scaling == SPLA_ROPE_RAMP &&
      (!(c->original_len > 0.0) || !isfinite(c->original_len) || !(c->ramp_high > c->ramp_low) || !isfinite(c->ramp_high) || !isfinite(c->ramp_low)))
    return SPLA_ERR_INVALID_ARG;
  if (c->head_dim % 8 || c->head_dim > 2 * kRopeMaxPairs) return SPLA_ERR_UNSUPPORTED;
  const double two_pi = 6.283185307179586476925286766559;
  const double base = c->scaling == SPLA_ROPE_BASE ? base0 * pow(factor, (double)rot / (rot - 2)) : base0;
  spla_rope* r = new (std::nothrow) spla_rope;
  if (!r) return SPLA_ERR_INVALID_ARG;
  memset(r, 0, sizeof(*r));
  r->t.dim = c->head_dim;
  r->t.rot = rot;
  r->t.interleaved = c->interleaved;
  r->t.amplitude = (float)amplitude;
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (c->scaling == SPLA_ROPE_LINEAR) f /= factor;
    if (c->scaling == SPLA_ROPE_RAMP) {
      double w = (c->original_len * f / two_pi - c->ramp_low) / (c->ramp_high - c->ramp_low);
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      f = w * f + (1.0 - w) * f / factor;
    }
    const double turns = f / two_pi, part = turns - floor(turns);                  // a turn per position more or less changes nothing
    const double scaled = ldexp(part, 64);
    r->t.freq[i] = scaled >= 18446744073709551616.0 ? 0ull : (unsigned long long)scaled;
  }
  *rope_out = r;
  return SPLA_OK;
}

extern "C" int spla_rope_destroy(spla_rope_t* rope) {
  delete rope;
  return SPLA_OK;
}

// One group of heads of spla_rope_apply.
static int rope_group(const spla_rope_tensor_t* t, int dtype, RopeGroup* g) {
  if (!t->in || !t->out || t->n_heads < 1) return SPLA_ERR_INVALID_ARG;
  if (t->n_heads > kRopeMaxHeads) return SPLA_ERR_UNSUPPORTED;
  const size_t e = dtype_bytes(dtype);
  if (!aligned(t->in, e) || !aligned(t->out, e)) return SPLA_ERR_INVALID_ARG;
  if (t->in == t->out && (t->in_batch != t->out_batch || t->in_token != t->out_token || t->in_head != t->out_head)) return SPLA_ERR_INVALID_ARG;
  *g = RopeGroup{t->in, t->out, t->n_heads, 1, t->in_batch, t->in_token, t->in_head, t->out_batch, t->out_token, t->out_head, dtype == SPLA_F32};
  return SPLA_OK;
}

extern "C" int spla_rope_apply(const spla_rope_t* rope, const int32_t* positions, int32_t batch, int32_t n_tokens,
                               const spla_rope_tensor_t* q, const spla_rope_tensor_t* k, int32_t dtype, int32_t transpose, void* stream) {
  if (!rope || !positions || !q || batch < 1 || n_tokens < 1 || !is_dtype(dtype) || !aligned(positions, 4)) return SPLA_ERR_INVALID_ARG;
  RopeGroup g[2];
  int rc = rope_group(q, dtype, &g[0]);
  if (rc == SPLA_OK && k) rc = rope_group(k, dtype, &g[1]);
  if (rc != SPLA_OK) return rc;
  cudaError_t e = launch_rope(rope->t, positions, batch, n_tokens, g, k ? 2 : 1, nullptr, nullptr, nullptr, nullptr, transpose != 0, (cudaStream_t)stream);
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_rope_apply");
}

// ---- the paged cache -------------------------------------------------------------------------------------------------
extern "C" int spla_paged_create(const spla_paged_config_t* c, void* k_pages, void* v_pages, int32_t* status, spla_paged_t** paged_out) {
  if (!c || !k_pages || !v_pages || !status || !paged_out) return SPLA_ERR_INVALID_ARG;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_pages < 1) return SPLA_ERR_INVALID_ARG;
  if (!is_dtype(c->kv_dtype) || !is_dtype(c->q_dtype)) return SPLA_ERR_INVALID_ARG;
  if (!(c->sm_scale >= 0.f) || !isfinite(c->sm_scale * kLog2e) || (c->flags & ~SPLA_GENERAL_KERNELS)) return SPLA_ERR_INVALID_ARG;
  if (c->page_stride < 0 || c->head_stride < 0) return SPLA_ERR_INVALID_ARG;
  if (!aligned(k_pages, 256) || !aligned(v_pages, 256) || !aligned(status, 4)) return SPLA_ERR_INVALID_ARG;
  const int G = c->n_q_heads / c->n_kv_heads, P = c->page_size;
  if (G > kMaxGroup || (c->head_dim != 64 && c->head_dim != 128)) return SPLA_ERR_UNSUPPORTED;
  if (P != 16 && P != 32 && P != 64 && P != 128) return SPLA_ERR_UNSUPPORTED;
  if (c->n_q_heads > kRopeMaxHeads) return SPLA_ERR_UNSUPPORTED;
  const int64_t hs = c->head_stride ? c->head_stride : P, ps = c->page_stride ? c->page_stride : (int64_t)c->n_kv_heads * P;
  if (hs < P || ps < P) return SPLA_ERR_INVALID_ARG;                               // rows of neighbouring heads or pages would overlap
  if (ps >= (1ll << 31) || hs >= (1ll << 31)) return SPLA_ERR_UNSUPPORTED;
  spla_paged* p = new (std::nothrow) spla_paged;
  if (!p) return SPLA_ERR_INVALID_ARG;
  memset(p, 0, sizeof(*p));
  p->cfg = *c;
  p->pl.Hq = c->n_q_heads; p->pl.Hkv = c->n_kv_heads; p->pl.G = G; p->pl.d = c->head_dim; p->pl.P = P;
  for (p->pl.log_p = 0; (1 << p->pl.log_p) < P;) ++p->pl.log_p;
  p->pl.n_pages = c->n_pages;
  p->pl.page_stride = ps;
  p->pl.head_stride = hs;
  p->pl.status = status;
  p->k_pages = k_pages;
  p->v_pages = v_pages;
  if (p->cfg.sm_scale == 0.f) p->cfg.sm_scale = 1.0f / sqrtf((float)c->head_dim);
  p->sm_count = device_sm_count();
  // the tensor-core kernel: bf16, rows that a TMA coordinate can name
  const int64_t rows = (c->n_pages - 1) * ps + (c->n_kv_heads - 1) * hs + P;
  p->tensor = c->kv_dtype == SPLA_BF16 && c->q_dtype == SPLA_BF16 && !(c->flags & SPLA_GENERAL_KERNELS) && rows < (1ll << 31) - 256 &&
              make_kv_map(p->maps.k, k_pages, c->head_dim, P, rows) && make_kv_map(p->maps.v, v_pages, c->head_dim, P, rows);
  *paged_out = p;
  return SPLA_OK;
}

extern "C" int spla_paged_destroy(spla_paged_t* paged) {
  delete paged;
  return SPLA_OK;
}

static int check_batch(const spla_paged* p, const spla_paged_batch_t* b, bool pointers) {
  if (!p || !b) return SPLA_ERR_INVALID_ARG;
  if (b->batch < 1 || b->total_new < 1 || b->max_new < 1 || b->max_len < b->max_new || b->table_stride < 1) return SPLA_ERR_INVALID_ARG;
  if (b->max_len > (int64_t)b->table_stride * p->pl.P) return SPLA_ERR_INVALID_ARG;
  if (b->max_len > (1 << 24)) return SPLA_ERR_UNSUPPORTED;
  if (pointers && (!b->cu_new || !b->seq_lens || !b->page_table || !aligned(b->cu_new, 4) || !aligned(b->seq_lens, 4) || !aligned(b->page_table, 4)))
    return SPLA_ERR_INVALID_ARG;
  return SPLA_OK;
}

static PagedBatch device_batch(const spla_paged_batch_t* b) {
  return PagedBatch{b->cu_new, b->seq_lens, b->page_table, b->batch, b->total_new, b->max_new < b->total_new ? b->max_new : b->total_new,
                    b->max_len, b->table_stride, 0};
}

extern "C" int spla_paged_append(spla_paged_t* p, const spla_paged_batch_t* batch, const spla_rope_t* rope, const int32_t* positions,
                                 const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
                                 void* q_out, int64_t q_out_stride, void* stream) {
  const int rc = check_batch(p, batch, true);
  if (rc != SPLA_OK) return rc;
  if (!k_new || !v_new || (q == nullptr) != (q_out == nullptr) || (rope && rope->t.dim != p->pl.d)) return SPLA_ERR_INVALID_ARG;
  if (k_stride < 0 || v_stride < 0 || q_stride < 0 || q_out_stride < 0) return SPLA_ERR_INVALID_ARG;
  const int d = p->pl.d, ke = dtype_bytes(p->cfg.kv_dtype), qe = dtype_bytes(p->cfg.q_dtype);
  const int64_t kv_row = (int64_t)p->pl.Hkv * d, q_row = (int64_t)p->pl.Hq * d;
  if (!k_stride) k_stride = kv_row;
  if (!v_stride) v_stride = kv_row;
  if (!q_stride) q_stride = q_row;
  if (!q_out_stride) q_out_stride = q_row;
  if (k_stride < kv_row || v_stride < kv_row || (q && (q_stride < q_row || q_out_stride < q_row))) return SPLA_ERR_INVALID_ARG;
  if (!aligned(k_new, ke) || !aligned(v_new, ke) || (q && (!aligned(q, qe) || !aligned(q_out, qe)))) return SPLA_ERR_INVALID_ARG;
  if (q && q == q_out && q_stride != q_out_stride) return SPLA_ERR_INVALID_ARG;
  if (positions && !aligned(positions, 4)) return SPLA_ERR_INVALID_ARG;
  RopeTable none;
  if (!rope) {
    memset(&none, 0, sizeof(none));
    none.dim = d;
  }
  const int kv32 = p->cfg.kv_dtype == SPLA_F32, q32 = p->cfg.q_dtype == SPLA_F32, turn = rope != nullptr;
  const RopeGroup g[3] = {{q, q_out, q ? p->pl.Hq : 0, turn, 0, q_stride, d, 0, q_out_stride, d, q32},
                          {k_new, nullptr, p->pl.Hkv, turn, 0, k_stride, d, 0, 0, 0, kv32},
                          {v_new, nullptr, p->pl.Hkv, 0, 0, v_stride, d, 0, 0, 0, kv32}};
  const PagedBatch pb = device_batch(batch);
  cudaError_t e = launch_rope(rope ? rope->t : none, positions, 1, batch->total_new, g, 3, &pb, &p->pl, p->k_pages, p->v_pages, 0, (cudaStream_t)stream);
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_paged_append");
}

// The plan of one launch (a batch of at most kPagedMaxBatch sequences), the bytes of its partial results and of the sums of long walks,
// and their places in the workspace, where there is one (no cuts: whole units only).
static size_t plan_attend(const spla_paged* p, const PagedBatch& pb, bool tensor, PagedWork* w, void* workspace) {
  if (tensor) paged_plan_mma(w, pb, p->pl, p->sm_count);
  else paged_plan_general(w, pb, p->pl, p->sm_count);
  size_t used = 0;
  auto take = [&](size_t bytes) {
    char* at = workspace ? reinterpret_cast<char*>(workspace) + used : nullptr;
    used += align_up(bytes, 256);
    return reinterpret_cast<void*>(at);
  };
  if (!w->by_unit && w->n_cta >= 2) {
    const size_t rows = (size_t)2 * w->n_cta * w->rows;
    w->part_o = reinterpret_cast<float*>(take(rows * p->pl.d * 4));
    w->part_ml = reinterpret_cast<float2*>(take(rows * 8));
    w->cuts = reinterpret_cast<int4*>(take((size_t)w->n_cta * 16));
  }
  const size_t drain = tensor ? paged_mma_drain_bytes(*w, pb, p->pl) : 0;
  if (drain) w->drain = reinterpret_cast<float*>(take(drain));
  return used;
}

static PagedBatch part_of(PagedBatch b, int first) {
  b.first = first;
  b.cu += first; b.lens += first; b.table += (long long)first * b.table_stride;
  b.batch = b.batch - first < kPagedMaxBatch ? b.batch - first : kPagedMaxBatch;
  return b;
}

// The queries as [token][head][half of 64 channels], boxes of G heads x the tokens of a row tile: its rows, in their order.
static bool make_q_map(void* out128, const void* q, const PagedLayout& pl, int64_t q_stride, const PagedBatch& pb) {
  return make_tile_map_4d(out128, const_cast<void*>(q), 64u, (unsigned)(pl.d / 64), (unsigned)pl.Hq, (unsigned)pb.total_new, 128ull, (unsigned long long)pl.d * 2,
                          (unsigned long long)q_stride * 2, (unsigned)pl.G, (unsigned)paged_mma_positions(pb, pl));
}

// Whether the tensor-core kernel's polynomial for scores under a cap has finite coefficients (the largest is 0.0483 s log2 e (s / cap)^6); with a scale so far
// above the cap (s = 3 and a cap of 10^-6, s = 4 10^5 and a cap of 1), the general kernel's tanh serves the call.
static bool cap_fits(float sm_scale, float softcap) {
  const double s = sm_scale, u = s / softcap;
  return softcap == 0.f || 0.0697 * s * u * u * u * u * u * u < 1e38;
}

extern "C" int spla_paged_query_workspace(const spla_paged_t* p, const spla_paged_batch_t* batch, size_t* bytes_out) {
  const int rc = check_batch(p, batch, false);
  if (rc != SPLA_OK) return rc;
  if (!bytes_out) return SPLA_ERR_INVALID_ARG;
  const PagedBatch pb = device_batch(batch);
  size_t most = 0;
  for (int first = 0; first < batch->batch; first += kPagedMaxBatch) {
    PagedBatch part = pb;
    part.batch = pb.batch - first < kPagedMaxBatch ? pb.batch - first : kPagedMaxBatch;
    for (int tensor = 0; tensor <= (p->tensor ? 1 : 0); ++tensor) {   // (queries that TMA does not take go to the general kernel)
      PagedWork w = {};
      const size_t n = plan_attend(p, part, tensor != 0, &w, nullptr);
      if (n > most) most = n;
    }
  }
  *bytes_out = most;
  return SPLA_OK;
}

extern "C" int spla_paged_attend(spla_paged_t* p, const spla_paged_batch_t* batch, const void* q, int64_t q_stride,
                                 const spla_paged_mask_t* mask, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_batch(p, batch, true);
  if (rc != SPLA_OK) return rc;
  const int qe = dtype_bytes(p->cfg.q_dtype);
  const int64_t q_row = (int64_t)p->pl.Hq * p->pl.d;
  if (!q || !out || q_stride < 0 || !aligned(q, qe) || !aligned(out, 16) || (lse && !aligned(lse, 4))) return SPLA_ERR_INVALID_ARG;
  if (!q_stride) q_stride = q_row;
  if (q_stride < q_row) return SPLA_ERR_INVALID_ARG;
  if (workspace && !aligned(workspace, 256)) return SPLA_ERR_INVALID_ARG;
  spla_paged_mask_t none;
  memset(&none, 0, sizeof(none));
  if (!mask) mask = &none;
  if (!(mask->softcap >= 0.f) || !isfinite(mask->softcap) || (mask->softcap > 0.f && mask->softcap < 1e-6f) || mask->window < 0) return SPLA_ERR_INVALID_ARG;
  if ((mask->slopes && !aligned(mask->slopes, 4)) || (mask->first_key && !aligned(mask->first_key, 4)) || (mask->prefix_lens && !aligned(mask->prefix_lens, 4)))
    return SPLA_ERR_INVALID_ARG;
  size_t need = 0;
  spla_paged_query_workspace(p, batch, &need);
  if (need && (!workspace || workspace_bytes < need)) return SPLA_ERR_INVALID_ARG;

  PagedAttend a = {};
  a.pl = p->pl;
  a.q = q;
  a.q_stride = q_stride;
  a.out = out;
  a.lse = lse;
  a.sm_scale = p->cfg.sm_scale;
  a.softcap = mask->softcap;
  a.window = mask->window;
  a.slopes = mask->slopes;
  a.first_key = mask->first_key;
  a.wait_limit = p->wait_limit;
  a.dbg_tx_extra = p->dbg_tx_extra;
  const PagedBatch pb = device_batch(batch);
  const int q16 = p->cfg.q_dtype == SPLA_BF16, kv16 = p->cfg.kv_dtype == SPLA_BF16;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  PagedMaps maps;
  const bool tensor = p->tensor && aligned(q, 16) && q_stride % 8 == 0 && cap_fits(p->cfg.sm_scale, mask->softcap) && make_q_map(maps.q, q, p->pl, q_stride, pb);
  if (tensor) {
    memcpy(maps.k, p->maps.k, sizeof(maps.k));
    memcpy(maps.v, p->maps.v, sizeof(maps.v));
  }
  for (int first = 0; first < batch->batch && e == cudaSuccess; first += kPagedMaxBatch) {
    a.pb = part_of(pb, first);
    a.prefix = mask->prefix_lens ? mask->prefix_lens + first : nullptr;
    a.w = PagedWork{};
    plan_attend(p, a.pb, tensor, &a.w, workspace);
    e = tensor ? launch_paged_mma(a, maps, s) : launch_paged_general(a, p->k_pages, p->v_pages, q16, kv16, s);
    if (e == cudaSuccess) e = launch_paged_join(a, q16, s);
  }
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_paged_attend");
}

extern "C" int spla_paged_sync_status(spla_paged_t* p, void* stream) {
  if (!p) return SPLA_ERR_INVALID_ARG;
  int st = 0;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaMemcpyAsync(&st, p->pl.status, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && st != 0) e = cudaMemsetAsync(p->pl.status, 0, sizeof(int), s);
  if (e != cudaSuccess) return cuda_fail(e, "spla_paged_sync_status");
  return st;
}

extern "C" int spla_paged_debug_wait_hook(spla_paged_t* p, int32_t max_wait_polls, int32_t extra_expected_bytes) {
  if (!p || max_wait_polls < 0 || extra_expected_bytes < 0 || (extra_expected_bytes % 16)) return SPLA_ERR_INVALID_ARG;
  p->wait_limit = max_wait_polls;
  p->dbg_tx_extra = extra_expected_bytes;
  return SPLA_OK;
}
