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
  PagedPages pages;
  PagedMaps maps;
  bool tensor;                          // bf16 cache and queries, tensor maps made: the tensor-core kernel serves it
  bool few;                             // 8-bit pages and bf16 queries, maps made: paged_few.cu serves sequences of few rows, the tensor-core kernel the others
  bool few32;                           // fp32 queries: paged_few.cu serves sequences of few rows, the fp32 kernel the others
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

static bool norm_fits(const spla_head_norm_t* n) {
  return n->eps >= 0.f && isfinite(n->eps) && (!n->q_weight || aligned(n->q_weight, 4)) && (!n->k_weight || aligned(n->k_weight, 4));
}

static bool rope_norm_tensor(const spla_rope_tensor_t* t, int dtype, bool out) {
  const size_t e = dtype_bytes(dtype);
  return t->in && aligned(t->in, e) && t->n_heads >= 1 && (!out || (t->out && aligned(t->out, e)));
}
static NormGroup norm_group(const spla_rope_tensor_t* x, const spla_rope_tensor_t* dy, const float* weight) {
  NormGroup g = {};
  if (!x) return g;
  const spla_rope_tensor_t* o = dy ? dy : x;
  g.x = x->in; g.out = o->out; g.weight = weight; g.n_heads = x->n_heads;
  g.x_batch = x->in_batch; g.x_token = x->in_token; g.x_head = x->in_head;
  g.out_batch = o->out_batch; g.out_token = o->out_token; g.out_head = o->out_head;
  if (dy) { g.dy = dy->in; g.dy_batch = dy->in_batch; g.dy_token = dy->in_token; g.dy_head = dy->in_head; }
  return g;
}
static bool same_in_place(const void* in, int64_t b, int64_t t, int64_t h, const spla_rope_tensor_t* o) {
  return in != o->out || (b == o->out_batch && t == o->out_token && h == o->out_head);
}
static int check_norm(const spla_rope_t* rope, const int32_t* positions, int32_t batch, int32_t n_tokens, const spla_rope_tensor_t* q, const spla_rope_tensor_t* k,
                      int32_t dtype, const spla_head_norm_t* norm, bool out) {
  if (!rope || !positions || !q || batch < 1 || n_tokens < 1 || !is_dtype(dtype) || !aligned(positions, 4) || !norm || !norm_fits(norm)) return SPLA_ERR_INVALID_ARG;
  if (!norm->q_weight || (k && !norm->k_weight) || !rope_norm_tensor(q, dtype, out) || (k && !rope_norm_tensor(k, dtype, out))) return SPLA_ERR_INVALID_ARG;
  if (q->n_heads > kRopeMaxHeads || (k && k->n_heads > kRopeMaxHeads) || (int64_t)batch * n_tokens >= (1ll << 31)) return SPLA_ERR_UNSUPPORTED;
  return SPLA_OK;
}

extern "C" int spla_rope_norm_apply(const spla_rope_t* rope, const int32_t* positions, int32_t batch, int32_t n_tokens, const spla_rope_tensor_t* q,
                                    const spla_rope_tensor_t* k, int32_t dtype, const spla_head_norm_t* norm, void* stream) {
  const int rc = check_norm(rope, positions, batch, n_tokens, q, k, dtype, norm, true);
  if (rc != SPLA_OK) return rc;
  if (!same_in_place(q->in, q->in_batch, q->in_token, q->in_head, q) || (k && !same_in_place(k->in, k->in_batch, k->in_token, k->in_head, k))) return SPLA_ERR_INVALID_ARG;
  cudaError_t e = launch_norm(rope->t, positions, batch, n_tokens, norm_group(q, nullptr, norm->q_weight), norm_group(k, nullptr, norm->k_weight), norm->eps,
                              dtype == SPLA_F32, false, nullptr, nullptr, nullptr, (cudaStream_t)stream);
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_rope_norm_apply");
}

extern "C" int spla_rope_norm_query_workspace(const spla_rope_t* rope, int32_t batch, int32_t n_tokens, int32_t n_heads, size_t* bytes_out) {
  if (!rope || batch < 1 || n_tokens < 1 || n_heads < 1 || !bytes_out) return SPLA_ERR_INVALID_ARG;
  if (n_heads > 2 * kRopeMaxHeads || (int64_t)batch * n_tokens >= (1ll << 31)) return SPLA_ERR_UNSUPPORTED;
  *bytes_out = norm_part_bytes(rope->t, batch, n_tokens, n_heads, device_sm_count());
  return SPLA_OK;
}

extern "C" int spla_rope_norm_backward(const spla_rope_t* rope, const int32_t* positions, int32_t batch, int32_t n_tokens, const spla_rope_tensor_t* q_grad,
                                       const spla_rope_tensor_t* q, const spla_rope_tensor_t* k_grad, const spla_rope_tensor_t* k, int32_t dtype,
                                       const spla_head_norm_t* norm, float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_norm(rope, positions, batch, n_tokens, q, k, dtype, norm, false);
  if (rc != SPLA_OK) return rc;
  if (!q_grad || (k == nullptr) != (k_grad == nullptr) || !dq_weight || (k && !dk_weight) || !aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return SPLA_ERR_INVALID_ARG;
  if (!rope_norm_tensor(q_grad, dtype, true) || q_grad->n_heads != q->n_heads || (k && (!rope_norm_tensor(k_grad, dtype, true) || k_grad->n_heads != k->n_heads)))
    return SPLA_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i) {                                                    // (dx may take the place of dy or of x)
    const spla_rope_tensor_t *g = i ? k_grad : q_grad, *x = i ? k : q;
    if (g && (!same_in_place(g->in, g->in_batch, g->in_token, g->in_head, g) || !same_in_place(x->in, x->in_batch, x->in_token, x->in_head, g))) return SPLA_ERR_INVALID_ARG;
  }
  size_t need = 0;
  const int rw = spla_rope_norm_query_workspace(rope, batch, n_tokens, q->n_heads + (k ? k->n_heads : 0), &need);
  if (rw != SPLA_OK) return rw;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < need) return SPLA_ERR_INVALID_ARG;
  cudaError_t e = launch_norm(rope->t, positions, batch, n_tokens, norm_group(q, q_grad, norm->q_weight), norm_group(k, k_grad, norm->k_weight), norm->eps,
                              dtype == SPLA_F32, true, dq_weight, dk_weight, workspace, (cudaStream_t)stream);
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_rope_norm_backward");
}

// ---- the paged cache -------------------------------------------------------------------------------------------------
// k_scales: null for pages of 16 or 32 bits.
static int create_paged(const spla_paged_config_t* c, void* k_pages, void* v_pages, uint8_t* k_scales, uint8_t* v_scales, int32_t* status, spla_paged_t** paged_out) {
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
  // (a row's scale is found by its number: pages and heads without gaps; a row of new tokens is one launch's)
  if (k_scales && (hs != P || ps != (int64_t)c->n_kv_heads * P || c->q_dtype != c->kv_dtype)) return SPLA_ERR_UNSUPPORTED;
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
  p->pages = PagedPages{k_pages, v_pages, k_scales, v_scales, k_scales ? kPagesE4m3 : c->kv_dtype == SPLA_F32 ? kPagesF32 : kPagesBf16};
  if (p->cfg.sm_scale == 0.f) p->cfg.sm_scale = 1.0f / sqrtf((float)c->head_dim);
  p->sm_count = device_sm_count();
  // the tensor-core kernel: bf16, rows that a TMA coordinate can name
  const int64_t rows = (c->n_pages - 1) * ps + (c->n_kv_heads - 1) * hs + P;
  p->tensor = !k_scales && c->kv_dtype == SPLA_BF16 && c->q_dtype == SPLA_BF16 && !(c->flags & SPLA_GENERAL_KERNELS) && rows < (1ll << 31) - 256 &&
              make_kv_map(p->maps.k, k_pages, c->head_dim, P, rows) && make_kv_map(p->maps.v, v_pages, c->head_dim, P, rows);
  // (scales of 2^60 and more would leave the range that its exponents are kept in)
  const bool bytes = k_scales && !(c->flags & SPLA_GENERAL_KERNELS) && rows < (1ll << 31) - 256 && p->cfg.sm_scale < 1.15e18f &&
           make_byte_map(p->maps.k, k_pages, c->head_dim, P, rows) && make_byte_map(p->maps.v, v_pages, c->head_dim, P, rows);
  p->few = bytes && c->q_dtype == SPLA_BF16;
  p->few32 = bytes && c->q_dtype == SPLA_F32;
  *paged_out = p;
  return SPLA_OK;
}

extern "C" int spla_paged_create(const spla_paged_config_t* c, void* k_pages, void* v_pages, int32_t* status, spla_paged_t** paged_out) {
  return create_paged(c, k_pages, v_pages, nullptr, nullptr, status, paged_out);
}

extern "C" int spla_paged_create_scaled(const spla_paged_config_t* c, void* k_pages, void* v_pages, uint8_t* k_scales, uint8_t* v_scales, int32_t* status,
                                      spla_paged_t** paged_out) {
  if (!k_scales || !v_scales) return SPLA_ERR_INVALID_ARG;
  return create_paged(c, k_pages, v_pages, k_scales, v_scales, status, paged_out);
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

extern "C" int spla_paged_append_norm(spla_paged_t* p, const spla_paged_batch_t* batch, const spla_rope_t* rope, const int32_t* positions,
                                      const spla_head_norm_t* norm, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                                      const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, void* stream) {
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
  if (norm && !norm_fits(norm)) return SPLA_ERR_INVALID_ARG;
  const bool normed = norm && (norm->k_weight || (q && norm->q_weight));
  const int kv32 = p->cfg.kv_dtype == SPLA_F32, q32 = p->cfg.q_dtype == SPLA_F32, turn = rope != nullptr;
  const PagedBatch pb = device_batch(batch);
  cudaError_t e;
  if (p->pages.type == kPagesE4m3 || normed) {
    const StoreGroups g{q, k_new, v_new, q_out, q_stride, k_stride, v_stride, q_out_stride, q32, kv32, norm ? norm->q_weight : nullptr,
                        norm ? norm->k_weight : nullptr, norm ? norm->eps : 0.f, positions};
    e = launch_store(rope ? &rope->t : nullptr, g, pb, p->pl, p->pages, (cudaStream_t)stream);
  } else {
    RopeTable none;
    if (!rope) {
      memset(&none, 0, sizeof(none));
      none.dim = d;
    }
    const RopeGroup g[3] = {{q, q_out, q ? p->pl.Hq : 0, turn, 0, q_stride, d, 0, q_out_stride, d, q32},
                            {k_new, nullptr, p->pl.Hkv, turn, 0, k_stride, d, 0, 0, 0, kv32},
                            {v_new, nullptr, p->pl.Hkv, 0, 0, v_stride, d, 0, 0, 0, kv32}};
    e = launch_rope(rope ? rope->t : none, positions, 1, batch->total_new, g, 3, &pb, &p->pl, p->pages.k, p->pages.v, 0, (cudaStream_t)stream);
  }
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_paged_append");
}

extern "C" int spla_paged_append(spla_paged_t* p, const spla_paged_batch_t* batch, const spla_rope_t* rope, const int32_t* positions,
                                 const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
                                 void* q_out, int64_t q_out_stride, void* stream) {
  return spla_paged_append_norm(p, batch, rope, positions, nullptr, k_new, k_stride, v_new, v_stride, q, q_stride, q_out, q_out_stride, stream);
}

extern "C" int spla_paged_read(spla_paged_t* p, const spla_paged_batch_t* batch, void* k_out, void* v_out, int32_t out_dtype, void* stream) {
  const int rc = check_batch(p, batch, true);
  if (rc != SPLA_OK) return rc;
  if (!k_out || !v_out || !is_dtype(out_dtype) || !aligned(k_out, 16) || !aligned(v_out, 16)) return SPLA_ERR_INVALID_ARG;
  cudaError_t e = launch_read(device_batch(batch), p->pl, p->pages, k_out, v_out, out_dtype == SPLA_F32, (cudaStream_t)stream);
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_paged_read");
}

// Which kernel a launch is: fp32 arithmetic, bf16 on the tensor cores, 8-bit pages with few rows, 8-bit pages on the tensor cores, the same widened to bf16 before.
enum PagedKernel { kGeneral, kTensor, kFew, kTensorBytes, kTensorWide };

// 8-bit pages, sequences of more rows than few: where there are enough rows for each key, the keys and values (with a window, its and the sinks') are widened to
// bf16 in a pass of their own, once for all rows, and the kernel for bf16 pages does the rest.  Graphs, us, this way and over the 8-bit pages: a prompt of 8192 tokens 539 and
// 688, of 1000 43 and 55, of 64 31 and 41; ragged ones of up to 2000 x16 307 and 436; 4000 on 4000 with a window of 512 119 and 162; 1 to 600 on 100 to 9000 x24 with a window of
// 2048 182 and 217; 512 on 3500 x4 186 and 207, on 7000 x2 174 and 186.
// It pays from 1000 to 1500 rows of queries for each key on (32 heads in 8 groups of 128: 512 tokens, 2048 rows, on 8000 117 and 127, on 32768 x4 1243 and 1299, 2048 tokens there 4507 and
// 5256; 128 tokens on 8000 x4 150 and 127, on 32768 x4 473 and 363), and on caches of no more than 2000 with any number, where it is a launch less, or two (33 tokens on none 27 and 39, on
// 2000 41 and 47).  What is looked at here instead is memory: up to four times the queries' parts, or eight where the sequences have 512 rows on average (200 on 2800 x8 170 and 177), so that
// the longest caches are left to the slower way (512 on 32768 360 in place of 330, 2048 on 32768 x4 5174 of 4507).  (Documents: which keys are looked at is not known before; they go without.)
// Weights are rounded to bf16 this way, 2^-8, to fp16 the other, 2^-11: the error of out against float64 (2-norm) is 2.0e-3 in place of 1.7e-3, which is what the rounding of
// out takes alone.  It goes by the call's sizes, so a sequence may be served the one way in one batch and the other in the next.
static size_t wide_most(const spla_paged* p, const PagedBatch& pb) {
  size_t exps;
  return ((long long)pb.total_new * p->pl.G >= 512ll * pb.batch ? 8 : 4) * paged_split_bytes(p->pl, pb.total_new, &exps);
}
// Bytes of the workspace's front, the same for all launches of a call: the queries' parts, or the widened tokens as far as they may be widened.
static size_t front_bytes(const spla_paged* p, const PagedBatch& pb) {
  if (!p->few || pb.max_new <= paged_few_positions(p->pl)) return 0;
  size_t exps;
  const size_t parts = paged_split_bytes(p->pl, pb.total_new, &exps), limit = wide_most(p, pb);
  const PagedWide w = paged_wide(p->pl, pb, 0, 0);                                 // (less with a window, which is not known here)
  const size_t most = w.fits && w.bytes < limit ? w.bytes : limit;
  return most > parts ? most : parts;
}

// The plan of one launch (a batch of at most kPagedMaxBatch sequences), the bytes of its partial results and of the sums of long walks,
// and their places in the workspace, where there is one (no cuts: whole units only).
// (8-bit pages: where a sequence may have more rows than the kernel for few takes, the queries' parts lie in front, the same for all launches of a call; or in
// their place, where they take no more than that, the widened tokens.)
static size_t plan_attend(const spla_paged* p, PagedBatch pb, PagedKernel kernel, size_t front, PagedWork* w, void* workspace) {
  const bool tensor = kernel == kTensor || kernel == kTensorBytes || kernel == kTensorWide;
  const bool parts = kernel != kGeneral && kernel != kTensor && pb.max_new > paged_few_positions(p->pl);
  if (kernel == kFew && pb.max_new > paged_few_positions(p->pl)) pb.max_new = paged_few_positions(p->pl);   // (the others are another launch's)
  if (tensor) paged_plan_mma(w, pb, p->pl, p->sm_count);
  else if (kernel == kFew) paged_plan_few(w, pb, p->pl, p->sm_count);
  else paged_plan_general(w, pb, p->pl, p->sm_count);
  size_t used = 0;
  if (parts) used = align_up(front, 256);
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

// The queries as [token][head][half of 64 channels], boxes of G heads x the tokens of a row tile: its rows, in their order.  (The parts of paged_split.cu lie
// the same way: 2 d bytes a head, in pieces of 128.)
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
  const size_t front = front_bytes(p, pb);
  size_t most = 0;
  for (int first = 0; first < batch->batch; first += kPagedMaxBatch) {
    PagedBatch part = pb;
    part.batch = pb.batch - first < kPagedMaxBatch ? pb.batch - first : kPagedMaxBatch;
    for (PagedKernel kernel : {kGeneral, kTensor, kFew, kTensorBytes}) {   // (queries that TMA does not take go to the general kernel)
      if ((kernel == kTensor && !p->tensor) || (kernel == kFew && !p->few && !p->few32) || (kernel == kTensorBytes && !p->few)) continue;
      PagedWork w = {};
      const size_t n = plan_attend(p, part, kernel, front, &w, nullptr);
      if (n > most) most = n;
    }
  }
  *bytes_out = most;
  return SPLA_OK;
}

extern "C" int spla_paged_attend_sinks(spla_paged_t* p, const spla_paged_batch_t* batch, const void* q, int64_t q_stride, const spla_paged_mask_t* mask,
                                       int32_t sinks, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
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
  if (sinks < 0) return SPLA_ERR_INVALID_ARG;
  if (sinks > 0 && mask->first_key) return SPLA_ERR_UNSUPPORTED;                   // (which document's first tokens?)
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
  a.sinks = mask->window > 0 ? sinks : 0;
  a.slopes = mask->slopes;
  a.first_key = mask->first_key;
  a.wait_limit = p->wait_limit;
  a.dbg_tx_extra = p->dbg_tx_extra;
  const PagedBatch pb = device_batch(batch);
  a.k_scales = p->pages.k_scales;
  a.v_scales = p->pages.v_scales;
  const int q16 = p->cfg.q_dtype == SPLA_BF16;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  PagedMaps maps;
  const bool rows16 = aligned(q, 16) && q_stride % 8 == 0, few = p->few && rows16, few32 = p->few32 && aligned(q, 16) && q_stride % 4 == 0;
  const bool parts = few && pb.max_new > paged_few_positions(p->pl);               // some sequences may have more rows: their queries in two parts
  const bool tensor_fits = (p->tensor || parts) && rows16 && cap_fits(p->cfg.sm_scale, mask->softcap);
  const PagedWide w = paged_wide(p->pl, pb, a.window, a.sinks);
  const size_t front_size = front_bytes(p, pb);
  size_t exps = 0;
  char* front = reinterpret_cast<char*>(workspace);
  PagedMaps wide_maps;
  const bool wide = tensor_fits && parts && !mask->first_key && w.fits && w.bytes <= wide_most(p, pb) &&
                    make_kv_map(wide_maps.k, front, p->pl.d, kWidePage, (unsigned long long)w.pl.n_pages * w.pl.page_stride) &&
                    make_kv_map(wide_maps.v, front + w.v_at, p->pl.d, kWidePage, (unsigned long long)w.pl.n_pages * w.pl.page_stride) &&
                    make_q_map(wide_maps.q, q, p->pl, q_stride, pb);
  const bool tensor = !wide && tensor_fits && make_q_map(maps.q, parts ? workspace : q, p->pl, parts ? q_row : q_stride, pb);
  if (tensor || few || few32) {
    memcpy(maps.k, p->maps.k, sizeof(maps.k));
    memcpy(maps.v, p->maps.v, sizeof(maps.v));
  }
  auto launch = [&](PagedKernel kernel, int from_new, int to_new) {
    if (e != cudaSuccess) return;
    a.from_new = from_new;
    a.to_new = to_new;
    a.w = PagedWork{};
    plan_attend(p, a.pb, kernel, front_size, &a.w, workspace);
    switch (kernel) {
      case kTensor: e = launch_paged_mma(a, maps, s); break;
      case kFew: e = launch_paged_few(a, maps, !q16, s); break;
      case kTensorWide: {
        PagedAttend b = a;
        b.pl = w.pl;
        b.pb.table = reinterpret_cast<const int*>(front + w.table_at) + (long long)a.pb.first * w.cols;
        b.pb.table_stride = w.cols;
        e = launch_paged_mma(b, wide_maps, s);
        break;
      }
      case kTensorBytes: e = p->pl.d == 128 ? launch_paged_mma_bytes128(a, maps, s) : launch_paged_mma_bytes64(a, maps, s); break;
      default: e = launch_paged_general(a, p->pages, q16, s);
    }
    if (e == cudaSuccess) e = launch_paged_join(a, q16, s);
  };
  if (wide) {
    e = launch_paged_widen(pb, p->pl, p->pages, w, a.window, front, s);
  } else if (parts && tensor) {
    paged_split_bytes(p->pl, pb.total_new, &exps);
    unsigned char* at = reinterpret_cast<unsigned char*>(workspace);
    a.q_exp = reinterpret_cast<signed char*>(at + exps);
    e = launch_paged_split(p->pl, q, q_stride, pb.total_new, at, reinterpret_cast<signed char*>(at + exps), s);
  }
  for (int first = 0; first < batch->batch && e == cudaSuccess; first += kPagedMaxBatch) {
    a.pb = part_of(pb, first);
    a.prefix = mask->prefix_lens ? mask->prefix_lens + first : nullptr;
    if (wide) {                                                                    // (sequences of few rows too: one launch less)
      launch(kTensorWide, 0, 0);
    } else if (few || few32) {                                                           // two launches where a sequence may have more rows (see paged_few_positions)
      const int most = paged_few_positions(p->pl);
      launch(kFew, 0, most);
      if (pb.max_new > most) launch(tensor ? kTensorBytes : kGeneral, most + 1, 0x7fffffff);
    } else {
      launch(tensor ? kTensor : kGeneral, 0, 0);
    }
  }
  return e == cudaSuccess ? SPLA_OK : cuda_fail(e, "spla_paged_attend");
}

extern "C" int spla_paged_attend(spla_paged_t* p, const spla_paged_batch_t* batch, const void* q, int64_t q_stride,
                                 const spla_paged_mask_t* mask, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return spla_paged_attend_sinks(p, batch, q, q_stride, mask, 0, out, lse, workspace, workspace_bytes, stream);
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
