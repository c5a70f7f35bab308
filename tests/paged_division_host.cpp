// The division of the paged attention's work (csrc/paged.h), run on the CPU: the device functions of one CTA of one warp, as they are, in 32
// fibers that change at every warp instruction.  Built and called by test_paged_division.py.
#include <math.h>
#include <ucontext.h>

#include <algorithm>
#include <cstdio>
#include <memory>
#include <vector>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace warp {
constexpr int kLanes = 32;
static ucontext_t home, lanes[kLanes];
static bool over[kLanes];
static int lane;
static long long box[2][kLanes];
static int turn[kLanes];
static void (*body)();

static void next_lane() {                                          // round robin: every lane runs from one warp instruction to the next
  const int from = lane;
  lane = (lane + 1) % kLanes;
  swapcontext(&lanes[from], &lanes[lane]);
}
// All lanes' values of this instruction (two boxes in turn: the next instruction's come while the last lanes still read).
static const long long* meet(long long v) {
  const int t = turn[lane]++ & 1;
  box[t][lane] = v;
  next_lane();
  return box[t];
}
static void start() {
  body();
  over[lane] = true;
  if (lane == kLanes - 1) setcontext(&home);
  const int from = lane++;
  swapcontext(&lanes[from], &lanes[lane]);
}
static void run(void (*f)()) {
  static std::vector<char> stacks(kLanes * 256 * 1024);
  body = f;
  for (int i = 0; i < kLanes; ++i) {
    turn[i] = 0;
    over[i] = false;
    getcontext(&lanes[i]);
    lanes[i].uc_stack.ss_sp = stacks.data() + i * 256 * 1024;
    lanes[i].uc_stack.ss_size = 256 * 1024;
    lanes[i].uc_link = nullptr;
    makecontext(&lanes[i], start, 0);
  }
  lane = 0;
  swapcontext(&home, &lanes[0]);
}
struct Index { int x; };
}  // namespace warp

#define threadIdx (warp::Index{warp::lane})
#define blockIdx (warp::Index{0})
using std::max;
using std::min;
template <typename T> static T __ldg(const T* p) { return *p; }
template <typename T> static T __ldcg(const T* p) { return *p; }
template <typename T> static T __shfl_sync(unsigned, T v, int from) { return (T)warp::meet((long long)v)[from & 31]; }
template <typename T> static T __shfl_up_sync(unsigned, T v, int by) { const int me = warp::lane; const long long* all = warp::meet((long long)v); return (T)all[me >= by ? me - by : me]; }
template <typename T> static T __shfl_xor_sync(unsigned, T v, int by) { const int me = warp::lane; return (T)warp::meet((long long)v)[me ^ by]; }
static unsigned __ballot_sync(unsigned, bool p) { const long long* all = warp::meet(p); unsigned m = 0; for (int i = 0; i < 32; ++i) m |= (unsigned)(all[i] != 0) << i; return m; }
static int __any_sync(unsigned m, bool p) { return __ballot_sync(m, p) != 0; }
static int __all_sync(unsigned m, bool p) { return __ballot_sync(m, p) == 0xffffffffu; }
static int __reduce_add_sync(unsigned, int v) { const long long* all = warp::meet(v); unsigned s = 0; for (int i = 0; i < 32; ++i) s += (unsigned)all[i]; return (int)s; }
static int __reduce_max_sync(unsigned, int v) { const long long* all = warp::meet(v); return (int)*std::max_element(all, all + 32); }
static int __reduce_min_sync(unsigned, int v) { const long long* all = warp::meet(v); return (int)*std::min_element(all, all + 32); }
static void __syncthreads() { warp::meet(0); }
static int __syncthreads_or(int p) { return __ballot_sync(0xffffffffu, p) != 0; }
static int __popc(unsigned v) { return __builtin_popcount(v); }
static int __ffs(int v) { return __builtin_ffs(v); }
static int atomicExch(int* p, int v) { const int o = *p; *p = v; return o; }
// (used by device code of the headers that is not run here)
static void __nanosleep(unsigned) {}
static float __uint_as_float(unsigned v) { float f; __builtin_memcpy(&f, &v, 4); return f; }
static unsigned __float_as_uint(float f) { unsigned v; __builtin_memcpy(&v, &f, 4); return v; }
static float __fmul_rn(float a, float b) { return a * b; }
static float __fadd_rn(float a, float b) { return a + b; }
static int __float_as_int(float f) { return (int)__float_as_uint(f); }
static float __int_as_float(int v) { return __uint_as_float((unsigned)v); }
static size_t __cvta_generic_to_shared(const void* p) { return (size_t)p; }

#include "paged.h"

namespace {
spla::PagedAttend A;
std::unique_ptr<spla::PagedSeqs> seqs;
long long total, share;
int cta;
long long* seg_out;
int seg_room, seg_count;
int cut_out[4];

void fill() {
  const long long all = spla::paged_fill_seqs(A, *seqs, warp::lane, 32);
  if (warp::lane == 0) { total = all; share = spla::paged_share(A.w, all); }
}
int owner_base, owner_step, owner_of[4];
void owner() {
  const int b = spla::paged_owner<4>(A.pb, owner_base, owner_step, warp::lane);
  if (warp::lane < 4) owner_of[warp::lane] = b;
}
void walk() {
  spla::PagedWalk wk;
  const bool any = wk.seek(A, *seqs, cta * share, share);
  const int4 cut = wk.cut_here(A, any, share);
  int n = 0;
  while (any && n < seg_room && wk.next(A, *seqs)) {
    if (warp::lane == 0) {
      const long long v[8] = {wk.b, wk.h, wk.u_cur, wk.t0, wk.t1, wk.head, wk.tail, wk.n_pos(A.w)};
      for (int i = 0; i < 8; ++i) seg_out[8 * n + i] = v[i];
    }
    ++n;
  }
  if (warp::lane == 0) { seg_count = n; cut_out[0] = cut.x; cut_out[1] = cut.y; cut_out[2] = cut.z; cut_out[3] = cut.w; }
}
}  // namespace

extern "C" {
// plan: ppos, upos, log_tk, by_unit, n_cta, min_tiles, extra, Hkv, G, total_new, max_new, max_len, window, narrow (-1: as the launch would have it), first
// (sequences of earlier launches: cu, lens and prefix start with theirs).
// out: total, share, status, narrow; pre[batch + 1], n[batch]
void division_fill(const int* plan, int batch, const int* cu, const int* lens, const int* prefix, const int* first_key, long long* out, long long* pre, int* n) {
  static int status;
  status = 0;
  A = spla::PagedAttend{};
  A.w.ppos = plan[0]; A.w.upos = plan[1]; A.w.log_tk = plan[2]; A.w.by_unit = plan[3]; A.w.n_cta = plan[4]; A.w.min_tiles = plan[5]; A.w.extra = plan[6];
  A.pl.Hkv = plan[7]; A.pl.G = plan[8]; A.pl.status = &status;
  A.pb.first = plan[14];
  A.pb.cu = cu + plan[14]; A.pb.lens = lens + plan[14]; A.pb.batch = batch; A.pb.total_new = plan[9]; A.pb.max_new = plan[10]; A.pb.max_len = plan[11];
  A.window = plan[12]; A.prefix = prefix ? prefix + plan[14] : nullptr; A.first_key = first_key;
  A.w.narrow = plan[13] < 0 ? spla::paged_narrow(A.w, A.pb, A.pl) : plan[13];
  if (!seqs) seqs.reset(new spla::PagedSeqs);
  warp::run(fill);
  out[0] = total; out[1] = share; out[2] = status; out[3] = A.w.narrow;
  for (int b = 0; b <= batch; ++b) pre[b] = seqs->pre[b];
  for (int b = 0; b < batch; ++b) n[b] = seqs->n[b];
}
// The sequences that the append looks up for the tokens base + k step, k < 4 (-1: none), in the batch of the last division_fill.
void division_owner(int base, int step, int* out) {
  owner_base = base; owner_step = step;
  warp::run(owner);
  std::copy(owner_of, owner_of + 4, out);
}
// Segments of one CTA: [count][b, h, u, t0, t1, head, tail, positions]; the cut at its start: rows, parts, first row, head.
int division_walk(int which, int room, long long* segments, int* cut) {
  cta = which; seg_out = segments; seg_room = room;
  warp::run(walk);
  std::copy(cut_out, cut_out + 4, cut);
  return seg_count;
}
}
