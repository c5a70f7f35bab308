// The tensor-core attention over bf16 pages (paged_mma.cuh), and the division of its work.
#include "paged_mma.cuh"

namespace spla {

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
  return a.pl.d == 128 ? mma_d<128, false>(a, maps, s) : mma_d<64, false>(a, maps, s);
}

}  // namespace spla
