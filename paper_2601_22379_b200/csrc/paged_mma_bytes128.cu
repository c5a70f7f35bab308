// The tensor-core attention over 8-bit pages (paged_mma.cuh), heads of 128.
#include "paged_mma.cuh"

namespace spla {

cudaError_t launch_paged_mma_bytes128(const PagedAttend& a, const PagedMaps& maps, cudaStream_t s) { return mma_d<128, true>(a, maps, s); }

}  // namespace spla
