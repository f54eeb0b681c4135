// Instances of the score-cache kernel over a bf16 cache with a scale for each page.
#include "verify_sm100_cached.cuh"

namespace spec {
namespace sm100 {

int launch_cached_scaled_pages(const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq, const FastParams& fp, int grid,
                         size_t smem_bytes, cudaStream_t stream)
{
    return launch_rows<false, 2, false, false>(tk, tv, tq, fp, grid, smem_bytes, stream);
}

}  // namespace sm100
}  // namespace spec
