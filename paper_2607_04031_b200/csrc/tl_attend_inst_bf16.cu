// Instances of the attention kernel for few rows over a bf16 cache.
#include "tl_attend_inst.cuh"

namespace tl {
int attend_small_bf16(bool launch, int dim, int rows, int* tile, int* per_sm, const AttendParams* p, int ctas, cudaStream_t stream) {
    return attend_small<TL_KV_BF16>(launch, dim, rows, tile, per_sm, p, ctas, stream);
}
}  // namespace tl
