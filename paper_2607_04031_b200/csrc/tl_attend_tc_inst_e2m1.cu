// Instances of the tensor-core attention kernel over an e2m1 cache.
#include "tl_attend_tc_inst.cuh"

namespace tl {
int attend_tc_e2m1(int dim, int blocks, const tl_kv_cache* cache, const AttendParams& p, cudaStream_t stream) {
    return attend_tc<TL_KV_E2M1>(dim, blocks, cache, p, stream);
}
}  // namespace tl
