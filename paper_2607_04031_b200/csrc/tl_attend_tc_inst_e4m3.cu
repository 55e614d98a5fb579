// Instances of the tensor-core attention kernel over a e4m3 cache.
#include "tl_attend_tc_inst.cuh"

namespace tl {
int attend_tc_e4m3(int dim, int blocks, const tl_kv_cache* cache, const AttendParams& p, cudaStream_t stream) {
    return attend_tc<TL_KV_E4M3>(dim, blocks, cache, p, stream);
}
}  // namespace tl
