// Instances of the attention kernel for few rows over a 4-bit cache.
#include "tl_attend_four.cuh"

namespace tl {
int attend_small_e2m1(bool launch, int dim, int rows, int* tile, int* per_sm, const AttendParams* p, int ctas, cudaStream_t stream) {
    auto pick = [&](auto one, auto two, auto four) { return (rows == 8 ? one : rows == 16 ? two : four)(launch, tile, per_sm, p, ctas, stream); };
    if (dim == 64) return pick(attend_four_one<64, 1>, attend_four_one<64, 2>, attend_four_one<64, 4>);
    if (dim == 128) return pick(attend_four_one<128, 1>, attend_four_one<128, 2>, attend_four_one<128, 4>);
    return pick(attend_four_one<256, 1>, attend_four_one<256, 2>, attend_four_one<256, 2>);
}
}  // namespace tl
