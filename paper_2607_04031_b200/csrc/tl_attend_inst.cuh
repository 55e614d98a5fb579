// Dispatch of the attention kernel for few rows over head dimension and row count, for one cache format.
#pragma once

#include "tl_attend_small.cuh"

namespace tl {

template <int kDim, int kFmt, int kMT>
int attend_small_one(bool launch, int* tile, int* per_sm, const AttendParams* p, int ctas, cudaStream_t stream) {
    using S = SmallShape<kDim, kFmt, kMT>;
    if (launch) return launch_attend_small<kDim, kFmt, kMT>(*p, ctas, stream);
    *tile = S::kTile;
    *per_sm = S::kCtasPerSm;
    return TL_OK;
}
template <int kFmt>
int attend_small(bool launch, int dim, int rows, int* tile, int* per_sm, const AttendParams* p, int ctas, cudaStream_t stream) {
    if (dim == 64) return rows == 32 ? attend_small_one<64, kFmt, 2>(launch, tile, per_sm, p, ctas, stream)
                                     : attend_small_one<64, kFmt, 1>(launch, tile, per_sm, p, ctas, stream);
    if (dim == 128) return rows == 32 ? attend_small_one<128, kFmt, 2>(launch, tile, per_sm, p, ctas, stream)
                                      : attend_small_one<128, kFmt, 1>(launch, tile, per_sm, p, ctas, stream);
    return attend_small_one<256, kFmt, 1>(launch, tile, per_sm, p, ctas, stream);
}

}  // namespace tl
