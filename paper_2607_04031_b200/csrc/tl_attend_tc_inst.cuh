// Launch of the tensor-core attention kernel for one cache format.
#pragma once

#include <algorithm>
#include <cstring>

#include "tl_attend_tc.cuh"

namespace tl {

template <int kDim, int kFmt, int kBlocks>
int launch_attend_tc(const tl_kv_cache* cache, const AttendParams& p, cudaStream_t stream) {
    using S = TcShape<kDim, kBlocks>;
    AttendTcParams tp;
    memset(&tp, 0, sizeof tp);
    tp.a = p;
    tp.wait_ns = wait_limit_ns();
    if (opt(TL_OPT_STALL_ONCE) == 5) {
        tp.stall = 1;
        tl_set_option(TL_OPT_STALL_ONCE, 0);
    }
    tp.box_tokens = std::min(cache->page_tokens, kTcTile);
    if (kFmt == TL_KV_BF16) {
        // [page][head][token][dim]; a box holds 64 dimensions (128 bytes, the swizzle's width) of one page's tokens
        const uint64_t dims[4] = {uint64_t(kDim), uint64_t(cache->page_tokens), uint64_t(p.cache.heads), uint64_t(p.cache.pages)};
        const uint64_t strides[4] = {2, uint64_t(p.cache.token_stride), uint64_t(p.cache.head_stride), uint64_t(p.cache.page_stride)};
        const uint32_t box[4] = {64, uint32_t(tp.box_tokens), 1, 1};
        for (int i = 0; i < 2; ++i)
            if (int rc = encode_tensor_map(&tp.map[i], p.cache.base[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, 4, dims, strides, box))
                return rc;
    }
    if (int rc = ensure_smem_attr(reinterpret_cast<const void*>(attend_tc_kernel<kDim, kFmt, kBlocks>), S::kSmem)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(p.ctas));
    cfg.blockDim = dim3(kTcThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = opt(TL_OPT_PDL) != 0 ? 1 : 0;
    return check_cuda(cudaLaunchKernelEx(&cfg, attend_tc_kernel<kDim, kFmt, kBlocks>, tp));
}

template <int kFmt>
int attend_tc(int dim, int blocks, const tl_kv_cache* cache, const AttendParams& p, cudaStream_t stream) {
    if (dim == 64) return blocks == 2 ? launch_attend_tc<64, kFmt, 2>(cache, p, stream) : launch_attend_tc<64, kFmt, 1>(cache, p, stream);
    return blocks == 2 ? launch_attend_tc<128, kFmt, 2>(cache, p, stream) : launch_attend_tc<128, kFmt, 1>(cache, p, stream);
}

}  // namespace tl
