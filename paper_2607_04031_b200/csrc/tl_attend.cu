// tl_tree_attention: argument checks, the choice of kernel, and the kernel that joins the parts of split sequences.
#include "tl_attend.cuh"

#include <algorithm>
#include <cmath>

namespace tl {

// Joins the units that cross a border between CTA ranges.  Blocks (c, *) look at the border in front of CTA c + 1; the
// borders inside one unit share its rows out among themselves, and so do the blocks of a border (one per 16 rows of the
// unit: with one block a border, 256-row units took 33 to 60 us here, a chain of dependent loads per row).
constexpr int kCombineThreads = 256, kCombineRows = 16;
// From this many parts of a unit on four lanes share an element's: units in so many parts are few or narrow, and most
// threads would have nothing to do.  Whole calls over 4100 positions, one lane / four lanes: 1 request of 16 rows E4M3 (33
// parts) 35.8 / 27.6 us, bf16 of 32 rows (17) 31.7 / 29.7, 4 requests of 16 rows E4M3 (14) 35.8 / 33.8; 512 rows over 16000
// (10 parts of 256 rows) 76.8 / 78.8.
constexpr int kCombineMany = 12;

struct CombineUnit {
    AttendPlace w;
    int c0, c1;                          // the CTAs that hold parts
    int rows, share, shares;
};
template <int kLanes>
__device__ __forceinline__ void combine_unit(const AttendParams& p, const CombineUnit& u, int dim) {
    const int vecs = dim / 4;
    // (a row has 16 elements of four dimensions at least: with four lanes each, a warp is inside or outside as a whole)
    for (int x = u.share * kCombineThreads + int(threadIdx.x); x < u.rows * vecs * kLanes; x += u.shares * kCombineThreads) {
        const int e = x / kLanes, sub = x % kLanes;
        const int r = e / vecs, d = e % vecs * 4;
        // CTA c0 ends inside the unit it began (its second slot); the others begin inside it (their first)
        auto slot = [&](int c) { return int64_t(c) * 2 + (c == u.c0 ? 1 : 0); };
        float top = -INFINITY;
#pragma unroll 4
        for (int c = u.c0 + sub; c <= u.c1; c += kLanes) top = fmaxf(top, p.part_ml[slot(c) * p.rows_block + r].x);
#pragma unroll
        for (int k = 1; k < kLanes; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        const float use = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = u.c0 + sub; c <= u.c1; c += kLanes) {
            const float2 ml = p.part_ml[slot(c) * p.rows_block + r];
            const float4 v = *reinterpret_cast<const float4*>(p.part + (slot(c) * p.rows_block + r) * dim + d);
            const float f = ex2(ml.x - use);
            sum = fmaf(ml.y, f, sum);
            o.x = fmaf(v.x, f, o.x), o.y = fmaf(v.y, f, o.y), o.z = fmaf(v.z, f, o.z), o.w = fmaf(v.w, f, o.w);
        }
#pragma unroll
        for (int k = 1; k < kLanes; k <<= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, k);
            o.x += __shfl_xor_sync(0xffffffffu, o.x, k), o.y += __shfl_xor_sync(0xffffffffu, o.y, k);
            o.z += __shfl_xor_sync(0xffffffffu, o.z, k), o.w += __shfl_xor_sync(0xffffffffu, o.w, k);
        }
        if (kLanes > 1 && sub != 0) continue;
        const AttendPlace& w = u.w;
        const int row = w.block * p.rows_block + r, tok = row / p.group, hq = w.head * p.group + row % p.group;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint2*>(p.out + int64_t(w.a.r.first + tok) * p.out_stride + int64_t(hq) * dim + d) =
            make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        if (p.lse && d == 0) p.lse[int64_t(w.a.r.first + tok) * p.q_heads + hq] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

__global__ void __launch_bounds__(kCombineThreads) attend_combine_kernel(const AttendParams p, int dim) {
    pdl_launch_dependents();
    // (The lengths may be read ahead of the wait: every CTA of the attention kernel has let this one start after its own
    // wait, so whatever wrote them is over.)
    int per, border, border_end;
    CombineUnit u;
    AttendPlace& w = u.w;
    if (!attend_range(p, int(blockIdx.x) + 1, &per, &border, &border_end, &w) || w.tile == 0) {
        // Nothing to join: the line ends ahead of the border, or the border lies between two units.  One block waits all the
        // same: what follows waits for this grid alone, which must not be over before the attention kernel is.
        if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();
        return;
    }
    const int u0 = border - w.tile, u1 = u0 + w.a.tiles;
    u.c0 = int(uint32_t(u0) / uint32_t(per)), u.c1 = int(uint32_t(u1 - 1) / uint32_t(per));
    u.share = (int(blockIdx.x) - u.c0) * int(gridDim.y) + int(blockIdx.y), u.shares = (u.c1 - u.c0) * int(gridDim.y);
    u.rows = min(p.rows_block, w.a.r.n * p.group - w.block * p.rows_block);
    pdl_wait();
    if (u.c1 - u.c0 + 1 >= kCombineMany) combine_unit<4>(p, u, dim);
    else combine_unit<1>(p, u, dim);
}

int attend_small_bf16(bool, int, int, int*, int*, const AttendParams*, int, cudaStream_t);
int attend_small_e4m3(bool, int, int, int*, int*, const AttendParams*, int, cudaStream_t);
int attend_small_int8(bool, int, int, int*, int*, const AttendParams*, int, cudaStream_t);
static auto attend_small_of(int format) {
    return format == TL_KV_BF16 ? attend_small_bf16 : format == TL_KV_E4M3 ? attend_small_e4m3 : attend_small_int8;
}

int attend_tc_bf16(int, int, const tl_kv_cache*, const AttendParams&, cudaStream_t);
int attend_tc_e4m3(int, int, const tl_kv_cache*, const AttendParams&, cudaStream_t);
int attend_tc_int8(int, int, const tl_kv_cache*, const AttendParams&, cudaStream_t);
static auto attend_tc_of(int format) {
    return format == TL_KV_BF16 ? attend_tc_bf16 : format == TL_KV_E4M3 ? attend_tc_e4m3 : attend_tc_int8;
}

// Which kernel a call runs, from what the host knows: the query rows per key/value head of an average request, and the
// most tiles there can be.  Measured with 64 query and 8 key/value heads over 4100 positions (2000 with 64 requests):
//   few-row kernel or tcgen05, us:   head_dim 128    24 rows: 16 requests bf16 81 / 87, 64 requests INT8 89 / 128,
//                                                    4 requests INT8 34 / 28
//                                                    32 rows: 16 requests bf16 87 / 87, E4M3 77 / 71, 64 requests INT8 144 / 130
//                                    head_dim 64     32 rows: 16 requests bf16 60 / 69, E4M3 48 / 60; one request equal
//                                    (either)        64 rows: 16 requests bf16 146 / 93, E4M3 126 / 77
//   blocks of 128 or 256 rows, us:   256 rows, contexts of half the length to all of it:
//                                    1 request over 4100 (1.8 tiles of 256 rows per SM) bf16 34 / 44, E4M3 36 / 42
//                                    4 over 8000 (10.8) bf16 76 / 79, E4M3 73 / 76; 8 over 2000 (5.6) 65 / 68, 55 / 60
//                                    8 over 3000 (8.3) 76 / 75, 72 / 71; 8 over 4100 (11.2) 91 / 83, 83 / 80
//                                    16 over 2000 (10.9) 116 / 94, 92 / 91; 192 rows, 8 over 8000 (21.6) 124 / 103, 120 / 108
//                                    160 rows, 8 over 8000 E4M3 97 / 108
// Blocks of 256 fetch and convert every tile for two streams at once, but need rows to fill them and more than a few
// tiles per SM to pay for the wider joins.  The lengths are on the device; what the host knows is that they fit the table's rows and,
// pages being one request's alone, the pool: a table as wide as the longest sequence there may ever be says little.
constexpr int kBlockRowsFrom = 192, kBlockTilesFrom = 8;
static int attend_plan(const tl_kv_cache* cache, const tl_kv_batch* batch, int q_heads, AttendPlan* plan) {
    const int group = q_heads / cache->heads;
    const int64_t rows = ceil_div(batch->tokens, batch->requests) * group;
    const int64_t room = std::min(batch->table_stride * cache->page_tokens, kKvMaxTokens);
    int64_t sms = dev().sm_count;
    if (opt(TL_OPT_SM_LIMIT) > 0) sms = std::min(sms, opt(TL_OPT_SM_LIMIT));
    if (cache->head_dim <= 128 && rows > (cache->head_dim == 128 ? 24 : 32)) {
        plan->tile_tokens = 128;
        plan->ctas_per_sm = 1;
        const double positions = std::min(double(batch->requests) * double(room), double(cache->pages) * cache->page_tokens);
        const double tiles256 = cache->heads * double(ceil_div(rows, 256)) * std::ceil(positions / 128);
        plan->mma_rows = rows >= kBlockRowsFrom && tiles256 >= double(kBlockTilesFrom * sms) ? 256 : 128;
    } else {
        plan->mma_rows = rows > 16 && cache->head_dim <= 128 ? 32 : 16;
        if (int rc = attend_small_of(cache->format)(false, cache->head_dim, plan->mma_rows, &plan->tile_tokens, &plan->ctas_per_sm, nullptr, 0, nullptr)) return rc;
    }
    // no more CTAs than there can be tiles (the length is bounded by the page table)
    const int64_t tiles = ceil_div(room, plan->tile_tokens);
    const int64_t units = (ceil_div(int64_t(batch->tokens) * group, plan->mma_rows) + batch->requests) * cache->heads;
    if (double(tiles) * double(units) >= double(INT32_MAX)) return TL_ERR_UNSUPPORTED;
    int64_t ctas = sms * plan->ctas_per_sm;
    if (tiles < ctas && units < ctas) ctas = std::min(ctas, tiles * units);
    plan->ctas = int(ctas);
    const bool split = plan->ctas > 1 && tiles > 1;
    plan->part_bytes = split ? size_t(2) * plan->ctas * plan->mma_rows * cache->head_dim * sizeof(float) : 0;
    plan->ml_bytes = split ? size_t(2) * plan->ctas * plan->mma_rows * sizeof(float2) : 0;
    return TL_OK;
}

static int attend_check(const tl_kv_cache* cache, const tl_kv_batch* batch, int q_heads, AttendParams* p) {
    if (int rc = kv_view(cache, &p->cache)) return rc;
    if (int rc = kv_batch_view(batch, &p->batch)) return rc;
    if (q_heads < 1 || q_heads % cache->heads) return TL_ERR_INVALID_ARG;
    if (int64_t(batch->tokens) * q_heads > INT32_MAX / 2) return TL_ERR_UNSUPPORTED;
    return TL_OK;
}

}  // namespace tl

extern "C" {

size_t tl_tree_attention_workspace_bytes(const tl_kv_cache* cache, const tl_kv_batch* batch, int q_heads) {
    using namespace tl;
    AttendParams p = {};
    if (attend_check(cache, batch, q_heads, &p) || batch->requests == 0 || batch->tokens == 0) return 0;
    ApiLock lock;
    if (ensure_device_info()) return 0;
    AttendPlan plan = {};
    if (attend_plan(cache, batch, q_heads, &plan)) return 0;
    return plan.part_bytes + plan.ml_bytes;
}

int tl_tree_attention(const tl_kv_cache* cache, const tl_kv_batch* batch, const void* d_q, int64_t q_stride, int q_heads,
                      const uint32_t* d_mask, int mask_words, float scale, void* d_out, int64_t out_stride, float* d_lse,
                      void* cuda_stream) {
    using namespace tl;
    AttendParams p = {};
    if (int rc = attend_check(cache, batch, q_heads, &p)) return rc;
    if (d_mask && mask_words < 1) return TL_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return TL_ERR_INVALID_ARG;
    if (batch->requests == 0 || batch->tokens == 0) return TL_OK;
    const int64_t wide = int64_t(q_heads) * cache->head_dim;
    if (!d_q || !d_out || q_stride < wide || out_stride < wide) return TL_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(d_q) % 16 || reinterpret_cast<uintptr_t>(d_out) % 16 || q_stride % 8 || out_stride % 8 ||
        !words_aligned(d_mask, d_lse))
        return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    AttendPlan plan = {};
    if (int rc = attend_plan(cache, batch, q_heads, &plan)) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    void* ws = nullptr;
    if (int rc = get_workspace(plan.part_bytes + plan.ml_bytes, &ws, stream)) return rc;
    p.q = static_cast<const __nv_bfloat16*>(d_q);
    p.out = static_cast<__nv_bfloat16*>(d_out);
    p.lse = d_lse;
    p.mask = d_mask;
    p.mask_words = mask_words;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.group = q_heads / cache->heads;
    p.q_heads = q_heads;
    p.rows_block = plan.mma_rows;
    for (p.rows_shift = 0; (1 << p.rows_shift) < plan.mma_rows; ++p.rows_shift) {}
    for (p.tile_shift = 0; (1 << p.tile_shift) < plan.tile_tokens; ++p.tile_shift) {}
    p.ctas = plan.ctas;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.part = static_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.part_bytes);
    p.status = dev().ctl.d_status;
    if (int rc = plan.mma_rows >= 128
                     ? attend_tc_of(cache->format)(cache->head_dim, plan.mma_rows / 128, cache, p, stream)
                     : attend_small_of(cache->format)(true, cache->head_dim, plan.mma_rows, nullptr, nullptr, &p, plan.ctas, stream))
        return rc;
    if (plan.part_bytes == 0) return TL_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(plan.ctas - 1), unsigned(plan.mma_rows / kCombineRows));
    cfg.blockDim = dim3(kCombineThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = opt(TL_OPT_PDL) != 0 ? 1 : 0;
    return check_cuda(cudaLaunchKernelEx(&cfg, attend_combine_kernel, p, int(cache->head_dim)));
}

}  // extern "C"
