// The paged key/value cache: quantising rows into it, reading them back, moving accepted rows together.
//
// All three are copies with a conversion on the way: a group of head_dim / 8 lanes owns one head's row of one token (16 bytes
// of bf16 and 8 of codes per lane), so that every access of the group is one contiguous row.  8192 new rows of 8 heads x 128
// appended as INT8 and 27000 read back, both from and to bf16: 46.6 us for 219 MB (4.7 TB/s, 0.72 of a plain copy).  The floor
// is HBM.  Apart and cold: append 20.0 us for 50 MB, latency bound (issue slots 64 %, 44 % of the warps), read 29.4 us for 167 MB (issue
// slots 71 %).
#include "tl_kv.cuh"

#include <algorithm>

namespace tl {

int kv_view(const tl_kv_cache* c, KvView* out) {
    if (!c || !out) return TL_ERR_INVALID_ARG;
    if (c->format < TL_KV_BF16 || c->format > TL_KV_INT8) return TL_ERR_INVALID_ARG;
    if (!c->k || !c->v || c->pages <= 0 || c->heads <= 0 || c->head_dim <= 0 || c->page_tokens <= 0) return TL_ERR_INVALID_ARG;
    if (c->format != TL_KV_BF16 && (!c->k_scale || !c->v_scale)) return TL_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return TL_ERR_UNSUPPORTED;
    if (!is_pow2(c->page_tokens) || c->page_tokens < 16 || c->page_tokens > 1024) return TL_ERR_UNSUPPORTED;
    const int64_t s = kv_item(c->format);
    int64_t page = c->page_stride, head = c->head_stride, token = c->token_stride;
    if (page == 0 && head == 0 && token == 0) {
        token = c->head_dim;
        head = token * c->page_tokens;
        page = head * c->heads;
    }
    int64_t spage = c->scale_page_stride, shead = c->scale_head_stride;
    if (spage == 0 && shead == 0) {
        shead = c->page_tokens;
        spage = shead * c->heads;
    }
    // (one head, or one page, makes the stride over it meaningless, but it still has to be a legal one)
    if (page <= 0 || head <= 0 || token < c->head_dim || spage <= 0 || shead <= 0) return TL_ERR_INVALID_ARG;
    if ((page * s) % 16 || (head * s) % 16 || (token * s) % 16) return TL_ERR_ALIGNMENT;
    if (token * s > (int64_t(1) << 26)) return TL_ERR_UNSUPPORTED;      // sixteen tokens' offsets fit 32 bits
    if (reinterpret_cast<uintptr_t>(c->k) % 16 || reinterpret_cast<uintptr_t>(c->v) % 16) return TL_ERR_ALIGNMENT;
    if (c->format != TL_KV_BF16) {
        if (spage % 4 || shead % 4) return TL_ERR_ALIGNMENT;
        if (reinterpret_cast<uintptr_t>(c->k_scale) % 16 || reinterpret_cast<uintptr_t>(c->v_scale) % 16) return TL_ERR_ALIGNMENT;
    }
    out->base[0] = static_cast<char*>(c->k);
    out->base[1] = static_cast<char*>(c->v);
    out->scale[0] = c->format == TL_KV_BF16 ? nullptr : c->k_scale;
    out->scale[1] = c->format == TL_KV_BF16 ? nullptr : c->v_scale;
    out->page_stride = page * s;
    out->head_stride = head * s;
    out->token_stride = token * s;
    out->scale_page_stride = spage;
    out->scale_head_stride = shead;
    out->pages = c->pages;
    out->heads = c->heads;
    out->page_shift = 0;
    while ((1 << out->page_shift) < c->page_tokens) ++out->page_shift;
    return TL_OK;
}

int kv_batch_view(const tl_kv_batch* b, KvBatchView* out) {
    if (!b || !out || b->requests < 0 || b->tokens < 0) return TL_ERR_INVALID_ARG;
    if (b->requests > 0 && (!b->page_table || !b->start || !b->token_offsets || b->table_stride < 1)) return TL_ERR_INVALID_ARG;
    if (b->table_stride > (int64_t(1) << 40)) return TL_ERR_INVALID_ARG;
    if (!words_aligned(b->page_table, b->start, b->token_offsets)) return TL_ERR_ALIGNMENT;
    out->page_table = b->page_table;
    out->start = b->start;
    out->offsets = b->token_offsets;
    out->table_stride = b->table_stride;
    out->requests = b->requests;
    out->tokens = b->tokens;
    return TL_OK;
}

struct KvCopyParams {
    KvView cache;
    KvBatchView batch;
    char* rows[2];              // the step's keys and values
    int64_t row_stride;         // bytes
    uint32_t* status;
};

// The request that owns `row`: the last one whose first row is not behind it.  Called by a whole warp with one row;
// requests are looked at 32 at a time.  (Offsets do not decrease, so the count of offsets <= row names it; an empty
// request in front of the owner is passed over because its end is <= row too.)
__device__ __forceinline__ int warp_request_of(const KvBatchView& bv, int row) {
    int count = 0;
    for (int b0 = 0; b0 < bv.requests; b0 += 32) {
        const int b = b0 + int(lane_id());
        const bool before = b < bv.requests && bv.offsets[b + 1] <= row;
        const int n = __popc(__ballot_sync(0xffffffffu, before));
        count += n;
        if (n < 32) break;
    }
    return count;
}

// Address of a position's row in the cache (keys or values), or null when there is no page for it.
__device__ __forceinline__ char* kv_row(const KvView& c, const KvBatchView& bv, int b, int pos, int which, int head,
                                        float** scale) {
    if (pos < 0 || pos >= kv_room(bv, c.page_shift)) return nullptr;
    const int64_t page = bv.page_table[int64_t(b) * bv.table_stride + (pos >> c.page_shift)];
    if (page < 0 || page >= c.pages) return nullptr;
    const int line = pos & ((1 << c.page_shift) - 1);
    if (scale) *scale = c.scale[which] + page * c.scale_page_stride + int64_t(head) * c.scale_head_stride + line;
    return c.base[which] + page * c.page_stride + int64_t(head) * c.head_stride + line * c.token_stride;
}

__device__ __forceinline__ void load8(const char* src, bool f32, float (&x)[8]) {
    if (f32) {
        const float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 16);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(src);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ void store8(char* dst, bool f32, const float (&x)[8]) {
    if (f32) {
        *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(dst + 16) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
}

// A warp takes one row's keys or values, up to kCopyAhead groups of heads at a time: one look at the request and the page
// table, then all the loads of the group are in flight before the first is used.  (One vector per lane and turn read a
// context of 22000 tokens, 8 heads, INT8 to bf16 at 2.1 TB/s, the loads of a warp waiting one by one.)
constexpr int kCopyThreads = 256, kCopyAhead = 4;

// Where the warp's row lies in the cache (offsets of head 0, the same for keys and values); false when no request owns the
// row.
struct KvRowPlace {
    bool page;                  // there is one
    int64_t at, scale_at;       // bytes, floats
};
__device__ __forceinline__ bool kv_locate_row(const KvCopyParams& p, int row, KvRowPlace* out) {
    // the request that owns the row, looked for 32 at a time; each lane has its request's data at hand (a look at them once
    // the owner is known would be one more round trip)
    const KvBatchView& bv = p.batch;
    KvRequest r = {};
    int b = bv.requests;
    for (int b0 = 0; b0 < bv.requests; b0 += 32) {
        const int mine = min(b0 + int(lane_id()), bv.requests - 1);
        const KvRequest q = kv_request(bv, p.cache.page_shift, mine);
        const uint32_t owner = __ballot_sync(0xffffffffu, b0 + int(lane_id()) < bv.requests && row >= q.first && row < q.first + q.n);
        if (owner) {
            const int l = __ffs(int(owner)) - 1;
            b = b0 + l;
            r.first = __shfl_sync(0xffffffffu, q.first, l);
            r.start = __shfl_sync(0xffffffffu, q.start, l);
            break;
        }
    }
    if (b >= bv.requests) return false;
    const int pos = r.start + (row - r.first);
    out->page = false;
    out->at = out->scale_at = 0;
    if (pos >= kv_room(p.batch, p.cache.page_shift)) return true;
    const int64_t page = p.batch.page_table[int64_t(b) * p.batch.table_stride + (pos >> p.cache.page_shift)];
    const int line = pos & ((1 << p.cache.page_shift) - 1);
    out->page = page >= 0 && page < p.cache.pages;
    if (!out->page) return true;
    out->at = page * p.cache.page_stride + line * p.cache.token_stride;
    out->scale_at = page * p.cache.scale_page_stride + line;
    return true;
}

// Eight codes of a lane and the values they stand for.
template <int kFmt>
struct KvCodes {
    using type = uint2;
    __device__ static void expand(uint2 c, float s, float (&x)[8]) {
        uint32_t h[4];
        codes4_to_f16<kFmt>(c.x, h[0], h[1]);
        codes4_to_f16<kFmt>(c.y, h[2], h[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
            x[2 * e] = f.x * s;
            x[2 * e + 1] = f.y * s;
        }
    }
};
template <>
struct KvCodes<TL_KV_BF16> {
    using type = uint4;
    __device__ static void expand(uint4 c, float, float (&x)[8]) {
        const uint32_t u[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(u[e] << 16);
            x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
        }
    }
};

template <int kFmt, int kDim, bool kF32>
__global__ void __launch_bounds__(kCopyThreads) kv_append_kernel(const KvCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kLanes = kDim / 8, kPerWarp = 32 / kLanes, kItem = kF32 ? 4 : 2;
    const int heads = p.cache.heads, which = int(blockIdx.y) & 1;
    const int sub = int(lane_id()) / kLanes, l = int(lane_id()) % kLanes, head0 = int(blockIdx.y >> 1) * kPerWarp * kCopyAhead + sub;
    const int64_t step = int64_t(gridDim.x) * (kCopyThreads / 32);
    for (int64_t at_row = blockIdx.x * int64_t(kCopyThreads / 32) + threadIdx.x / 32; at_row < p.batch.tokens; at_row += step) {
        const int row = int(at_row);
        // (as they come: 16 or 32 bytes of a head's row)
        struct Raw { uint4 v[kF32 ? 2 : 1]; } raw[kCopyAhead];
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i)
            if (head0 + i * kPerWarp < heads)
                raw[i] = *reinterpret_cast<const Raw*>(p.rows[which] + int64_t(row) * p.row_stride + (int64_t(head0 + i * kPerWarp) * kDim + l * 8) * kItem);
        KvRowPlace at;
        if (!kv_locate_row(p, row, &at)) continue;
        if (!at.page) {
            if (lane_id() == 0) atomicCAS(p.status, 0u, kBadPage);
            continue;
        }
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            const int head = head0 + i * kPerWarp;
            if (head >= heads) continue;                      // (whole groups leave together; no shuffle spans groups)
            char* const dst = p.cache.base[which] + at.at + int64_t(head) * p.cache.head_stride;
            float x[8];
            load8(reinterpret_cast<const char*>(&raw[i]), kF32, x);
            if (kFmt == TL_KV_BF16) {
                store8(dst + l * 16, false, x);
                continue;
            }
            // the largest magnitude, as bits: a NaN's pattern is above an infinity's, so either makes the scale NaN
            uint32_t top = 0;
            if (kF32) {
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            } else {
                const uint32_t u[4] = {raw[i].v[0].x, raw[i].v[0].y, raw[i].v[0].z, raw[i].v[0].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) top = __vmaxu2(top, u[e] & 0x7fff7fffu);          // two bf16 patterns at a time
                top = max(top & 0xffff0000u, top << 16);
            }
            const uint32_t group = (kLanes == 32 ? 0xffffffffu : ((1u << kLanes) - 1u) << (sub * kLanes));
#pragma unroll
            for (int d = kLanes / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(group, top, d));
            constexpr float kTop = kFmt == TL_KV_E4M3 ? 448.0f : 127.0f;
            const bool finite = top < 0x7f800000u;
            const float s = finite ? __fmul_rn(__uint_as_float(top), 1.0f / kTop) : __uint_as_float(0x7fc00000u);
            uint32_t lo = 0, hi = 0;
            if (finite && s > 0.0f) {
                float y[8];
                if (s > 0x1p-90f && s < 0x1p90f) {
                    // x / s with the row's reciprocal: given the correctly rounded 1 / s, one FMA correction of x * (1 / s) is
                    // the correctly rounded quotient (Markstein 1990).  The remainder must not underflow: it is at least
                    // 2^-35 s where the quotient is 2^-11 or more, and below that any quotient rounds to code 0.
                    const float inv = __frcp_rn(s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float q = __fmul_rn(x[e], inv);
                        y[e] = __fmaf_rn(__fmaf_rn(-q, s, x[e]), inv, q);
                    }
                } else {
                    // (a subnormal scale is rounded to a few bits, down to two thirds of top * c: the quotient is clamped)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(__fdiv_rn(x[e], s), -kTop), kTop);
                }
                if (kFmt == TL_KV_E4M3) {
                    // (the saturating conversion keeps the last bit of a quotient just above 448)
                    auto two = [](float a, float c) -> uint32_t {
                        uint16_t q;
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(c), "f"(a));
                        return q;
                    };
                    lo = two(y[0], y[1]) | two(y[2], y[3]) << 16;
                    hi = two(y[4], y[5]) | two(y[6], y[7]) << 16;
                } else {
                    // |y| <= 127 (1 + 2^-22) where the scale is normal, so rounding needs no clamp; 1.5 x 2^23 leaves the integer in
                    // the low bits
                    uint32_t z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = __float_as_uint(__fadd_rn(y[e], 12582912.0f));
                    lo = __byte_perm(__byte_perm(z[0], z[1], 0x0040), __byte_perm(z[2], z[3], 0x0040), 0x5410);
                    hi = __byte_perm(__byte_perm(z[4], z[5], 0x0040), __byte_perm(z[6], z[7], 0x0040), 0x5410);
                }
            }
            *reinterpret_cast<uint2*>(dst + l * 8) = make_uint2(lo, hi);
            if (l == 0) p.cache.scale[which][at.scale_at + int64_t(head) * p.cache.scale_head_stride] = s;
        }
    }
}

template <int kFmt, int kDim, bool kF32>
__global__ void __launch_bounds__(kCopyThreads) kv_read_kernel(const KvCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kLanes = kDim / 8, kPerWarp = 32 / kLanes, kItem = kF32 ? 4 : 2;
    const int heads = p.cache.heads, which = int(blockIdx.y) & 1;
    const int sub = int(lane_id()) / kLanes, l = int(lane_id()) % kLanes, head0 = int(blockIdx.y >> 1) * kPerWarp * kCopyAhead + sub;
    const int64_t step = int64_t(gridDim.x) * (kCopyThreads / 32);
    for (int64_t at_row = blockIdx.x * int64_t(kCopyThreads / 32) + threadIdx.x / 32; at_row < p.batch.tokens; at_row += step) {
        const int row = int(at_row);
        KvRowPlace at;
        if (!kv_locate_row(p, row, &at)) continue;
        if (!at.page && lane_id() == 0) atomicCAS(p.status, 0u, kBadPage);
        using Codes = typename KvCodes<kFmt>::type;
        Codes c[kCopyAhead];
        float s[kCopyAhead];
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            const int head = head0 + i * kPerWarp;
            c[i] = Codes{};
            s[i] = 0.0f;
            if (head >= heads || !at.page) continue;
            c[i] = *reinterpret_cast<const Codes*>(p.cache.base[which] + at.at + int64_t(head) * p.cache.head_stride + l * int(sizeof(Codes)));
            if (kFmt != TL_KV_BF16) s[i] = p.cache.scale[which][at.scale_at + int64_t(head) * p.cache.scale_head_stride];
        }
        char* const dst = p.rows[which] + int64_t(row) * p.row_stride + (int64_t(head0) * kDim + l * 8) * kItem;
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            if (head0 + i * kPerWarp >= heads) continue;
            float x[8];
            KvCodes<kFmt>::expand(c[i], s[i], x);
            store8(dst + int64_t(i) * kPerWarp * kDim * kItem, kF32, x);
        }
    }
}

// One group of threads per (request, keys or values, head); thread l owns the same 16 bytes of every row and walks the
// accepted list upwards.  The source of entry i is at or behind i, so a row that is overwritten has been read in an
// earlier step, by the same thread.
struct KvCommitParams {
    KvView cache;
    KvBatchView batch;
    const int32_t* accepted;
    const int32_t* n_accepted;
    int32_t* new_start;
    int64_t accepted_stride;
    uint32_t* status;
    int chunks;                 // 16-byte pieces of a row
};
constexpr int kCommitThreads = 512;
constexpr int kCommitAhead = 4;

// One CTA per request, so that the new length (which may overwrite batch.start) is written when every thread has read
// the old one.
__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const KvCommitParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int lanes = p.chunks + 1;                           // the extra one moves the scales
    const int b = blockIdx.x;
    const KvRequest r = kv_request(p.batch, p.cache.page_shift, b);
    const int n = int(min(int64_t(min(max(p.n_accepted[b], 0), r.n)), p.accepted_stride));
    const bool has_scales = p.cache.scale[0] != nullptr;
    for (int e = threadIdx.x; e < 2 * p.cache.heads * lanes; e += blockDim.x) {
        const int l = e % lanes, which = e / lanes % 2, head = e / lanes / 2;
        if (l == p.chunks && !has_scales) continue;
        for (int i0 = 0; i0 < n; i0 += kCommitAhead) {
            uint4 row[kCommitAhead];
            float scale[kCommitAhead];
            bool have[kCommitAhead];
#pragma unroll
            for (int k = 0; k < kCommitAhead; ++k) {
                const int i = i0 + k;
                have[k] = false;
                if (i >= n) continue;
                const int a = p.accepted[int64_t(b) * p.accepted_stride + i];
                if (a < i || a >= r.n) {
                    atomicCAS(p.status, 0u, kBadAccepted);
                    continue;
                }
                if (a == i) continue;                         // it is there already
                float* s = nullptr;
                const char* src = kv_row(p.cache, p.batch, b, r.start + a, which, head, has_scales ? &s : nullptr);
                if (!src) {
                    atomicCAS(p.status, 0u, kBadPage);
                    continue;
                }
                have[k] = true;
                if (l < p.chunks) row[k] = *reinterpret_cast<const uint4*>(src + l * 16);
                else scale[k] = *s;
            }
#pragma unroll
            for (int k = 0; k < kCommitAhead; ++k) {
                if (!have[k]) continue;
                float* s = nullptr;
                char* dst = kv_row(p.cache, p.batch, b, r.start + i0 + k, which, head, has_scales ? &s : nullptr);
                if (!dst) continue;                           // a page in front of one that exists: reported by the writer
                if (l < p.chunks) *reinterpret_cast<uint4*>(dst + l * 16) = row[k];
                else *s = scale[k];
            }
        }
    }
    if (p.new_start) {
        __syncthreads();
        if (threadIdx.x == 0) p.new_start[b] = int32_t(r.start + n);
    }
}

// Row i's mask: it climbs from i to the root.  Parents lie strictly below, so the climb ends.
__global__ void tree_mask_kernel(const int32_t* parents, const int32_t* offsets, int requests, int tokens, uint32_t* mask,
                                 int words) {
    pdl_wait();
    pdl_launch_dependents();
    KvBatchView bv = {};
    bv.offsets = offsets;
    bv.requests = requests;
    bv.tokens = tokens;
    const int row = blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    if (row >= tokens) return;
    const int b = warp_request_of(bv, row);
    const int first = b < requests ? min(max(offsets[b], 0), tokens) : row;
    for (int w = int(lane_id()); w < words; w += 32) {
        uint32_t bits = 0;
        int i = b < requests && row >= first ? row - first : -1;
        while (i >= 0) {
            if ((i >> 5) == w) bits |= 1u << (i & 31);
            if ((i >> 5) < w) break;                          // ancestors only get smaller
            const int up = parents[first + i];
            i = up < i ? up : -1;
        }
        mask[int64_t(row) * words + w] = bits;
    }
}

template <typename K, typename... Args>
static int kv_launch(K kernel, dim3 grid, int threads, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = opt(TL_OPT_PDL) != 0 ? 1 : 0;
    return check_cuda(cudaLaunchKernelEx(&cfg, kernel, args...));
}

using CopyKernel = void (*)(KvCopyParams);

template <int kFmt, bool kF32>
static CopyKernel pick_copy(bool append, int dim) {
    switch (dim) {
        case 64: return append ? kv_append_kernel<kFmt, 64, kF32> : kv_read_kernel<kFmt, 64, kF32>;
        case 128: return append ? kv_append_kernel<kFmt, 128, kF32> : kv_read_kernel<kFmt, 128, kF32>;
        default: return append ? kv_append_kernel<kFmt, 256, kF32> : kv_read_kernel<kFmt, 256, kF32>;
    }
}

static int kv_copy(bool append, const tl_kv_cache* cache, const tl_kv_batch* batch, const void* k, const void* v, int elem,
                   int64_t row_stride, void* cuda_stream) {
    KvCopyParams p = {};
    if (int rc = kv_view(cache, &p.cache)) return rc;
    if (int rc = kv_batch_view(batch, &p.batch)) return rc;
    if (elem != TL_ELEM_BF16 && elem != TL_ELEM_F32) return TL_ERR_INVALID_ARG;
    if (p.batch.tokens == 0 || p.batch.requests == 0) return TL_OK;
    if (!k || !v || row_stride < int64_t(cache->heads) * cache->head_dim) return TL_ERR_INVALID_ARG;
    const int64_t item = elem == TL_ELEM_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(k) % 16 || reinterpret_cast<uintptr_t>(v) % 16 || (row_stride * item) % 16) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    p.rows[0] = static_cast<char*>(const_cast<void*>(k));
    p.rows[1] = static_cast<char*>(const_cast<void*>(v));
    p.row_stride = row_stride * item;
    p.status = dev().ctl.d_status;
    const bool f32 = elem == TL_ELEM_F32;
    CopyKernel kernel = nullptr;
    switch (cache->format) {
        case TL_KV_BF16: kernel = f32 ? pick_copy<TL_KV_BF16, true>(append, cache->head_dim) : pick_copy<TL_KV_BF16, false>(append, cache->head_dim); break;
        case TL_KV_E4M3: kernel = f32 ? pick_copy<TL_KV_E4M3, true>(append, cache->head_dim) : pick_copy<TL_KV_E4M3, false>(append, cache->head_dim); break;
        default: kernel = f32 ? pick_copy<TL_KV_INT8, true>(append, cache->head_dim) : pick_copy<TL_KV_INT8, false>(append, cache->head_dim); break;
    }
    const int64_t chunks = ceil_div(cache->heads, int64_t(kCopyAhead) * (32 / (cache->head_dim / 8)));
    if (2 * chunks > 65535) return TL_ERR_UNSUPPORTED;
    const int64_t blocks = std::min<int64_t>(ceil_div(p.batch.tokens, kCopyThreads / 32), std::max<int64_t>(int64_t(dev().sm_count) * 16 / chunks, 1));
    return kv_launch(kernel, dim3(unsigned(blocks), unsigned(2 * chunks)), kCopyThreads, static_cast<cudaStream_t>(cuda_stream), p);
}

}  // namespace tl

extern "C" {

int tl_kv_append(const tl_kv_cache* cache, const tl_kv_batch* batch, const void* d_k, const void* d_v, int elem,
                 int64_t row_stride, void* cuda_stream) {
    return tl::kv_copy(true, cache, batch, d_k, d_v, elem, row_stride, cuda_stream);
}

int tl_kv_read(const tl_kv_cache* cache, const tl_kv_batch* batch, void* d_k, void* d_v, int elem, int64_t row_stride,
               void* cuda_stream) {
    return tl::kv_copy(false, cache, batch, d_k, d_v, elem, row_stride, cuda_stream);
}

int tl_kv_commit(const tl_kv_cache* cache, const tl_kv_batch* batch, const int32_t* d_accepted, int64_t accepted_stride,
                 const int32_t* d_n_accepted, int32_t* d_new_start, void* cuda_stream) {
    using namespace tl;
    KvCommitParams p = {};
    if (int rc = kv_view(cache, &p.cache)) return rc;
    if (int rc = kv_batch_view(batch, &p.batch)) return rc;
    if (p.batch.requests == 0) return TL_OK;
    if (!d_accepted || !d_n_accepted || accepted_stride < 1) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_accepted, d_n_accepted, d_new_start)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    p.accepted = d_accepted;
    p.n_accepted = d_n_accepted;
    p.new_start = d_new_start;
    p.accepted_stride = accepted_stride;
    p.status = dev().ctl.d_status;
    p.chunks = cache->head_dim * kv_item(cache->format) / 16;
    const int64_t items = int64_t(2) * cache->heads * (p.chunks + 1);
    const int threads = int(std::min<int64_t>(ceil_div(items, 32) * 32, kCommitThreads));
    return kv_launch(kv_commit_kernel, dim3(unsigned(p.batch.requests)), threads, static_cast<cudaStream_t>(cuda_stream), p);
}

int tl_tree_mask(const int32_t* d_parents, const int32_t* d_token_offsets, int requests, int tokens, uint32_t* d_mask,
                 int mask_words, void* cuda_stream) {
    using namespace tl;
    if (requests < 0 || tokens < 0 || mask_words < 1) return TL_ERR_INVALID_ARG;
    if (requests == 0 || tokens == 0) return TL_OK;
    if (!d_parents || !d_token_offsets || !d_mask) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_parents, d_token_offsets, d_mask)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    return kv_launch(tree_mask_kernel, dim3(unsigned(ceil_div(tokens, 8))), 256, static_cast<cudaStream_t>(cuda_stream),
                     d_parents, d_token_offsets, requests, tokens, d_mask, mask_words);
}

}  // extern "C"
