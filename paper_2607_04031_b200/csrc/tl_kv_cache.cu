// The paged key/value cache: quantising rows into it, reading them back, moving accepted rows together.
//
// All three are copies with a conversion on the way: a group of head_dim / 8 lanes owns one head's row of one token (16 bytes
// of bf16 and 8 of codes per lane), so that every access of the group is one contiguous row.  8192 new rows of 8 heads x 128
// appended as INT8 and 27000 read back, both from and to bf16: 46.6 us for 219 MB (4.7 TB/s, 0.72 of a plain copy).  The floor
// is HBM.  Apart and cold: append 20.0 us for 50 MB, latency bound (issue slots 64 %, 44 % of the warps), read 29.4 us for 167 MB (issue
// slots 71 %).
#include "tl_kv_rows.cuh"

#include <algorithm>

namespace tl {

int kv_view(const tl_kv_cache* c, KvView* out) {
    if (!c || !out) return TL_ERR_INVALID_ARG;
    const bool four = c->format == TL_KV_E2M1;
    if ((c->format < TL_KV_BF16 || c->format > TL_KV_INT8) && !four) return TL_ERR_INVALID_ARG;
    if (!c->k || !c->v || c->pages <= 0 || c->heads <= 0 || c->head_dim <= 0 || c->page_tokens <= 0) return TL_ERR_INVALID_ARG;
    if (c->format != TL_KV_BF16 && (!c->k_scale || !c->v_scale)) return TL_ERR_INVALID_ARG;
    if (four && (!c->k_group || !c->v_group)) return TL_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return TL_ERR_UNSUPPORTED;
    if (!is_pow2(c->page_tokens) || c->page_tokens < 16 || c->page_tokens > 1024) return TL_ERR_UNSUPPORTED;
    const int64_t per16 = 256 / kv_bytes(c->format, 16);                    // elements of 16 bytes
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
    if (page % per16 || head % per16 || token % per16) return TL_ERR_ALIGNMENT;
    if (token / per16 * 16 > (int64_t(1) << 26)) return TL_ERR_UNSUPPORTED;      // sixteen tokens' offsets fit 32 bits
    if (reinterpret_cast<uintptr_t>(c->k) % 16 || reinterpret_cast<uintptr_t>(c->v) % 16) return TL_ERR_ALIGNMENT;
    if (c->format != TL_KV_BF16) {
        if (spage % 4 || shead % 4) return TL_ERR_ALIGNMENT;
        if (reinterpret_cast<uintptr_t>(c->k_scale) % 16 || reinterpret_cast<uintptr_t>(c->v_scale) % 16) return TL_ERR_ALIGNMENT;
    }
    int64_t gpage = 0, ghead = 0;
    if (four) {
        gpage = c->group_page_stride, ghead = c->group_head_stride;
        if (gpage == 0 && ghead == 0) {
            ghead = int64_t(c->page_tokens) * (c->head_dim / 16);
            gpage = ghead * c->heads;
        }
        if (gpage <= 0 || ghead <= 0) return TL_ERR_INVALID_ARG;
        if (gpage % 16 || ghead % 16 || reinterpret_cast<uintptr_t>(c->k_group) % 16 || reinterpret_cast<uintptr_t>(c->v_group) % 16)
            return TL_ERR_ALIGNMENT;
    }
    out->group[0] = four ? reinterpret_cast<char*>(c->k_group) : nullptr;
    out->group[1] = four ? reinterpret_cast<char*>(c->v_group) : nullptr;
    out->group_page_stride = gpage;
    out->group_head_stride = ghead;
    out->base[0] = static_cast<char*>(c->k);
    out->base[1] = static_cast<char*>(c->v);
    out->scale[0] = c->format == TL_KV_BF16 ? nullptr : c->k_scale;
    out->scale[1] = c->format == TL_KV_BF16 ? nullptr : c->v_scale;
    out->page_stride = page / per16 * 16;
    out->head_stride = head / per16 * 16;
    out->token_stride = token / per16 * 16;
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

// Address of a position's row in the cache (keys or values), or null when there is no page for it.  extra: 0 the row's scale in
// *scale, n > 0 (kFour) word n - 1 of its group scales in its place.
template <bool kFour>
__device__ __forceinline__ char* kv_row(const KvView& c, const KvBatchView& bv, int b, int pos, int which, int head,
                                        float** scale, int group_words, int extra) {
    if (pos < 0 || pos >= kv_room(bv, c.page_shift)) return nullptr;
    const int64_t page = bv.page_table[int64_t(b) * bv.table_stride + (pos >> c.page_shift)];
    if (page < 0 || page >= c.pages) return nullptr;
    const int line = pos & ((1 << c.page_shift) - 1);
    if (scale && (!kFour || extra <= 0)) *scale = c.scale[which] + page * c.scale_page_stride + int64_t(head) * c.scale_head_stride + line;
    else if (scale) *scale = reinterpret_cast<float*>(c.group[which] + page * c.group_page_stride + int64_t(head) * c.group_head_stride) + line * group_words + extra - 1;
    return c.base[which] + page * c.page_stride + int64_t(head) * c.head_stride + line * c.token_stride;
}

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
        if (!kv_locate_row(p.cache, p.batch, row, kDim / 16, &at)) continue;
        if (!at.page) {
            if (lane_id() == 0) atomicCAS(p.status, 0u, kBadPage);
            continue;
        }
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            const int head = head0 + i * kPerWarp;
            if (head >= heads) continue;                      // (whole groups leave together; no shuffle spans groups)
            float x[8];
            load8(reinterpret_cast<const char*>(&raw[i]), kF32, x);
            if constexpr (kFmt == TL_KV_BF16) store8(p.cache.base[which] + at.at + int64_t(head) * p.cache.head_stride + l * 16, false, x);
            else kv_store_codes<kFmt, kDim>(p.cache, which, at, head, l, sub, x, kF32 ? kv_top_f32(x) : kv_top_bf16(raw[i].v[0]));
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
        if (!kv_locate_row(p.cache, p.batch, row, kDim / 16, &at)) continue;
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

// The same two for 4-bit caches.  A lane owns the 16 elements of a group scale (32 bytes of bf16, 8 of codes), a group of kDim / 16
// lanes a row's head, and a warp several neighbouring rows, whose places are looked up together: with 4 bits a row of 8 heads is
// 512 bytes, too little for a warp to wait for alone.  8192 rows of 8 heads x 128 appended and 26200 read back, from and to bf16: 42 us
// for 187 MB (floor 28.5); one row per warp and eight elements per lane 55 us.  Apart and cold: append 16.6 to 17.8 us for 44 MB, bound by the
// quotients' instructions (issue slots 65 to 69 %), read 29 us for 139 MB, most of them written (issue slots 59 %).
// Heads per warp, append and read together, caches cold: 8 read and 4 appended at a time 50 us, 4 and 4 48, 4 and 2 46, 2 and 2 50.
constexpr int kFourHeads = 4, kFourAppendHeads = 2, kFourReadCtas = 4;

// 32 bytes at once where they are aligned so.
__device__ __forceinline__ void load32(const char* src, bool wide, uint32_t (&v)[8]) {
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(src));
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(src), b = *reinterpret_cast<const uint4*>(src + 16);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}
__device__ __forceinline__ void store32(char* dst, bool wide, const uint32_t (&v)[8]) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "l"(dst) : "memory");
    } else {
        *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<uint4*>(dst + 16) = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// Where the lane's row lies, for rows base + lane / (32 / kRows) of a warp.  False: no request owns it.
template <int kRows>
__device__ __forceinline__ bool kv_locate_rows(const KvView& cache, const KvBatchView& bv, int base, int groups, KvRowPlace* out) {
    const int sub = int(lane_id()) / (32 / kRows), row = base + sub;
    int b = -1, first = 0, start = 0;
    for (int b0 = 0; b0 < bv.requests; b0 += 32) {
        const int mine = min(b0 + int(lane_id()), bv.requests - 1);
        const KvRequest q = kv_request(bv, cache.page_shift, mine);
        uint32_t found = 0;                                   // of the lane's row
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const uint32_t owner = __ballot_sync(0xffffffffu, b0 + int(lane_id()) < bv.requests && base + r >= q.first && base + r < q.first + q.n);
            if (r == sub) found = owner;
        }
        const int l = found ? __ffs(int(found)) - 1 : 0;
        const int f = __shfl_sync(0xffffffffu, q.first, l), st = __shfl_sync(0xffffffffu, q.start, l);
        if (found) b = b0 + l, first = f, start = st;
        if (__all_sync(0xffffffffu, b >= 0)) break;
    }
    out->page = false;
    out->pos = start + (row - first);
    out->at = out->scale_at = out->group_at = 0;
    if (b < 0) return false;
    if (out->pos >= kv_room(bv, cache.page_shift)) return true;
    const int64_t page = bv.page_table[int64_t(b) * bv.table_stride + (out->pos >> cache.page_shift)];
    const int line = out->pos & ((1 << cache.page_shift) - 1);
    out->page = page >= 0 && page < cache.pages;
    if (!out->page) return true;
    out->at = page * cache.page_stride + line * cache.token_stride;
    out->scale_at = page * cache.scale_page_stride + line;
    out->group_at = page * cache.group_page_stride + line * groups;
    return true;
}

template <int kDim, bool kF32>
__global__ void __launch_bounds__(kCopyThreads) kv_four_append_kernel(const KvCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kLanes = kDim / 16, kRows = 32 / kLanes, kItem = kF32 ? 4 : 2, kWords = kF32 ? 2 : 1;
    const int which = int(blockIdx.y) & 1, head0 = int(blockIdx.y >> 1) * kFourAppendHeads, heads = min(p.cache.heads - head0, kFourAppendHeads);
    const int sub = int(lane_id()) / kLanes, l = int(lane_id()) % kLanes;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.rows[which]) | uintptr_t(p.row_stride)) & 31u) == 0;
    const int64_t step = int64_t(gridDim.x) * (kCopyThreads / 32) * kRows;
    for (int64_t base = (blockIdx.x * int64_t(kCopyThreads / 32) + threadIdx.x / 32) * kRows; base < p.batch.tokens; base += step) {
        const int64_t row = base + sub;
        const char* const src = p.rows[which] + (row < p.batch.tokens ? row : base) * p.row_stride + (int64_t(head0) * kDim + l * 16) * kItem;
        uint32_t raw[kFourAppendHeads][kWords][8];
#pragma unroll
        for (int i = 0; i < kFourAppendHeads; ++i)
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (i < heads) load32(src + int64_t(i) * kDim * kItem + w * 32, wide, raw[i][w]);
        KvRowPlace at;
        const bool owned = kv_locate_rows<kRows>(p.cache, p.batch, int(base), kDim / 16, &at) && row < p.batch.tokens;
        if (owned && !at.page && l == 0) atomicCAS(p.status, 0u, kBadPage);
        const bool write = owned && at.page;
#pragma unroll
        for (int i = 0; i < kFourAppendHeads; ++i) {
            if (i >= heads) continue;
            float x[2][8];
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (kF32) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[k][e] = __uint_as_float(raw[i][kF32 ? k : 0][e]);
                    top = max(top, kv_top_f32(x[k]));
                } else {
                    const uint4 v = make_uint4(raw[i][0][4 * k], raw[i][0][4 * k + 1], raw[i][0][4 * k + 2], raw[i][0][4 * k + 3]);
                    load8(reinterpret_cast<const char*>(&v), false, x[k]);
                    top = max(top, kv_top_bf16(v));
                }
            }
            uint32_t row_top = top;
#pragma unroll
            for (int d = kLanes / 2; d > 0; d >>= 1) row_top = max(row_top, __shfl_xor_sync(0xffffffffu, row_top, d));
            const E2m1Row r = e2m1_row(row_top);
            const uint32_t byte = e2m1_group(top, r), lo = e2m1_codes(x[0], byte, r), hi = e2m1_codes(x[1], byte, r);
            if (!write) continue;
            const int64_t head = head0 + i;
            *reinterpret_cast<uint2*>(p.cache.base[which] + at.at + head * p.cache.head_stride + l * 8) = make_uint2(lo, hi);
            p.cache.group[which][at.group_at + head * p.cache.group_head_stride + l] = char(byte);
            if (l == 0) p.cache.scale[which][at.scale_at + head * p.cache.scale_head_stride] = r.scale;
        }
    }
}

// (The next rows' places are looked up while these rows' codes are on their way.)
template <int kDim, bool kF32>
__global__ void __launch_bounds__(kCopyThreads, kFourReadCtas) kv_four_read_kernel(const KvCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kLanes = kDim / 16, kRows = 32 / kLanes, kItem = kF32 ? 4 : 2;
    const int which = int(blockIdx.y) & 1, head0 = int(blockIdx.y >> 1) * kFourHeads, heads = min(p.cache.heads - head0, kFourHeads);
    const int sub = int(lane_id()) / kLanes, l = int(lane_id()) % kLanes;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.rows[which]) | uintptr_t(p.row_stride)) & 31u) == 0;
    const int64_t step = int64_t(gridDim.x) * (kCopyThreads / 32) * kRows;
    int64_t base = (blockIdx.x * int64_t(kCopyThreads / 32) + threadIdx.x / 32) * kRows;
    if (base >= p.batch.tokens) return;
    KvRowPlace at;
    bool owned = kv_locate_rows<kRows>(p.cache, p.batch, int(base), kDim / 16, &at);
    while (true) {
        const int64_t row = base + sub;
        const bool here = owned && row < p.batch.tokens, page = here && at.page;
        if (here && !page && l == 0) atomicCAS(p.status, 0u, kBadPage);
        const char* const codes = p.cache.base[which] + at.at + int64_t(head0) * p.cache.head_stride + l * 8;
        const char* const group = p.cache.group[which] + at.group_at + int64_t(head0) * p.cache.group_head_stride + l;
        const float* const scale = p.cache.scale[which] + at.scale_at + int64_t(head0) * p.cache.scale_head_stride;
        uint2 c[kFourHeads];
        uint32_t g[kFourHeads];
        float s[kFourHeads];
#pragma unroll
        for (int i = 0; i < kFourHeads; ++i) {
            c[i] = make_uint2(0, 0), g[i] = 0, s[i] = 0.0f;
            if (i >= heads || !page) continue;
            c[i] = *reinterpret_cast<const uint2*>(codes + i * p.cache.head_stride);
            g[i] = uint8_t(group[i * p.cache.group_head_stride]);
            s[i] = scale[i * p.cache.scale_head_stride];
        }
        base += step;
        const bool more = base < p.batch.tokens;
        if (more) owned = kv_locate_rows<kRows>(p.cache, p.batch, int(base), kDim / 16, &at);
        char* const dst = p.rows[which] + row * p.row_stride + (int64_t(head0) * kDim + l * 16) * kItem;
#pragma unroll
        for (int i = 0; i < kFourHeads; ++i) {
            if (i >= heads || !here) continue;
            float x[2][8];
            const uint32_t g2 = group_f16x2(g[i], 0, 0, 0);
            KvCodes<TL_KV_E2M1>::expand(c[i].x, g2, s[i], x[0]);
            KvCodes<TL_KV_E2M1>::expand(c[i].y, g2, s[i], x[1]);
            uint32_t v[8];
#pragma unroll
            for (int w = 0; w < (kF32 ? 2 : 1); ++w) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = kF32 ? __float_as_uint(x[w][e]) : pack_bf16(x[e / 4][e % 4 * 2], x[e / 4][e % 4 * 2 + 1]);
                store32(dst + int64_t(i) * kDim * kItem + w * 32, wide, v);
            }
        }
        if (!more) break;
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
    int group_words;            // 4-byte words of its group scales (4-bit caches)
};
constexpr int kCommitThreads = 512;
constexpr int kCommitAhead = 4;

// One CTA per request, so that the new length (which may overwrite batch.start) is written when every thread has read
// the old one.
template <bool kFour>
__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const KvCommitParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int lanes = p.chunks + 1 + (kFour ? p.group_words : 0);           // the extra ones move the scales
    const int b = blockIdx.x;
    const KvRequest r = kv_request(p.batch, p.cache.page_shift, b);
    const int n = int(min(int64_t(min(max(p.n_accepted[b], 0), r.n)), p.accepted_stride));
    const bool has_scales = p.cache.scale[0] != nullptr;
    for (int e = threadIdx.x; e < 2 * p.cache.heads * lanes; e += blockDim.x) {
        const int l = e % lanes, which = e / lanes % 2, head = e / lanes / 2;
        if (l >= p.chunks && !has_scales) continue;
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
                const char* src = kv_row<kFour>(p.cache, p.batch, b, r.start + a, which, head, has_scales ? &s : nullptr, p.group_words, l - p.chunks);
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
                char* dst = kv_row<kFour>(p.cache, p.batch, b, r.start + i0 + k, which, head, has_scales ? &s : nullptr, p.group_words, l - p.chunks);
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

using CopyKernel = void (*)(KvCopyParams);

template <int kFmt, bool kF32>
static CopyKernel pick_copy(bool append, int dim) {
    switch (dim) {
        case 64: return append ? kv_append_kernel<kFmt, 64, kF32> : kv_read_kernel<kFmt, 64, kF32>;
        case 128: return append ? kv_append_kernel<kFmt, 128, kF32> : kv_read_kernel<kFmt, 128, kF32>;
        default: return append ? kv_append_kernel<kFmt, 256, kF32> : kv_read_kernel<kFmt, 256, kF32>;
    }
}

template <bool kF32>
static CopyKernel pick_four(bool append, int dim) {
    switch (dim) {
        case 64: return append ? kv_four_append_kernel<64, kF32> : kv_four_read_kernel<64, kF32>;
        case 128: return append ? kv_four_append_kernel<128, kF32> : kv_four_read_kernel<128, kF32>;
        default: return append ? kv_four_append_kernel<256, kF32> : kv_four_read_kernel<256, kF32>;
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
        case TL_KV_E2M1: kernel = f32 ? pick_four<true>(append, cache->head_dim) : pick_four<false>(append, cache->head_dim); break;
        default: kernel = f32 ? pick_copy<TL_KV_INT8, true>(append, cache->head_dim) : pick_copy<TL_KV_INT8, false>(append, cache->head_dim); break;
    }
    const bool four = cache->format == TL_KV_E2M1;
    const int64_t chunks = four ? ceil_div(cache->heads, append ? kFourAppendHeads : kFourHeads) : ceil_div(cache->heads, int64_t(kCopyAhead) * (32 / (cache->head_dim / 8)));
    if (2 * chunks > 65535) return TL_ERR_UNSUPPORTED;
    const int64_t rows = kCopyThreads / 32 * int64_t(four ? 512 / cache->head_dim : 1);                  // of a block at a time
    const int64_t most = four && !append ? int64_t(dev().sm_count) * kFourReadCtas / (2 * chunks) : int64_t(dev().sm_count) * 16 / chunks;
    const int64_t blocks = std::min<int64_t>(ceil_div(p.batch.tokens, rows), std::max<int64_t>(most, 1));
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
    p.chunks = int(kv_bytes(cache->format, cache->head_dim) / 16);
    p.group_words = cache->format == TL_KV_E2M1 ? cache->head_dim / 64 : 0;
    const int64_t items = int64_t(2) * cache->heads * (p.chunks + 1 + p.group_words);
    const int threads = int(std::min<int64_t>(ceil_div(items, 32) * 32, kCommitThreads));
    return kv_launch(p.group_words ? kv_commit_kernel<true> : kv_commit_kernel<false>, dim3(unsigned(p.batch.requests)), threads, static_cast<cudaStream_t>(cuda_stream), p);
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
