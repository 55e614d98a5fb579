// What the attention kernels share: their parameters and the division of the work.
//
// A unit is (request, key/value head, block of query rows); a row is (token, query head of the group).  A unit's
// sequence is cut into tiles of 2^tile_shift positions; all tiles of all units form one line, in the order request,
// head, row block, tile, and CTA c owns the tiles [c * per, (c + 1) * per) of it.  Lengths live on the device, so every
// CTA works its range out by itself (a warp scan over the requests).  A unit inside one CTA's range is finished there;
// one that crosses a border leaves its parts (unnormalised sums, running maximum and sum of every row) in the
// workspace, two slots per CTA, and the combine kernel behind adds them in the order of the CTAs: no atomics, the same
// bits every time.
#pragma once

#include "tl_kv.cuh"

namespace tl {

struct AttendParams {
    KvView cache;
    KvBatchView batch;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;
    const uint32_t* mask;
    int64_t q_stride, out_stride;        // elements
    int mask_words;
    int group, q_heads;
    int rows_block, rows_shift;          // query rows of a unit, a power of two
    int tile_shift, ctas;                // positions of a tile, a power of two
    float scale_log2;                    // scale * log2(e)
    float* part;                         // [2 * ctas][rows_block][dim]
    float2* part_ml;                     // [2 * ctas][rows_block]: maximum (log2 units) and sum
    uint32_t* status;
};

// A row's weights are taken against a reference that stands for its maximum: a new one is taken when a score exceeds it by more than
// kLag + attend_head (log2), attend_head below the score.  With 8-bit caches the weight (times the value's scale) enters the second product in
// f16: at most 2^15 and, of the largest, 2^7 at least, it has all of f16's exponents, and one that is subnormal is off by 2^-32 of
// the largest.  bf16 has fp32's exponents: the maximum itself.
constexpr float kLag = 8.0f;
__host__ __device__ constexpr float attend_head(int format) { return format == TL_KV_BF16 ? 0.0f : 7.0f; }

// 8-bit caches: the least scale of a value.  Its reciprocal enters the sum of the weights, which has room for 2^22 rows at the floor
// whose weights are all 2^15 (2^30 of 2^7).  Weights of their own for smaller scales (a branch behind the exponentials, one more vote
// of the producers) were measured: 1 to 2 % of every call with an 8-bit cache.
constexpr float kScaleFloor = 0x1p-90f;

#ifdef __CUDACC__

struct AttendRequest {
    KvRequest r;
    int row_blocks;
    int tiles;                           // per unit
};
__device__ __forceinline__ AttendRequest attend_request(const AttendParams& p, int b) {
    AttendRequest a;
    a.r = kv_request(p.batch, p.cache.page_shift, b);
    a.row_blocks = (a.r.n * p.group + p.rows_block - 1) >> p.rows_shift;
    a.tiles = (a.r.len + (1 << p.tile_shift) - 1) >> p.tile_shift;
    return a;
}
__device__ __forceinline__ int attend_per_cta(int total, int ctas) { return int(uint32_t(total + ctas - 1) / uint32_t(ctas)); }

struct AttendPlace {
    int b, head, block;
    int tile;
    AttendRequest a;
};
// Whole warp: the tiles of CTA `cta` are [*x, *x_end) of the line; w: where tile *x lies.  False: there are none.  (The host refuses batches that could have 2^31 tiles or more.)
__device__ __forceinline__ bool attend_range(const AttendParams& p, int cta, int* per_out, int* x, int* x_end, AttendPlace* w) {
    const int lane = int(lane_id());
    // the requests' tiles, 32 at a time; a batch of up to 32 is looked at once, each lane keeping its request
    AttendRequest mine;
    int tiles = 0, total = 0;
    for (int b = lane; b - lane < p.batch.requests; b += 32) {
        tiles = 0;
        if (b < p.batch.requests) {
            mine = attend_request(p, b);
            tiles = mine.tiles * mine.row_blocks * p.cache.heads;
        }
        total += tiles;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    const int per = attend_per_cta(total, p.ctas);
    const int64_t at = int64_t(cta) * per;
    *per_out = per;
    if (at >= total) return false;
    *x = int(at);
    *x_end = *x + min(per, total - *x);
    int before = 0, owner = 0;
    for (int b0 = 0;; b0 += 32) {
        if (p.batch.requests > 32) {
            tiles = 0;
            if (b0 + lane < p.batch.requests) {
                mine = attend_request(p, b0 + lane);
                tiles = mine.tiles * mine.row_blocks * p.cache.heads;
            }
        }
        int run = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, run, d);
            if (lane >= d) run += up;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + run > *x);
        if (past) {
            owner = __ffs(int(past)) - 1;
            w->b = b0 + owner;
            before += __shfl_sync(0xffffffffu, run - tiles, owner);
            break;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
    }
    w->a.r.first = __shfl_sync(0xffffffffu, mine.r.first, owner);
    w->a.r.n = __shfl_sync(0xffffffffu, mine.r.n, owner);
    w->a.r.start = __shfl_sync(0xffffffffu, mine.r.start, owner);
    w->a.r.len = __shfl_sync(0xffffffffu, mine.r.len, owner);
    w->a.row_blocks = __shfl_sync(0xffffffffu, mine.row_blocks, owner);
    w->a.tiles = __shfl_sync(0xffffffffu, mine.tiles, owner);
    const uint32_t y = uint32_t(*x - before), unit = y / uint32_t(w->a.tiles), head = unit / uint32_t(w->a.row_blocks);
    w->tile = int(y - unit * uint32_t(w->a.tiles));
    w->head = int(head);
    w->block = int(unit - head * uint32_t(w->a.row_blocks));
    return true;
}
// The first tile of the next unit; the caller knows that there is one.
__device__ __forceinline__ void attend_next_unit(const AttendParams& p, AttendPlace& w) {
    w.tile = 0;
    if (++w.block < w.a.row_blocks) return;
    w.block = 0;
    if (++w.head < p.cache.heads) return;
    w.head = 0;
    do {
        w.a = attend_request(p, ++w.b);
    } while (w.a.r.n == 0 && w.b + 1 < p.batch.requests);
}

// Whether the row's token (its place `tok` among the request's) sees token j of the step.
__device__ __forceinline__ bool attend_sees(const AttendParams& p, int row_of_token, int tok, int j) {
    if (j < 0) return true;
    if (!p.mask) return j <= tok;
    if ((j >> 5) >= p.mask_words) return false;
    return (p.mask[int64_t(row_of_token) * p.mask_words + (j >> 5)] >> (j & 31)) & 1u;
}

#endif  // __CUDACC__

struct AttendPlan {                      // host
    int mma_rows;                        // query rows of a unit
    int tile_tokens, ctas_per_sm, ctas;
    size_t part_bytes, ml_bytes;
};

}  // namespace tl
