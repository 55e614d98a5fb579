// Rotary positions: turning rows (tl_rope_rows), and a step's queries, keys and values on their way into attention and the cache
// (tl_rope_append).
//
// Angles.  A pair's frequency is kept as the 64-bit fraction of a turn it makes per position, so the angle of position t is the
// integer product t * turns modulo 2^64: no error but the frequency's own last bit, at any distance.  The two top bits (rounded) are
// the quadrant, the rest, at most an eighth of a turn either way, goes through sincospi in fp32.
#include "tl_kv_rows.cuh"

#include <algorithm>
#include <cmath>

namespace tl {

struct RopeView {
    const uint64_t* turns;
    float amplitude;
    int rot, interleaved;
};

__device__ __forceinline__ void rope_angle(uint64_t turns, int position, float amplitude, float* c, float* s) {
    const uint64_t phase = turns * uint64_t(int64_t(position));
    const uint32_t quadrant = uint32_t((phase + (uint64_t(1) << 61)) >> 62) & 3u;
    const int32_t rest = int32_t((phase - (uint64_t(quadrant) << 62)) >> 30);               // [-2^31, 2^31): 2^-33 of a half turn
    float sn, cs;
    sincospif(__int2float_rn(rest) * 0x1p-33f, &sn, &cs);
    const float a = quadrant & 1u ? sn : cs, b = quadrant & 1u ? cs : sn;
    *c = (quadrant == 1u || quadrant == 2u ? -a : a) * amplitude;
    *s = (quadrant >= 2u ? -b : b) * amplitude;
}

struct RopeRowsParams {
    RopeView rope;
    const char* x;
    char* out;
    int64_t x_stride, out_stride;        // bytes
    const int32_t* positions;
    int tokens, heads, dim, inverse;
    int heads_per_warp;
};
constexpr int kRopeThreads = 256;

// A warp turns rows of one token.  An item is what a thread holds at once: two vectors of eight elements that are eight pairs
// (pairs v * 8 .. + 7: one vector from each half of the turned part, or two neighbouring ones), or one vector of the elements that
// stay.  The items of a head lie on neighbouring lanes, so a lane works out its eight angles once for all the heads it sees.
// 8192 tokens x 72 heads x 128, bf16: 54 us for 302 MB (floor 46), HBM.  Angles through shared memory, worked out once per CTA, took
// 76 to 111 us (60 here by the same clock, cold); polynomials in place of sincospi changed nothing: the angles are not what a warp waits for.  Small
// calls are latency: 1501 tokens x 20 heads of 80 in fp32 8.2 us, floor 2.9.
template <bool kF32>
__global__ void __launch_bounds__(kRopeThreads, kF32 ? 3 : 4) rope_rows_kernel(const RopeRowsParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kItem = kF32 ? 4 : 2;
    const int pair_items = p.rope.rot / 16, items = pair_items + (p.out == p.x ? 0 : (p.dim - p.rope.rot) / 8);
    const int chunks = (p.heads + p.heads_per_warp - 1) / p.heads_per_warp;
    const int64_t warp = (blockIdx.x * int64_t(kRopeThreads) + threadIdx.x) / 32;
    const int64_t token = warp / chunks;
    if (token >= p.tokens) return;
    const int h0 = int(warp % chunks) * p.heads_per_warp, h1 = min(p.heads, h0 + p.heads_per_warp);
    const int position = p.positions[token];
    const int lane = int(lane_id());
    // lanes beside one another: items of one head, then the next head's
    const int lanes = items < 32 ? items : 32, side = 32 / lanes;
    if (lane >= lanes * side) return;
    const char* const x_row = p.x + token * p.x_stride;
    char* const out_row = p.out + token * p.out_stride;
    for (int item = lane % lanes; item < items; item += lanes) {
        if (item < pair_items) {
            const int a_at = (p.rope.interleaved ? item * 16 : item * 8) * kItem;
            const int b_at = (p.rope.interleaved ? item * 16 + 8 : p.rope.rot / 2 + item * 8) * kItem;
            // (a head's vectors are asked for ahead of the angles, or of the use of the last head's)
            struct Raw { uint4 v[kF32 ? 2 : 1]; } a_raw, b_raw, a_next = {}, b_next = {};
            auto fetch = [&](int h) {
                if (h >= h1) return;
                const char* const src = x_row + int64_t(h) * p.dim * kItem;
                a_next = *reinterpret_cast<const Raw*>(src + a_at);
                b_next = *reinterpret_cast<const Raw*>(src + b_at);
            };
            int h = h0 + lane / lanes;
            fetch(h);
            float c[8], s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                rope_angle(__ldg(p.rope.turns + item * 8 + e), position, p.rope.amplitude, &c[e], &s[e]);
                if (p.inverse) s[e] = -s[e];
            }
            for (; h < h1; h += side) {
                a_raw = a_next, b_raw = b_next;
                fetch(h + side);
                float a[8], b[8], u[8], v[8];
                const int64_t at = int64_t(h) * p.dim * kItem;
                load8(reinterpret_cast<const char*>(&a_raw), kF32, a);
                load8(reinterpret_cast<const char*>(&b_raw), kF32, b);
                if (p.rope.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        u[2 * e] = fmaf(a[2 * e], c[e], -(a[2 * e + 1] * s[e]));
                        u[2 * e + 1] = fmaf(a[2 * e + 1], c[e], a[2 * e] * s[e]);
                        v[2 * e] = fmaf(b[2 * e], c[4 + e], -(b[2 * e + 1] * s[4 + e]));
                        v[2 * e + 1] = fmaf(b[2 * e + 1], c[4 + e], b[2 * e] * s[4 + e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        u[e] = fmaf(a[e], c[e], -(b[e] * s[e]));
                        v[e] = fmaf(b[e], c[e], a[e] * s[e]);
                    }
                }
                store8(out_row + at + a_at, kF32, u);
                store8(out_row + at + b_at, kF32, v);
            }
        } else {
            const int at = (p.rope.rot + (item - pair_items) * 8) * kItem;
            for (int h = h0 + lane / lanes; h < h1; h += side) {
                float a[8];
                load8(x_row + int64_t(h) * p.dim * kItem + at, kF32, a);
                store8(out_row + int64_t(h) * p.dim * kItem + at, kF32, a);
            }
        }
    }
}

// Any even sizes, by elements: a thread owns a pair, or an element that stays, of one token and takes heads in turn.
// 8192 tokens x 72 heads of 128, bf16, 36 dimensions turned 210 us, 100 turned 194 (either layout; floor 46), fp32 with 36 280 (floor 92);
// 72 heads of 90 91 (32); 32 tokens of 72 heads 2.9.  Accesses of 2 and 4 bytes bound it: 2.5 times the vectors' warp instructions, 211 MB
// read and 136 written in 206 us, issue slots 27 % with 73 % of the warps.
template <bool kF32>
__global__ void __launch_bounds__(kRopeThreads) rope_rows_any_kernel(const RopeRowsParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int pairs = p.rope.rot / 2, items = pairs + (p.out == p.x ? 0 : p.dim - p.rope.rot);
    const int64_t at = blockIdx.x * int64_t(kRopeThreads) + threadIdx.x;
    const int64_t token = at / items;
    const int item = int(at % items);
    if (token >= p.tokens) return;
    auto get = [&](int64_t e) -> float {
        if (kF32) return reinterpret_cast<const float*>(p.x + token * p.x_stride)[e];
        return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.x + token * p.x_stride)[e]);
    };
    auto put = [&](int64_t e, float v) {
        if (kF32) reinterpret_cast<float*>(p.out + token * p.out_stride)[e] = v;
        else reinterpret_cast<__nv_bfloat16*>(p.out + token * p.out_stride)[e] = __float2bfloat16_rn(v);
    };
    const int h0 = int(blockIdx.y) * p.heads_per_warp, h1 = min(p.heads, h0 + p.heads_per_warp);
    if (item < pairs) {
        float c, s;
        rope_angle(p.rope.turns[item], p.positions[token], p.rope.amplitude, &c, &s);
        if (p.inverse) s = -s;
        const int i = p.rope.interleaved ? 2 * item : item, j = p.rope.interleaved ? i + 1 : i + pairs;
        for (int h = h0; h < h1; ++h) {
            const float a = get(int64_t(h) * p.dim + i), b = get(int64_t(h) * p.dim + j);
            put(int64_t(h) * p.dim + i, fmaf(a, c, -(b * s)));
            put(int64_t(h) * p.dim + j, fmaf(b, c, a * s));
        }
    } else {
        const int i = p.rope.rot + item - pairs;
        for (int h = h0; h < h1; ++h) put(int64_t(h) * p.dim + i, get(int64_t(h) * p.dim + i));
    }
}

struct RopeAppendParams {
    KvView cache;
    KvBatchView batch;
    RopeView rope;
    const int32_t* positions;
    const char* q;
    __nv_bfloat16* q_out;
    const char* rows[2];                 // keys, values
    int64_t q_stride, q_out_stride, row_stride;      // bytes
    uint32_t* status;
    int q_heads;
    int q_chunks, kv_chunks;             // of head groups, per row
};

// A lane's eight elements of a row turned: its own, and those they are paired with (in TL_ROPE_HALF other lanes' elements, which it
// reads again).  The angles are the lane's for every head.
struct RopeLane {
    float c[8], s[8];                    // s with the sign that the partner's term has; elements that stay: 1 and 0
    bool turned;
};
__device__ __forceinline__ void rope_lane(const RopeView& r, int d0, int position, RopeLane* out) {
    const int half = r.rot / 2;
    out->turned = d0 < r.rot;
#pragma unroll
    for (int e = 0; e < 8; ++e) out->c[e] = 1.0f, out->s[e] = 0.0f;
    if (!out->turned) return;
    if (r.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if (d0 + e >= r.rot) break;
            float c, s;
            rope_angle(__ldg(r.turns + (d0 + e) / 2), position, r.amplitude, &c, &s);
            out->c[e] = out->c[e + 1] = c;
            out->s[e] = -s, out->s[e + 1] = s;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = d0 + e;
        if (d >= r.rot) break;
        float c, s;
        rope_angle(__ldg(r.turns + (d < half ? d : d - half)), position, r.amplitude, &c, &s);
        out->c[e] = c;
        out->s[e] = d < half ? -s : s;
    }
}
// The partners of elements d0 .. d0 + 7 of the head's row at `row`.
template <bool kF32>
__device__ __forceinline__ void rope_partners(const RopeView& r, const char* row, int d0, const float (&x)[8], float (&y)[8]) {
    if (r.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
        return;
    }
    constexpr int kItem = kF32 ? 4 : 2;
    const int half = r.rot / 2;
    if (half % 8 == 0) {
        load8(row + (d0 < half ? d0 + half : d0 - half) * kItem, kF32, y);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = d0 + e;
        y[e] = 0.0f;
        if (d >= r.rot) continue;
        const int o = d < half ? d + half : d - half;
        y[e] = kF32 ? reinterpret_cast<const float*>(row)[o] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[o]);
    }
}

// A warp takes one row's heads, kCopyAhead groups of them: of the queries, of the keys or of the values (blockIdx.y).
// A step of 32 tokens (64 query and 8 key/value heads of 128): 8 us with the host's call, 4.4 back to back over bf16 and 6.1 over 4 bits, a
// chain of loads (the row's request, its page, positions, angles); rows and partners are asked for ahead of it.  It is made for steps: 1024
// rows take 19 to 21 us, 8192 119 (bf16), 132 (8 bits) and 135 (4 bits), where turning and appending by calls of their own take 66 to 70: a
// warp works out its angles for every eight heads of a row, partners are read twice, 80 to 90 million warp instructions, issue slots 59 %.
template <int kFmt, int kDim, bool kF32>
__global__ void __launch_bounds__(kCopyThreads, 2) rope_append_kernel(const RopeAppendParams p) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kLanes = kDim / 8, kPerWarp = 32 / kLanes, kItem = kF32 ? 4 : 2;
    const int part = int(blockIdx.y);
    const int which = part < p.q_chunks ? -1 : (part - p.q_chunks) & 1;                       // -1: queries
    const int chunk = part < p.q_chunks ? part : (part - p.q_chunks) >> 1;
    const int heads = which < 0 ? p.q_heads : p.cache.heads;
    const int sub = int(lane_id()) / kLanes, l = int(lane_id()) % kLanes, head0 = chunk * kPerWarp * kCopyAhead + sub;
    const int64_t step = int64_t(gridDim.x) * (kCopyThreads / 32);
    for (int64_t at_row = blockIdx.x * int64_t(kCopyThreads / 32) + threadIdx.x / 32; at_row < p.batch.tokens; at_row += step) {
        const int row = int(at_row);
        const char* const src = which < 0 ? p.q + row * p.q_stride : p.rows[which] + row * p.row_stride;
        float x[kCopyAhead][8];
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i)
            if (head0 + i * kPerWarp < heads) load8(src + (int64_t(head0 + i * kPerWarp) * kDim + l * 8) * kItem, kF32, x[i]);
        // (partners too, ahead of everything that is looked up)
        float y[kCopyAhead][8];
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i)
            if (which != 1 && l * 8 < p.rope.rot && head0 + i * kPerWarp < heads)
                rope_partners<kF32>(p.rope, src + int64_t(head0 + i * kPerWarp) * kDim * kItem, l * 8, x[i], y[i]);
        KvRowPlace at;
        at.pos = 0;
        const bool owned = kv_locate_row(p.cache, p.batch, row, kDim / 16, &at);
        if (which != 1) {
            RopeLane turn;
            rope_lane(p.rope, l * 8, p.positions ? p.positions[row] : owned ? at.pos : 0, &turn);
            __syncwarp();                                     // (queries may be turned in place: every lane has what it needs)
            if (turn.turned) {
#pragma unroll
                for (int i = 0; i < kCopyAhead; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (l * 8 + e < p.rope.rot) x[i][e] = fmaf(x[i][e], turn.c[e], y[i][e] * turn.s[e]);
            }
        }
        if (which < 0) {
#pragma unroll
            for (int i = 0; i < kCopyAhead; ++i)
                if (head0 + i * kPerWarp < heads)
                    store8(reinterpret_cast<char*>(p.q_out) + row * p.q_out_stride + (int64_t(head0 + i * kPerWarp) * kDim + l * 8) * 2, false, x[i]);
            continue;
        }
        if (!owned) continue;
        if (!at.page) {
            if (lane_id() == 0) atomicCAS(p.status, 0u, kBadPage);
            continue;
        }
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            const int head = head0 + i * kPerWarp;
            if (head >= heads) continue;                      // (whole groups leave together; no shuffle spans groups)
            if constexpr (kFmt == TL_KV_BF16) store8(p.cache.base[which] + at.at + int64_t(head) * p.cache.head_stride + l * 16, false, x[i]);
            else kv_store_codes<kFmt, kDim>(p.cache, which, at, head, l, sub, x[i], kv_top_f32(x[i]));
        }
    }
}

// A row's depth: the steps from it to the root.  Parents lie strictly below, so the climb ends.
__global__ void __launch_bounds__(256) tree_positions_kernel(const int32_t* parents, const int32_t* offsets, const int32_t* start, int requests, int tokens,
                                      int32_t* positions) {
    pdl_wait();
    pdl_launch_dependents();
    const int64_t at = int64_t(blockIdx.x) * 8 + threadIdx.x / 32;         // (a warp per row: threads pass 32 bits)
    if (at >= tokens) return;
    const int row = int(at);
    int b = -1, first = 0;
    for (int b0 = 0; b0 < requests && b < 0; b0 += 32) {
        const int mine = min(b0 + int(lane_id()), requests - 1);
        const int a = min(max(offsets[mine], 0), tokens), e = min(max(offsets[mine + 1], a), tokens);
        const uint32_t owner = __ballot_sync(0xffffffffu, b0 + int(lane_id()) < requests && row >= a && row < e);
        if (!owner) continue;
        b = b0 + __ffs(int(owner)) - 1;
        first = __shfl_sync(0xffffffffu, a, __ffs(int(owner)) - 1);
    }
    if (b < 0 || lane_id() != 0) return;
    int depth = 0;
    for (int i = row - first; i >= 0; ++depth) {
        const int up = parents[first + i];
        i = up < i ? up : -1;
    }
    positions[row] = start[b] + depth - 1;
}

static int rope_view(const tl_rope* r, int head_dim, RopeView* out) {
    if (!r || !r->turns || !std::isfinite(r->amplitude)) return TL_ERR_INVALID_ARG;
    if (r->layout != TL_ROPE_HALF && r->layout != TL_ROPE_INTERLEAVED) return TL_ERR_INVALID_ARG;
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > head_dim) return TL_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(r->turns) % 8) return TL_ERR_ALIGNMENT;
    out->turns = r->turns;
    out->amplitude = r->amplitude;
    out->rot = r->rotary_dim;
    out->interleaved = r->layout == TL_ROPE_INTERLEAVED;
    return TL_OK;
}

using RopeKernel = void (*)(RopeAppendParams);
template <int kFmt, bool kF32>
static RopeKernel pick_rope(int dim) {
    return dim == 64 ? rope_append_kernel<kFmt, 64, kF32> : dim == 128 ? rope_append_kernel<kFmt, 128, kF32> : rope_append_kernel<kFmt, 256, kF32>;
}
template <bool kF32>
static RopeKernel pick_rope_format(int format, int dim) {
    switch (format) {
        case TL_KV_BF16: return pick_rope<TL_KV_BF16, kF32>(dim);
        case TL_KV_E4M3: return pick_rope<TL_KV_E4M3, kF32>(dim);
        case TL_KV_INT8: return pick_rope<TL_KV_INT8, kF32>(dim);
        default: return pick_rope<TL_KV_E2M1, kF32>(dim);
    }
}

}  // namespace tl

extern "C" {

int tl_rope_turns(int rotary_dim, double base, int scaling, double factor, double original, double low, double high,
                  uint64_t* h_turns) {
    using namespace tl;
    if (!h_turns || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 1024) return TL_ERR_INVALID_ARG;
    if (!(base > 1.0) || !std::isfinite(base) || scaling < TL_ROPE_PLAIN || scaling > TL_ROPE_RAMP) return TL_ERR_INVALID_ARG;
    if (scaling != TL_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return TL_ERR_INVALID_ARG;
    if (scaling >= TL_ROPE_BANDS &&
        (!(original > 0.0) || !std::isfinite(original) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
        return TL_ERR_INVALID_ARG;
    using real = long double;                                 // 64 bits of mantissa: the fixed-point words are good to their last bits
    const real two_pi = 6.283185307179586476925286766559005768L;
    real from = 0, to = 0;
    if (scaling == TL_ROPE_RAMP) {
        // the pair that makes n turns over the original context: original * base^(-2i / rotary_dim) = 2 pi n
        auto pair = [&](double n) { return real(rotary_dim) * std::log(real(original) / (real(n) * two_pi)) / (2 * std::log(real(base))); };
        from = std::max<real>(std::floor(pair(high)), 0);
        to = std::min<real>(std::ceil(pair(low)), rotary_dim - 1);
        if (to <= from) to = from + 0.001L;
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        real f = std::pow(real(base), real(-2 * i) / real(rotary_dim));
        if (scaling == TL_ROPE_LINEAR) f /= real(factor);
        if (scaling == TL_ROPE_BANDS) {
            const real n = real(original) * f / two_pi;
            const real u = std::min<real>(std::max<real>((n - real(low)) / (real(high) - real(low)), 0), 1);
            f = (1 - u) * f / real(factor) + u * f;
        }
        if (scaling == TL_ROPE_RAMP) {
            const real u = std::min<real>(std::max<real>((i - from) / (to - from), 0), 1);
            f = u * f / real(factor) + (1 - u) * f;
        }
        h_turns[i] = uint64_t(std::floor(f / two_pi * 18446744073709551616.0L + 0.5L));       // f <= 1: less than a sixth of a turn
    }
    return TL_OK;
}

int tl_rope_rows(const tl_rope* rope, const void* d_x, int64_t x_stride, void* d_out, int64_t out_stride, int elem, int tokens,
                 int heads, int head_dim, const int32_t* d_positions, int inverse, void* cuda_stream) {
    using namespace tl;
    RopeRowsParams p = {};
    if (head_dim < 2 || head_dim > 1024 || head_dim % 2) return head_dim > 1024 ? TL_ERR_UNSUPPORTED : TL_ERR_INVALID_ARG;
    if (int rc = rope_view(rope, head_dim, &p.rope)) return rc;
    if (elem != TL_ELEM_BF16 && elem != TL_ELEM_F32) return TL_ERR_INVALID_ARG;
    if (tokens < 0 || heads < 0) return TL_ERR_INVALID_ARG;
    if (tokens == 0 || heads == 0) return TL_OK;
    const int64_t wide = int64_t(heads) * head_dim, item = elem == TL_ELEM_F32 ? 4 : 2;
    if (!d_x || !d_out || !d_positions || x_stride < wide || out_stride < wide) return TL_ERR_INVALID_ARG;
    if (d_x == d_out && x_stride != out_stride) return TL_ERR_INVALID_ARG;
    if (x_stride > (int64_t(1) << 40) || out_stride > (int64_t(1) << 40)) return TL_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(d_x) % item || reinterpret_cast<uintptr_t>(d_out) % item || !words_aligned(d_positions)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_device_info()) return rc;
    p.x = static_cast<const char*>(d_x);
    p.out = static_cast<char*>(d_out);
    p.x_stride = x_stride * item;
    p.out_stride = out_stride * item;
    p.positions = d_positions;
    p.tokens = tokens;
    p.heads = heads;
    p.dim = head_dim;
    p.inverse = inverse != 0;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool vectors = p.rope.rot % 16 == 0 && head_dim % 8 == 0 && (head_dim * item) % 16 == 0 && p.x_stride % 16 == 0 && p.out_stride % 16 == 0 &&
                         reinterpret_cast<uintptr_t>(d_x) % 16 == 0 && reinterpret_cast<uintptr_t>(d_out) % 16 == 0;
    // enough warps (threads) for every SM first, then as many heads to an angle as there are
    const int64_t want = int64_t(dev().sm_count) * (vectors ? 32 : 1024);
    if (vectors) {
        const int64_t chunks = std::min<int64_t>(heads, std::max<int64_t>(1, want / tokens));
        p.heads_per_warp = int(ceil_div(heads, chunks));
        const int64_t warps = int64_t(tokens) * ceil_div(heads, p.heads_per_warp);
        if (ceil_div(warps, kRopeThreads / 32) > INT32_MAX) return TL_ERR_UNSUPPORTED;
        return kv_launch(elem == TL_ELEM_F32 ? rope_rows_kernel<true> : rope_rows_kernel<false>, dim3(unsigned(ceil_div(warps, kRopeThreads / 32))), kRopeThreads, stream, p);
    }
    const int64_t items = p.rope.rot / 2 + (d_x == d_out ? 0 : head_dim - p.rope.rot);
    const int64_t chunks = std::min<int64_t>(std::min<int64_t>(heads, 65535), std::max<int64_t>(1, want / (tokens * items)));
    p.heads_per_warp = int(ceil_div(heads, chunks));
    if (ceil_div(tokens * items, kRopeThreads) > INT32_MAX) return TL_ERR_UNSUPPORTED;
    return kv_launch(elem == TL_ELEM_F32 ? rope_rows_any_kernel<true> : rope_rows_any_kernel<false>,
                     dim3(unsigned(ceil_div(tokens * items, kRopeThreads)), unsigned(ceil_div(heads, p.heads_per_warp))), kRopeThreads, stream, p);
}

int tl_rope_append(const tl_kv_cache* cache, const tl_kv_batch* batch, const tl_rope* rope, const int32_t* d_positions, const void* d_q,
                   int64_t q_stride, int q_heads, void* d_q_out, int64_t q_out_stride, const void* d_k, const void* d_v, int elem,
                   int64_t kv_stride, void* cuda_stream) {
    using namespace tl;
    RopeAppendParams p = {};
    if (int rc = kv_view(cache, &p.cache)) return rc;
    if (int rc = kv_batch_view(batch, &p.batch)) return rc;
    if (int rc = rope_view(rope, cache->head_dim, &p.rope)) return rc;
    if (elem != TL_ELEM_BF16 && elem != TL_ELEM_F32) return TL_ERR_INVALID_ARG;
    if (q_heads < 0 || (q_heads == 0) != (d_q == nullptr) || (d_q == nullptr) != (d_q_out == nullptr)) return TL_ERR_INVALID_ARG;
    if (p.batch.tokens == 0 || p.batch.requests == 0) return TL_OK;
    const int64_t item = elem == TL_ELEM_F32 ? 4 : 2, dim = cache->head_dim, most = int64_t(1) << 40;
    if (!d_k || !d_v || kv_stride < cache->heads * dim) return TL_ERR_INVALID_ARG;
    if (q_heads && (q_stride < q_heads * dim || q_out_stride < q_heads * dim)) return TL_ERR_INVALID_ARG;
    if (d_q && d_q == d_q_out && (elem != TL_ELEM_BF16 || q_stride != q_out_stride)) return TL_ERR_INVALID_ARG;
    if (kv_stride > most || (q_heads && (q_stride > most || q_out_stride > most))) return TL_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(d_k) % 16 || reinterpret_cast<uintptr_t>(d_v) % 16 || (kv_stride * item) % 16 ||
        !words_aligned(d_positions))
        return TL_ERR_ALIGNMENT;
    if (q_heads && (reinterpret_cast<uintptr_t>(d_q) % 16 || reinterpret_cast<uintptr_t>(d_q_out) % 16 || (q_stride * item) % 16 || (q_out_stride * 2) % 16))
        return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    p.positions = d_positions;
    p.q = static_cast<const char*>(d_q);
    p.q_out = static_cast<__nv_bfloat16*>(d_q_out);
    p.rows[0] = static_cast<const char*>(d_k);
    p.rows[1] = static_cast<const char*>(d_v);
    p.q_stride = q_stride * item;
    p.q_out_stride = q_out_stride * 2;
    p.row_stride = kv_stride * item;
    p.status = dev().ctl.d_status;
    p.q_heads = q_heads;
    const int64_t per = int64_t(kCopyAhead) * (32 / (cache->head_dim / 8));
    p.q_chunks = int(ceil_div(q_heads, per));
    p.kv_chunks = int(ceil_div(cache->heads, per));
    const int64_t parts = p.q_chunks + 2 * int64_t(p.kv_chunks);
    if (parts > 65535) return TL_ERR_UNSUPPORTED;
    const int64_t blocks = std::min<int64_t>(ceil_div(p.batch.tokens, kCopyThreads / 32), std::max<int64_t>(int64_t(dev().sm_count) * 32 / parts, 1));
    return kv_launch(elem == TL_ELEM_F32 ? pick_rope_format<true>(cache->format, cache->head_dim) : pick_rope_format<false>(cache->format, cache->head_dim),
                     dim3(unsigned(blocks), unsigned(parts)), kCopyThreads, static_cast<cudaStream_t>(cuda_stream), p);
}

int tl_tree_positions(const int32_t* d_parents, const int32_t* d_token_offsets, const int32_t* d_start, int requests, int tokens,
                      int32_t* d_positions, void* cuda_stream) {
    using namespace tl;
    if (requests < 0 || tokens < 0) return TL_ERR_INVALID_ARG;
    if (requests == 0 || tokens == 0) return TL_OK;
    if (!d_parents || !d_token_offsets || !d_start || !d_positions) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_parents, d_token_offsets, d_start, d_positions)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    return kv_launch(tree_positions_kernel, dim3(unsigned(ceil_div(tokens, 8))), 256, static_cast<cudaStream_t>(cuda_stream),
                     d_parents, d_token_offsets, d_start, requests, tokens, d_positions);
}

}  // extern "C"
