// Rows of the key/value cache as its copying kernels handle them: finding a row's place, quantising it, reading it back.
#pragma once

#include "tl_kv.cuh"

namespace tl {

#ifdef __CUDACC__

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
    int pos;                    // of the row in its sequence
    int64_t at, scale_at;       // bytes, floats
    int64_t group_at;           // bytes, for rows of `groups` group scales
};
__device__ __forceinline__ bool kv_locate_row(const KvView& cache, const KvBatchView& bv, int row, int groups, KvRowPlace* out) {
    // the request that owns the row, looked for 32 at a time; each lane has its request's data at hand (a look at them once
    // the owner is known would be one more round trip)
    KvRequest r = {};
    int b = bv.requests;
    for (int b0 = 0; b0 < bv.requests; b0 += 32) {
        const int mine = min(b0 + int(lane_id()), bv.requests - 1);
        const KvRequest q = kv_request(bv, cache.page_shift, mine);
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
    out->pos = pos;
    out->at = out->scale_at = out->group_at = 0;
    if (pos >= kv_room(bv, cache.page_shift)) return true;
    const int64_t page = bv.page_table[int64_t(b) * bv.table_stride + (pos >> cache.page_shift)];
    const int line = pos & ((1 << cache.page_shift) - 1);
    out->page = page >= 0 && page < cache.pages;
    if (!out->page) return true;
    out->at = page * cache.page_stride + line * cache.token_stride;
    out->scale_at = page * cache.scale_page_stride + line;
    out->group_at = page * cache.group_page_stride + line * groups;
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
struct KvCodes<TL_KV_E2M1> {
    using type = uint32_t;
    // (code times group scale is exact in f16; g: kGroupUnit times less than the scale)
    __device__ static void expand(uint32_t c, uint32_t g, float s, float (&x)[8]) {
        uint32_t h[4];
        e2m1x8_to_f16(c, g, h);
        s *= kGroupUnit;
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

// The largest magnitude of eight values, as bits.
__device__ __forceinline__ uint32_t kv_top_f32(const float (&x)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    return top;
}
__device__ __forceinline__ uint32_t kv_top_bf16(const uint4& v) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __vmaxu2(top, u[e] & 0x7fff7fffu);                          // two bf16 patterns at a time
    return max(top & 0xffff0000u, top << 16);
}
// The 4-bit format's rule, in three steps: the row's scale from its largest magnitude (as bits), a group's from its own, codes.
struct E2m1Row {
    float scale, to;                     // and 1 / scale (exact); 0 where every code is 0
};
__device__ __forceinline__ E2m1Row e2m1_row(uint32_t top) {
    const bool finite = top < 0x7f800000u, some = finite && top != 0;
    // the least power of two of which 6 * 448 = 1.3125 * 2^11 times is not below the largest magnitude
    const int k = max(int(top >> 23) - 138 + ((top & 0x7fffffu) > 0x280000u ? 1 : 0), -126);
    return {some ? __uint_as_float(uint32_t(k + 127) << 23) : finite ? 0.0f : __uint_as_float(0x7fc00000u),
            some ? __uint_as_float(uint32_t(127 - k) << 23) : 0.0f};
}
__device__ __forceinline__ uint32_t e2m1_group(uint32_t top, const E2m1Row& row) {
    // (rows without codes: 0; a row that is not finite must not bring its infinity in)
    const float want = row.to == 0.0f ? 0.0f : __fmul_rn(__fmul_rn(__uint_as_float(top), row.to), 1.0f / 6.0f);
    uint16_t two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.0f), "f"(want));
    return two;
}
__device__ __forceinline__ uint32_t e2m1_codes(const float (&x)[8], uint32_t byte, const E2m1Row& row) {
    if (byte == 0) return 0;
    const uint32_t wide = e4m3x2_to_f16x2(byte);
    const float g = __low2float(*reinterpret_cast<const __half2*>(&wide)), inv = __frcp_rn(g);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {                             // the correctly rounded quotient, as for the 8-bit codes
        // (With the remainder's sign the other way round a zero keeps its own: -0 * g + 0 = 0, then -0 * inv + -0 = -0.)
        const float xs = __fmul_rn(x[e], row.to), q = __fmul_rn(xs, inv);
        y[e] = __fmaf_rn(-__fmaf_rn(q, g, -xs), inv, q);
    }
    uint32_t codes;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(codes) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return codes;
}

// A lane's eight values of one head's row (the kDim / 8 lanes of the row call together) into codes and scale.  top: the lane's largest
// magnitude, as bits: a NaN's pattern is above an infinity's, so either makes the scale NaN.
template <int kFmt, int kDim>
__device__ __forceinline__ void kv_store_codes(const KvView& cache, int which, const KvRowPlace& at, int head, int l, int sub, const float (&x)[8], uint32_t top) {
    static_assert(kFmt != TL_KV_BF16, "codes");
    constexpr int kLanes = kDim / 8;
    char* const dst = cache.base[which] + at.at + int64_t(head) * cache.head_stride;
    const uint32_t group = (kLanes == 32 ? 0xffffffffu : ((1u << kLanes) - 1u) << (sub * kLanes));
    if constexpr (kFmt == TL_KV_E2M1) {
        // two lanes share a group scale
        const uint32_t pair = max(top, __shfl_xor_sync(group, top, 1));
        top = pair;
#pragma unroll
        for (int d = kLanes / 2; d > 1; d >>= 1) top = max(top, __shfl_xor_sync(group, top, d));
        const E2m1Row row = e2m1_row(top);
        const uint32_t byte = e2m1_group(pair, row), codes = e2m1_codes(x, byte, row);
        *reinterpret_cast<uint32_t*>(dst + l * 4) = codes;
        if ((l & 1) == 0) cache.group[which][at.group_at + int64_t(head) * cache.group_head_stride + (l >> 1)] = char(byte);
        if (l == 0) cache.scale[which][at.scale_at + int64_t(head) * cache.scale_head_stride] = row.scale;
    } else {
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
        if (l == 0) cache.scale[which][at.scale_at + int64_t(head) * cache.scale_head_stride] = s;
    }
}

// Launch with programmatic stream serialisation (unless it is switched off).
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

#endif  // __CUDACC__

}  // namespace tl
