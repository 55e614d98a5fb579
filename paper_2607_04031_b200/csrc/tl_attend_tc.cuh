// Attention for many query rows per key/value head (trees, chains of drafts, prompt chunks) on the 5th-generation
// tensor cores.
//
// One CTA per SM, four warpgroups: two for softmax (streams A and B), one of producers, and one whose first warp issues
// the matrix instructions; registers are moved from the last two to the first two (168 + 168 + 120 + 56 = 4 x 128 a thread).  A stream is an accumulator O (128 rows x dim) and a score tile S (128 x 128) in tensor memory.
//   kBlocks = 2  the streams hold different rows (256 rows a unit) and use every key/value tile together: each fetched
//                and converted element serves 256 rows;
//   kBlocks = 1  the streams hold the same 128 rows and take the tiles in turn; their sums are joined at the end.
// Either way one stream's products run while the other's softmax does.  Per tile and stream: S = Q K^T (both operands in
// shared memory, 128-byte swizzle), thread r of the warpgroup reads row r of S (no exchange between threads), writes the
// weights back over S as 16-bit values, and O += P V takes P from tensor memory and V from shared memory as an MN-major
// operand, so neither P nor V^T is ever laid out again.
//
// The row maximum is allowed to lag: weights are taken against the maximum known when the tile began, and only when a
// score exceeds that by more than 2^8 is the tile done again with the new maximum and O rescaled; sums are fp32 and f16
// has room for 2^15, so the lag costs no accuracy.  Scales of 8-bit caches enter as in the kernel for few rows (key's
// scale on the score, value's in the exponent), q is f16 scaled by a power of two per row; conversion to f16 is exact.
//
// 8-bit tiles are loaded by the producers into registers one tile ahead, converted and stored swizzled; full bf16 tiles
// come by TMA (128-byte-swizzled boxes, one per page and 64 dimensions); a tile with positions past the end, or with a
// page outside the pool, goes through registers too, with zeros in those places.
#pragma once

#include "tl_attend.cuh"

namespace tl {

enum : uint32_t { kWaitAttend = 0xC00 };

constexpr int kTcTile = 128, kTcThreads = 16 * 32;
constexpr int kTcSoftmaxWarps = 8, kTcProducerWarp = 8, kTcMmaWarp = 12;

struct AttendTcParams {
    AttendParams a;
    CUtensorMap map[2];                  // keys, values (bf16 caches)
    int box_tokens;
    uint64_t wait_ns;
};

template <int kDim, int kBlocks>
struct TcShape {
    static constexpr int kAtoms = kDim / 64;                       // 128-byte columns of a 16-bit operand tile
    static constexpr int kAtomBytes = kTcTile * 128;
    static constexpr int kOperand = kAtoms * kAtomBytes;           // one 128-row operand tile
    static constexpr int kKStages = 2, kVStages = kBlocks == 1 ? 3 : 2;
    static constexpr int kOffK = kBlocks * kOperand;
    static constexpr int kOffV = kOffK + kKStages * kOperand;
    static constexpr int kOffScale = kOffV + kVStages * kOperand;  // [stage][ks, log2 vs, 1 / vs][128]
    static constexpr int kOffStat = kOffScale + kVStages * 3 * kTcTile * 4;
    static constexpr int kOffBar = kOffStat + 2 * kTcTile * 16;
    static constexpr int kSmem = kOffBar + 256 + 1024;             // 1024: the base is aligned by hand
    static constexpr int kRows = kBlocks * 128;
    // tensor memory columns
    static constexpr int kS = 0, kO = 256;                         // S of stream x at x * 128, O at 256 + x * 128
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

#ifdef __CUDACC__

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, uint64_t* bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem desc]
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor without its address: 128-byte swizzle, leading and stride byte offsets.
__device__ __forceinline__ uint64_t tc_desc_hi(uint32_t lbo, uint32_t sbo) {
    return (uint64_t(lbo >> 4) << 16) | (uint64_t(sbo >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}

template <int kRegs>
__device__ __forceinline__ void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs>
__device__ __forceinline__ void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }

// Two fp32 operations per instruction.
struct F2 { float x, y; };
__device__ __forceinline__ uint64_t f2_bits(F2 a) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ F2 f2_of(uint64_t r) {
    F2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(r));
    return a;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)), "l"(f2_bits(c)));
    return f2_of(r);
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_of(r);
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_of(r);
}

// Barriers of the CTA.  Every wait on them is bounded.
struct TcBars {
    uint64_t q_full;                     // 8 softmax warps: queries are in place, the last unit's accumulators are read
    uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3];
    uint64_t s_full[2], p_full[2], pv_done[2];
    uint64_t exchange;                   // 8 softmax warps: statistics of the two streams are in place
    uint64_t drained;                    // the issuing thread's last commit, when it gives up
    uint32_t abort_flag, tmem_base;
    uint32_t meta[3];                    // per value stage: groups of 16 positions that should have a page and have none
    uint32_t odd[3][4];                  // per value stage and producer warp: values that are not finite were taken out
};
static_assert(sizeof(TcBars) <= 256, "barrier block");

template <int kDim, int kFmt, int kBlocks>
__global__ void __launch_bounds__(kTcThreads, 1) attend_tc_kernel(const __grid_constant__ AttendTcParams tp) {
    using S = TcShape<kDim, kBlocks>;
    constexpr bool kBf16 = kFmt == TL_KV_BF16;
    extern __shared__ char smem_raw[];
    char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    TcBars& bars = *reinterpret_cast<TcBars*>(smem + S::kOffBar);
    float* const scales = reinterpret_cast<float*>(smem + S::kOffScale);
    float4* const stats = reinterpret_cast<float4*>(smem + S::kOffStat);     // [stream][row]: maximum, sum, odd values seen
    const AttendParams& p = tp.a;
    const int warp = int(threadIdx.x) / 32, lane = int(lane_id());
    volatile uint32_t* const abort_ptr = &bars.abort_flag;

    if (threadIdx.x == 0) {
        mbar_init(&bars.q_full, kTcSoftmaxWarps);
        for (int i = 0; i < 3; ++i) {
            mbar_init(&bars.k_full[i], 4);
            mbar_init(&bars.k_empty[i], 1);
            mbar_init(&bars.v_full[i], 4);
            mbar_init(&bars.v_empty[i], 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&bars.s_full[x], 1);
            mbar_init(&bars.p_full[x], 4);
            mbar_init(&bars.pv_done[x], 1);
        }
        mbar_init(&bars.exchange, kTcSoftmaxWarps);
        mbar_init(&bars.drained, 1);
        bars.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kTcMmaWarp) {
        tmem_alloc(&bars.tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = bars.tmem_base;

    pdl_wait();
    pdl_launch_dependents();
    const int64_t total = attend_total(p);
    const int64_t per = attend_per_cta(total, p.ctas);
    int64_t x0 = int64_t(blockIdx.x) * per;
    const int64_t x_end = min(x0 + per, total);

    auto wait = [&](uint64_t* bar, uint32_t parity) {
        return mbar_wait_bounded(bar, parity, abort_ptr, p.status, kWaitAttend, tp.wait_ns);
    };
    auto warp_wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };

    if (x0 < x_end) {
        AttendPlace w = attend_locate(p, x0);
        uint32_t tiles_before = 0;                             // tiles of this CTA's earlier units: ring positions count on
        uint32_t unit = 0;
        bool alive = true;

        if (warp < kTcSoftmaxWarps) {
            // ============================================================ softmax
            // (every warpgroup of a CTA with work takes its share: together they are what the block was launched with)
            reg_inc<168>();
            const int stream = warp / 4, r = int(threadIdx.x) & 127;
            const uint32_t lanes = uint32_t(warp & 3) * 32u << 16;           // this warp's quarter of tensor memory
            const uint32_t s_tmem = tmem + lanes + S::kS + uint32_t(stream) * 128u;
            const uint32_t o_tmem = tmem + lanes + S::kO + uint32_t(stream) * 128u;
            uint32_t s_count = 0;
            while (true) {
                const int t0 = w.tile, t1 = int(min(int64_t(w.a.tiles), t0 + (x_end - x0)));
                const int tiles = t1 - t0;
                const int unit_rows = min(S::kRows, w.a.r.n * p.group - w.block * S::kRows);
                const int row = w.block * S::kRows + (kBlocks == 2 ? stream * 128 : 0) + r;
                const bool live = row - w.block * S::kRows < unit_rows;
                const int tok = live ? row / p.group : 0, hq = w.head * p.group + (live ? row % p.group : 0);
                const bool active = kBlocks == 2 ? stream * 128 < unit_rows : stream < tiles;
                float fac = p.scale_log2;
                {
                    // this row of q, converted, into the operand tile
                    uint4 q[kDim / 8];
                    const uint4* src = reinterpret_cast<const uint4*>(p.q + int64_t(w.a.r.first + tok) * p.q_stride + int64_t(hq) * kDim);
#pragma unroll
                    for (int c = 0; c < kDim / 8; ++c) q[c] = live ? src[c] : make_uint4(0, 0, 0, 0);
                    float mul = 1.0f;
                    if (!kBf16) {
                        uint32_t top = 0;
#pragma unroll
                        for (int c = 0; c < kDim / 8; ++c) {
                            const uint32_t u[4] = {q[c].x, q[c].y, q[c].z, q[c].w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) top = max(top, max((u[i] << 16) & 0x7fff0000u, u[i] & 0x7fff0000u));
                        }
                        const int e = int(top >> 23);
                        const int up = e == 0 || e == 255 ? 0 : min(127 + 14 - e, 100);
                        mul = __uint_as_float(uint32_t(127 + up) << 23);
                        fac *= __uint_as_float(uint32_t(127 - up) << 23);
                    }
                    if (kBlocks == 2 || stream == 0) {
                        char* const dst = smem + (kBlocks == 2 ? stream * S::kOperand : 0) + r * 128;
#pragma unroll
                        for (int c = 0; c < kDim / 8; ++c) {
                            uint4 v = q[c];
                            if (!kBf16) {
                                uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int i = 0; i < 4; ++i) u[i] = pack_f16(__uint_as_float(u[i] << 16) * mul, __uint_as_float(u[i] & 0xffff0000u) * mul);
                                v = make_uint4(u[0], u[1], u[2], u[3]);
                            }
                            *reinterpret_cast<uint4*>(dst + (c / 8) * S::kAtomBytes + (((c % 8) ^ (r & 7)) << 4)) = v;
                        }
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_full);

                float m = -INFINITY, l = 0.0f;
                bool odd = false;
                const int step = kBlocks == 2 ? 1 : 2;
                for (int n = kBlocks == 2 ? 0 : stream; active && n < tiles; n += step) {
                    const bool first = n < step;
                    const uint32_t at = (tiles_before + n) % S::kVStages;
                    alive = warp_wait(&bars.v_full[at], ((tiles_before + n) / S::kVStages) & 1u) &&
                            warp_wait(&bars.s_full[stream], s_count & 1u);
                    if (!alive) break;
                    ++s_count;
                    tc_fence_after_sync();
                    const uint32_t meta = bars.meta[at];
                    if (kBf16) odd |= (bars.odd[at][0] | bars.odd[at][1] | bars.odd[at][2] | bars.odd[at][3]) != 0;
                    const int64_t pos0 = int64_t(t0 + n) * kTcTile;
                    const bool edge = pos0 + kTcTile > w.a.r.start || meta != 0;
                    const float4* const ks = reinterpret_cast<const float4*>(scales + at * 3 * kTcTile);
                    const float4* const lv = ks + kTcTile / 4;
                    const float4* const rv = lv + kTcTile / 4;
                    // bit i: this row sees position pos0 + 32 c + i
                    auto sees32 = [&](int c) -> uint32_t {
                        const int64_t pos = pos0 + c * 32;
                        if (pos >= w.a.len) return 0u;
                        uint32_t see = w.a.len - pos >= 32 ? 0xffffffffu : (1u << int(w.a.len - pos)) - 1u;
                        if (meta & (1u << (2 * c))) see &= 0xffff0000u;
                        if (meta & (2u << (2 * c))) see &= 0x0000ffffu;
                        const int64_t j = pos - w.a.r.start;                 // the step's token at bit 0
                        if (j + 31 < 0) return see;
                        auto word = [&](int64_t k) -> uint32_t {             // tokens 32 k .. 32 k + 31
                            if (k < 0) return 0xffffffffu;
                            if (p.mask) return k < p.mask_words ? p.mask[int64_t(w.a.r.first + tok) * p.mask_words + k] : 0u;
                            const int64_t d = tok - k * 32;
                            return d >= 31 ? 0xffffffffu : d < 0 ? 0u : (2u << int(d)) - 1u;
                        };
                        const int64_t k = j >> 5;
                        return see & __funnelshift_r(word(k), word(k + 1), uint32_t(j & 31));
                    };
                    // scores of 32 columns in log2 units
                    auto load_scores = [&](int c, F2 (&t)[16]) {
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(s_tmem + uint32_t(c) * 32u, v);
                        tmem_ld_wait();
                        const F2 f = {fac, fac};
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            F2 a = {__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1])};
                            F2 b = {__uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3])};
                            if (kBf16) {
                                t[2 * i] = f2_mul(a, f);
                                t[2 * i + 1] = f2_mul(b, f);
                            } else {
                                const float4 k4 = ks[c * 8 + i], v4 = lv[c * 8 + i];
                                t[2 * i] = f2_fma(f2_mul(a, F2{k4.x, k4.y}), f, F2{v4.x, v4.y});
                                t[2 * i + 1] = f2_fma(f2_mul(b, F2{k4.z, k4.w}), f, F2{v4.z, v4.w});
                            }
                        }
                        if (edge) {
                            const uint32_t see = sees32(c);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                if (!(see >> (2 * i) & 1u)) t[i].x = -INFINITY;
                                if (!(see >> (2 * i + 1) & 1u)) t[i].y = -INFINITY;
                            }
                        }
                    };
                    uint32_t pw[64];
                    bool fresh = __any_sync(0xffffffffu, m == -INFINITY);
                    while (true) {
                        if (fresh) {
                            float top = -INFINITY;
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
                                F2 t[16];
                                load_scores(c, t);
#pragma unroll
                                for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(t[i].x, t[i].y));
                            }
                            const float m_new = fmaxf(m, top);
                            const float f = m == -INFINITY ? 0.0f : ex2(m - m_new);
                            if (!first && __any_sync(0xffffffffu, m_new > m)) {
                                // (S of this tile was issued after the previous O += P V had completed)
#pragma unroll 1
                                for (int c = 0; c < kDim / 32; ++c) {
                                    uint32_t v[32];
                                    tmem_ld_32x32b_x32(o_tmem + uint32_t(c) * 32u, v);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                                    tmem_st_32x32b_x32(o_tmem + uint32_t(c) * 32u, v);
                                }
                            }
                            l *= f;
                            m = m_new;
                        }
                        const float use = m == -INFINITY ? 0.0f : m;
                        const F2 minus = {-use, -use};
                        F2 top = {-INFINITY, -INFINITY}, sum = {0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            F2 t[16];
                            load_scores(c, t);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                top.x = fmaxf(top.x, t[i].x);
                                top.y = fmaxf(top.y, t[i].y);
                                const F2 d = f2_add(t[i], minus);
                                const F2 e = {ex2(d.x), ex2(d.y)};
                                if (kBf16) {
                                    sum = f2_add(sum, e);
                                    pw[c * 16 + i] = pack_bf16(e.x, e.y);
                                } else {
                                    const float2 r2 = reinterpret_cast<const float2*>(rv)[c * 16 + i];
                                    sum = f2_fma(e, F2{r2.x, r2.y}, sum);
                                    pw[c * 16 + i] = pack_f16(e.x, e.y);
                                }
                            }
                        }
                        if (!fresh && __any_sync(0xffffffffu, fmaxf(top.x, top.y) > use + 8.0f)) {
                            fresh = true;
                            continue;
                        }
                        l += sum.x + sum.y;
                        break;
                    }
                    tmem_st_32x32b_x32(s_tmem, pw);
                    tmem_st_32x32b_x32(s_tmem + 32u, pw + 32);
                    tmem_st_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.p_full[stream]);
                }
                if (!alive) break;
                // the last product of this stream
                if (active) {
                    alive = warp_wait(&bars.pv_done[stream], (s_count - 1) & 1u);
                    if (!alive) break;
                    tc_fence_after_sync();
                }
                float f_own = 1.0f, f_other = 0.0f, m_all = m, l_all = l;
                bool odd_all = odd;
                if (kBlocks == 1) {
                    stats[stream * kTcTile + r] = make_float4(m, l, odd ? 1.0f : 0.0f, 0.0f);
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.exchange);
                    alive = warp_wait(&bars.exchange, unit & 1u);
                    if (!alive) break;
                    tc_fence_after_sync();
                    const float4 o = stats[(stream ^ 1) * kTcTile + r];
                    m_all = fmaxf(m, o.x);
                    const float use = m_all == -INFINITY ? 0.0f : m_all;
                    f_own = ex2(m - use);
                    f_other = ex2(o.x - use);
                    l_all = l * f_own + o.y * f_other;
                    odd_all |= o.z != 0.0f;
                }
                if (kBlocks == 1 || active) {
                    const bool whole = t0 == 0 && t1 == w.a.tiles;
                    const int64_t slot = int64_t(blockIdx.x) * 2 + (t0 > 0 ? 0 : 1);
                    const float inv = whole ? (l_all == 0.0f ? 0.0f : 1.0f / l_all) : 1.0f;
                    const int prow = (kBlocks == 2 ? stream * 128 : 0) + r;
                    const bool two = kBlocks == 1 && tiles > 1;
                    // kBlocks = 1: each stream's threads write half of the columns
                    const int c_from = kBlocks == 1 ? stream * (kDim / 64) : 0, c_to = kBlocks == 1 ? c_from + kDim / 64 : kDim / 32;
                    const uint32_t o_a = tmem + lanes + S::kO;
                    const float fa = (stream == 0 ? f_own : f_other) * inv, fb = (stream == 0 ? f_other : f_own) * inv;
#pragma unroll 1
                    for (int c = c_from; c < c_to; ++c) {
                        uint32_t v[32];
                        float o[32];
                        if (kBlocks == 1) {
                            tmem_ld_32x32b_x32(o_a + uint32_t(c) * 32u, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(v[i]) * fa;
                            if (two) {
                                tmem_ld_32x32b_x32(o_a + 128u + uint32_t(c) * 32u, v);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = fmaf(__uint_as_float(v[i]), fb, o[i]);
                            }
                        } else {
                            tmem_ld_32x32b_x32(o_tmem + uint32_t(c) * 32u, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(v[i]) * inv;
                        }
                        if (!live) continue;
                        if (kBf16 && odd_all) {
                            // infinities and NaN among the values of the step's own tokens were taken out of the product
                            const int64_t from = max(w.a.r.start, int64_t(t0) * kTcTile), to = min(w.a.len, int64_t(t1) * kTcTile);
                            for (int64_t pos = from; pos < to; ++pos) {
                                if (!attend_sees(p, w.a.r.first + tok, tok, pos - w.a.r.start)) continue;
                                const int page = p.batch.page_table[int64_t(w.b) * p.batch.table_stride + (pos >> p.cache.page_shift)];
                                if (page < 0 || page >= p.cache.pages) continue;
                                const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                                    p.cache.base[1] + int64_t(page) * p.cache.page_stride + int64_t(w.head) * p.cache.head_stride +
                                    (pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride) + c * 32;
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const float e = __bfloat162float(v[i]);
                                    if (!(fabsf(e) < INFINITY)) o[i] += e;
                                }
                            }
                        }
                        if (whole) {
                            uint4* dst = reinterpret_cast<uint4*>(p.out + int64_t(w.a.r.first + tok) * p.out_stride + int64_t(hq) * kDim + c * 32);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                dst[i] = make_uint4(pack_bf16(o[8 * i], o[8 * i + 1]), pack_bf16(o[8 * i + 2], o[8 * i + 3]),
                                                    pack_bf16(o[8 * i + 4], o[8 * i + 5]), pack_bf16(o[8 * i + 6], o[8 * i + 7]));
                        } else {
                            float4* dst = reinterpret_cast<float4*>(p.part + (slot * S::kRows + prow) * kDim + c * 32);
#pragma unroll
                            for (int i = 0; i < 8; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                        }
                    }
                    if (live && c_from == 0) {
                        if (!whole) p.part_ml[slot * S::kRows + prow] = make_float2(m_all, l_all);
                        else if (p.lse)
                            p.lse[int64_t(w.a.r.first + tok) * p.q_heads + hq] = l_all == 0.0f ? -INFINITY : (m_all + log2f(l_all)) * 0.69314718055994531f;
                    }
                }
                x0 += tiles;
                if (x0 >= x_end) break;
                tiles_before += tiles;
                ++unit;
                attend_next_unit(p, w);
            }
        } else if (warp < kTcMmaWarp) {
            // ============================================================ producers
            reg_dec<120>();
            const int pt = int(threadIdx.x) - kTcProducerWarp * 32;
            uint32_t bad_any = 0;
            while (true) {
                const int t0 = w.tile, t1 = int(min(int64_t(w.a.tiles), t0 + (x_end - x0)));
                const int tiles = t1 - t0;
                const int32_t* const table = p.batch.page_table + int64_t(w.b) * p.batch.table_stride;
                const int64_t len = w.a.len;
                const int pos_mask = (1 << p.cache.page_shift) - 1;
                const char* const head_base[2] = {p.cache.base[0] + int64_t(w.head) * p.cache.head_stride,
                                                  p.cache.base[1] + int64_t(w.head) * p.cache.head_stride};
                auto page_at = [&](int64_t pos) -> int {                     // page number, -1 without one
                    if (pos >= len) return -1;
                    const int page = table[pos >> p.cache.page_shift];
                    return page >= 0 && page < p.cache.pages ? page : -1;
                };
                // groups of 16 positions that should have a page and have none
                auto bad_groups = [&](int64_t pos0) -> uint32_t {
                    const int64_t pos = pos0 + (lane & 7) * 16;
                    return __ballot_sync(0xffffffffu, pos < len && page_at(pos) < 0) & 255u;
                };
                if (!kBf16) {
                    constexpr int kPieces = kDim / 16;                       // 16-byte pieces of a row of codes
                    constexpr int kRowsPer = 128 / kPieces;                  // rows one round of the 128 threads covers
                    const int piece = pt % kPieces, row0 = pt / kPieces;
                    uint4 raw[2][kPieces];
                    float sc[2];
                    int pages[kPieces], page_own;
                    auto find = [&](int n) {                                 // pages of tile n
                        const int64_t pos0 = int64_t(t0 + n) * kTcTile;
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) pages[i] = n < tiles ? page_at(pos0 + row0 + i * kRowsPer) : -1;
                        page_own = n < tiles ? page_at(pos0 + pt) : -1;
                    };
                    auto fetch = [&](int n, int which) {
                        const int64_t pos0 = int64_t(t0 + n) * kTcTile;
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) {
                            const int64_t pos = pos0 + row0 + i * kRowsPer;
                            raw[which][i] = make_uint4(0, 0, 0, 0);
                            if (pages[i] >= 0)
                                raw[which][i] = __ldg(reinterpret_cast<const uint4*>(head_base[which] + int64_t(pages[i]) * p.cache.page_stride +
                                                                                     (pos & pos_mask) * p.cache.token_stride + piece * 16));
                        }
                        sc[which] = 0.0f;
                        if (page_own >= 0)
                            sc[which] = __ldg(p.cache.scale[which] + int64_t(page_own) * p.cache.scale_page_stride + int64_t(w.head) * p.cache.scale_head_stride +
                                              ((pos0 + pt) & pos_mask));
                    };
                    auto store = [&](int which, char* base) {
                        const int atom = piece / 4;
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) {
                            const int row = row0 + i * kRowsPer;
                            uint32_t h[8];
                            codes4_to_f16<kFmt>(raw[which][i].x, h[0], h[1]);
                            codes4_to_f16<kFmt>(raw[which][i].y, h[2], h[3]);
                            codes4_to_f16<kFmt>(raw[which][i].z, h[4], h[5]);
                            codes4_to_f16<kFmt>(raw[which][i].w, h[6], h[7]);
                            const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
                            char* const at = base + atom * S::kAtomBytes + row * 128;
                            const int c = (piece & 3) * 2;
                            // (the two atoms of a row lie on the same banks: their threads store the halves in opposite order)
                            const int a = atom & 1;
                            *reinterpret_cast<uint4*>(at + (((c + a) ^ (row & 7)) << 4)) = a ? hi : lo;
                            *reinterpret_cast<uint4*>(at + (((c + 1 - a) ^ (row & 7)) << 4)) = a ? lo : hi;
                        }
                    };
                    find(0);
                    fetch(0, 0);
                    fetch(0, 1);
                    for (int n = 0; n < tiles; ++n) {
                        const uint32_t at = tiles_before + n;
                        const uint32_t ki = uint32_t(at % S::kKStages), vi = uint32_t(at % S::kVStages);
                        const uint32_t bad = bad_groups(int64_t(t0 + n) * kTcTile);
                        const float ks = sc[0], vs = sc[1];
                        find(n + 1);
                        alive = warp_wait(&bars.k_empty[ki], (uint32_t(at / S::kKStages) & 1u) ^ 1u);
                        if (!alive) break;
                        store(0, smem + S::kOffK + ki * S::kOperand);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.k_full[ki]);
                        if (n + 1 < tiles) fetch(n + 1, 0);
                        alive = warp_wait(&bars.v_empty[vi], (uint32_t(at / S::kVStages) & 1u) ^ 1u);
                        if (!alive) break;
                        store(1, smem + S::kOffV + vi * S::kOperand);
                        {
                            float* const to = scales + vi * 3 * kTcTile + pt;
                            const float v = vs >= 1e-30f ? vs : 1e-30f;          // a row of zero values keeps its weight in the sum
                            to[0] = ks;
                            to[kTcTile] = fmaf(vs, 0.0f, lg2(v));                // a NaN scale reaches the score alone
                            to[2 * kTcTile] = __fdividef(1.0f, v);
                        }
                        if (pt == 0) bars.meta[vi] = bad;
                        bad_any |= bad;
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.v_full[vi]);
                        if (n + 1 < tiles) fetch(n + 1, 1);
                    }
                } else {
                    for (int n = 0; n < tiles; ++n) {
                        const uint32_t at = tiles_before + n;
                        const int64_t pos0 = int64_t(t0 + n) * kTcTile;
                        const uint32_t stage[2] = {uint32_t(at % S::kKStages), uint32_t(at % S::kVStages)};
                        const uint32_t phase[2] = {(uint32_t(at / S::kKStages) & 1u) ^ 1u, (uint32_t(at / S::kVStages) & 1u) ^ 1u};
                        const uint32_t bad = bad_groups(pos0);
                        bad_any |= bad;
                        const bool plain = bad == 0 && pos0 + kTcTile <= w.a.r.start;     // whole, and the context's alone
#pragma unroll
                        for (int which = 0; which < 2; ++which) {
                            uint64_t* const full = which ? &bars.v_full[stage[1]] : &bars.k_full[stage[0]];
                            char* const dst = smem + (which ? S::kOffV : S::kOffK) + stage[which] * S::kOperand;
                            alive = alive && warp_wait(which ? &bars.v_empty[stage[1]] : &bars.k_empty[stage[0]], phase[which]);
                            if (!alive) break;
                            if (plain) {
                                if (which && pt == 0) bars.meta[stage[1]] = 0;
                                if (which && lane == 0) bars.odd[stage[1]][warp - kTcProducerWarp] = 0;
                                if (pt == 0) {
                                    mbar_arrive_expect_tx(full, S::kOperand);
                                    for (int t = 0; t < kTcTile; t += tp.box_tokens) {
                                        const int64_t pos = pos0 + t;
                                        const int page = page_at(pos);
                                        for (int a = 0; a < S::kAtoms; ++a)
                                            tma_load_4d(smem_u32(dst + a * S::kAtomBytes + t * 128), &tp.map[which], full, a * 64,
                                                        int(pos & pos_mask), w.head, page);
                                    }
                                } else if (lane == 0) {
                                    mbar_arrive(full);
                                }
                            } else {
                                bool odd = false;
                                constexpr int kPieces = kDim / 8;
                                const int piece = pt % kPieces;
#pragma unroll 4
                                for (int row = pt / kPieces; row < kTcTile; row += 128 / kPieces) {
                                    const int64_t pos = pos0 + row;
                                    const int page = page_at(pos);
                                    uint4 v = make_uint4(0, 0, 0, 0);
                                    if (page >= 0)
                                        v = __ldg(reinterpret_cast<const uint4*>(head_base[which] + int64_t(page) * p.cache.page_stride +
                                                                                 (pos & pos_mask) * p.cache.token_stride + piece * 16));
                                    if (which && pos >= w.a.r.start) {
                                        // values of the step's own tokens: rows differ in what they see, so what is not finite
                                        // stays out of the product (a weight of 0 would not keep it out)
                                        uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                        for (int i = 0; i < 4; ++i) {
                                            if ((u[i] & 0x7f80u) == 0x7f80u) u[i] &= 0xffff0000u, odd = true;
                                            if ((u[i] & 0x7f800000u) == 0x7f800000u) u[i] &= 0xffffu, odd = true;
                                        }
                                        v = make_uint4(u[0], u[1], u[2], u[3]);
                                    }
                                    *reinterpret_cast<uint4*>(dst + (piece / 8) * S::kAtomBytes + row * 128 + (((piece % 8) ^ (row & 7)) << 4)) = v;
                                }
                                const bool any_odd = __any_sync(0xffffffffu, odd) != 0;
                                if (which && pt == 0) bars.meta[stage[1]] = bad;
                                if (which && lane == 0) bars.odd[stage[1]][warp - kTcProducerWarp] = any_odd;
                                fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(full);
                            }
                        }
                        if (!alive) break;
                    }
                }
                if (w.a.r.cut) bad_any |= 1u;
                if (!alive) break;
                x0 += tiles;
                if (x0 >= x_end) break;
                tiles_before += tiles;
                attend_next_unit(p, w);
            }
            if (bad_any && pt == 0) atomicCAS(p.status, 0u, kBadPage);
        } else {
            // ============================================================ matrix instructions
            reg_dec<56>();
            if (warp == kTcMmaWarp && lane == 0) {
            const uint32_t kind = kBf16 ? (1u << 7) | (1u << 10) : 0u;
            const uint32_t idesc_s = (1u << 4) | kind | ((128u >> 3) << 17) | ((128u >> 4) << 24);
            const uint32_t idesc_o = (1u << 4) | kind | (1u << 16) | ((uint32_t(kDim) >> 3) << 17) | ((128u >> 4) << 24);
            const uint64_t k_hi = tc_desc_hi(16u, 1024u), v_hi = tc_desc_hi(uint32_t(S::kAtomBytes), 1024u);
            const uint32_t q_addr = smem_u32(smem), k_addr = smem_u32(smem + S::kOffK), v_addr = smem_u32(smem + S::kOffV);
            uint32_t p_phase = 0;                            // bit x: parity of stream x's next product
            auto desc = [](uint32_t addr, uint64_t hi) { return uint64_t((addr & 0x3FFFFu) >> 4) | hi; };
            auto scores = [&](int x, uint32_t stage) {
                const uint32_t q = q_addr + (kBlocks == 2 ? uint32_t(x) * S::kOperand : 0u), k = k_addr + stage * S::kOperand;
#pragma unroll
                for (int j = 0; j < kDim / 16; ++j) {
                    const uint32_t off = uint32_t(j >> 2) * S::kAtomBytes + uint32_t(j & 3) * 32u;
                    umma_bf16(tmem + S::kS + uint32_t(x) * 128u, desc(q + off, k_hi), desc(k + off, k_hi), idesc_s, j > 0);
                }
                umma_commit(&bars.s_full[x]);
            };
            auto values = [&](int x, uint32_t stage, bool first) {
                const uint32_t v = v_addr + stage * S::kOperand;
#pragma unroll
                for (int j = 0; j < kTcTile / 16; ++j)
                    umma_ts(tmem + S::kO + uint32_t(x) * 128u, tmem + S::kS + uint32_t(x) * 128u + uint32_t(j) * 8u,
                            desc(v + uint32_t(j) * 2048u, v_hi), idesc_o, j > 0 || !first);
                umma_commit(&bars.pv_done[x]);
            };
            auto k_wait = [&](uint32_t at) { return wait(&bars.k_full[at % S::kKStages], uint32_t(at / S::kKStages) & 1u); };
            auto v_wait = [&](uint32_t at) { return wait(&bars.v_full[at % S::kVStages], uint32_t(at / S::kVStages) & 1u); };
            while (true) {
                const int t0 = w.tile, t1 = int(min(int64_t(w.a.tiles), t0 + (x_end - x0)));
                const int tiles = t1 - t0;
                const int unit_rows = min(S::kRows, w.a.r.n * p.group - w.block * S::kRows);
                const int streams = kBlocks == 2 ? (unit_rows > 128 ? 2 : 1) : min(tiles, 2);
                alive = wait(&bars.q_full, unit & 1u);
                if (!alive) break;
                tc_fence_after_sync();
                // the first score tiles
                for (int x = 0; alive && x < streams; ++x) {
                    const uint32_t at = tiles_before + (kBlocks == 2 ? 0 : x);
                    if (kBlocks == 1 || x == 0) alive = k_wait(at);
                    if (!alive) break;
                    tc_fence_after_sync();
                    scores(x, uint32_t(at % S::kKStages));
                    if (kBlocks == 1 || x == streams - 1) umma_commit(&bars.k_empty[at % S::kKStages]);
                }
                for (int n = 0; alive && n < tiles; ++n) {
                    const uint32_t at = tiles_before + n;
                    const uint32_t vi = uint32_t(at % S::kVStages);
                    for (int x = kBlocks == 2 ? 0 : n & 1; alive && x < (kBlocks == 2 ? streams : (n & 1) + 1); ++x) {
                        alive = v_wait(at) && wait(&bars.p_full[x], p_phase >> x & 1u);
                        if (!alive) break;
                        tc_fence_after_sync();
                        values(x, vi, n < (kBlocks == 2 ? 1 : 2));
                        if (kBlocks == 1 || x == streams - 1) umma_commit(&bars.v_empty[vi]);
                        const int next = n + (kBlocks == 2 ? 1 : 2);
                        if (next < tiles) {
                            // the weights lie where the next scores go: that product has to be over
                            alive = wait(&bars.pv_done[x], p_phase >> x & 1u) && k_wait(tiles_before + next);
                            if (!alive) break;
                            tc_fence_after_sync();
                            const uint32_t ki = uint32_t((tiles_before + next) % S::kKStages);
                            scores(x, ki);
                            if (kBlocks == 1 || x == streams - 1) umma_commit(&bars.k_empty[ki]);
                        }
                        p_phase ^= 1u << x;
                    }
                }
                if (!alive) break;
                x0 += tiles;
                if (x0 >= x_end) break;
                tiles_before += tiles;
                ++unit;
                attend_next_unit(p, w);
            }
            // whatever was issued has to be over before tensor and shared memory are given back
            umma_commit(&bars.drained);
            const uint64_t since = global_timer_ns();
            while (!mbar_try_wait(&bars.drained, 0) && global_timer_ns() - since < 2 * tp.wait_ns) {}
            }
        }
        // a producer that gave up waits (with a limit) for its own copies in flight
        if (kBf16 && !alive && warp == kTcProducerWarp && lane == 0) {
            const uint64_t since = global_timer_ns();
            while (global_timer_ns() - since < 2000000ull) {}
        }
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kTcMmaWarp) tmem_dealloc(tmem, 512);
}

#endif  // __CUDACC__

}  // namespace tl
