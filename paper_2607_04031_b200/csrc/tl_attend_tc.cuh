// Attention for many query rows per key/value head (trees, chains of drafts, prompt chunks) on the 5th-generation
// tensor cores.
//
// One CTA per SM, five warpgroups: two for softmax (streams A and B), two of producers, and one whose first warp issues
// the matrix instructions; registers are moved from the last three to the first two.  A stream is an accumulator O
// (128 rows x dim) and a score tile S (128 x 128) in tensor memory.
//   kBlocks = 2  the streams hold different rows (256 rows a unit) and use every key/value tile together: each fetched
//                and converted element serves 256 rows;
//   kBlocks = 1  the streams hold the same 128 rows and take the tiles in turn; their sums are joined at the end.
// Either way one stream's products run while the other's softmax does.  Per tile and stream: S = Q K^T (both operands in
// shared memory, 128-byte swizzle), the warpgroup reads S, writes the weights back over it as 16-bit values, and O += P V
// takes P from tensor memory and V from shared memory as an MN-major operand, so neither P nor V^T is ever laid out again.
//
// A row's reference may lag behind its maximum (attend_head): only when a score exceeds it by more than 2^8 are O, the sum and the
// tile's earlier weights rescaled; sums are fp32 and f16 has room for the weights, so the lag costs no accuracy.  Rows are
// rescaled by their own scores alone: a row's bits do not depend on what its neighbours see.  Scales of 8-bit caches enter as
// in the kernel for few rows (key's scale on the score, value's in the exponent), q is f16 scaled by a power of two per row;
// conversion to f16 is exact.
//
// 8-bit tiles are fetched by the producers one tile ahead, converted and stored swizzled; full bf16 tiles
// come by TMA (128-byte-swizzled boxes, one per page and 64 dimensions); a tile with positions past the end, or with a
// page outside the pool, goes through registers too, with zeros in those places.
//
// Weights over a bf16 cache enter the second product as one bf16 value (8 bits; the kernel for few rows takes two terms): their
// error is about that of the result's own rounding, 2.3e-3 of the result together instead of 1.7e-3 (1 tree of 64 over 100000).  Two
// terms here, hence a second product: 1.66e-3, and 354 us instead of 284 to 297 there, 90 instead of 83 us for 8 requests of 256
// rows over 4100, 37 instead of 34 for 1.
//
// What bounds it: the floor is the larger of one reading of the cache and the two products.  1 tree of 64 over 100000 (512 rows,
// bf16): 312 to 328 us, 640 to 670 TFLOP/s; a step of two streams takes some 5200 clocks, 3500 of them a stream's softmax (bound by
// the latency of reading scores, exponentials and writing weights; the exponentials alone are 2048) and 1500 to 1700 from its last
// weight over the second product to the next scores.  8 trees of 32 over 8000 (216 rows a head, E4M3): 112 us, 400 TFLOP/s;
// 6300 to 6700 clocks a step, 30 % of a stream's time without scores and 6 % without values.  48 trees of 16 over 6000 (104 rows,
// INT8): 241 to 247 us, 2.0 TB/s; 4250 clocks per tile of 128 rows, the streams without values for 39 % of their time while the
// producers wait for 16 % of theirs: fetching and converting the codes bounds it.  Tensor pipe in use: 38, 28 and 25 % of the time.
#pragma once

#include "tl_attend.cuh"

namespace tl {

enum : uint32_t { kWaitAttend = 0xC00 };

constexpr int kTcTile = 128, kTcThreads = 20 * 32;
constexpr int kTcSoftmaxWarps = 8, kTcProducerWarp = 8, kTcProducers = 8, kTcMmaWarp = 16;
constexpr int kTcProducerThreads = kTcProducers * 32;
// Registers per thread: the launch has 96 for each of 640 threads, 61440; 256 x 120 + 256 x 88 + 128 x 64 is as many.
constexpr int kTcSoftmaxRegs = 120, kTcProducerRegs = 88, kTcMmaRegs = 64;
constexpr float kTcNoMax = -3.0e38f;     // in place of a maximum while a row has seen nothing

struct AttendTcParams {
    AttendParams a;
    CUtensorMap map[2];                  // keys, values (bf16 caches)
    int box_tokens;
    int stall;                           // test hook: CTA 0's first key tile is never announced
    uint64_t wait_ns;
};

template <int kDim, int kBlocks>
struct TcShape {
    static constexpr int kAtoms = kDim / 64;                       // 128-byte columns of a 16-bit operand tile
    static constexpr int kAtomBytes = kTcTile * 128;
    static constexpr int kOperand = kAtoms * kAtomBytes;           // one 128-row operand tile
    static constexpr int kKStages = 2, kVStages = 2;
    static constexpr int kOffK = kBlocks * kOperand;
    static constexpr int kOffV = kOffK + kKStages * kOperand;
    static constexpr int kOffScale = kOffV + kVStages * kOperand;  // [stage][ks, log2 vs, 1 / vs][128]
    static constexpr int kOffStat = kOffScale + kVStages * 3 * kTcTile * 4;
    static constexpr int kOffBar = kOffStat + (kBlocks == 1 ? 2 * kTcTile * 16 : 0);
    // 8-bit caches: codes on their way to conversion, 16 bytes per producer thread and round, one round kept in registers
    static constexpr int kRounds = kDim / 32;                      // of 256 threads x 16 bytes, per tile of keys or values
    static constexpr int kOffRaw = kOffBar + 256;
    static constexpr int kRawSlots = 2 * kRounds - 1;
    static constexpr int kSmem = kOffRaw + kRawSlots * 4096 + 1024;    // 1024: the base is aligned by hand
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
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
        : "memory");
}
// 16 lanes x 32 columns: thread (g = lane / 4, t = lane % 4) gets, of every 8 columns, columns 2t and 2t + 1 of lane g and
// of lane g + 8 (4 registers).
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}
// 16 lanes x 16 columns: of every 4 columns, thread (g, t) gives or gets column t of lane g and of lane g + 8.
__device__ __forceinline__ void tmem_st_16x128b_x4(uint32_t taddr, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_16x128b_x4(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.16x128b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

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
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t s_full[2], p_full[2], pv_done[2];
    uint64_t exchange;                   // 8 softmax warps: statistics of the two streams are in place
    uint64_t drained;                    // the issuing thread's last commit, when it gives up
    uint32_t abort_flag, tmem_base;
    uint32_t meta[2];                    // per value stage: groups of 16 positions that should have a page and have none
    alignas(8) uint8_t odd[2][kTcProducers];        // per value stage and producer warp: values that are not finite were taken out
};
static_assert(sizeof(TcBars) <= 256, "barrier block");

template <int kDim, int kFmt, int kBlocks>
__global__ void __launch_bounds__(kTcThreads, 1) attend_tc_kernel(const __grid_constant__ AttendTcParams tp) {
    using S = TcShape<kDim, kBlocks>;
    constexpr bool kBf16 = kFmt == TL_KV_BF16;
    constexpr float kHead = attend_head(kFmt);
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
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.k_full[i], kTcProducers);
            mbar_init(&bars.k_empty[i], 1);
            mbar_init(&bars.v_full[i], kTcProducers);
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
    int per, x0 = 0, x_end = 0;
    AttendPlace w;
    const bool work = attend_range(p, int(blockIdx.x), &per, &x0, &x_end, &w);

    auto wait = [&](uint64_t* bar, uint32_t parity) {
        return mbar_wait_bounded(bar, parity, abort_ptr, p.status, kWaitAttend, tp.wait_ns);
    };
    auto warp_wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };

    // The end of every role, each with a copy of its own: a common one would have the compiler hold all of them to the
    // smallest register share.
    auto leave = [&]() {
        __syncwarp();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (warp == kTcMmaWarp) tmem_dealloc(tmem, 512);
    };

    if (work) {
        uint32_t tiles_before = 0;                             // tiles of this CTA's earlier units: ring positions count on
        uint32_t unit = 0;
        bool alive = true;
        if (warp < kTcSoftmaxWarps) {
            // ============================================================ softmax
            // (every warpgroup of a CTA with work takes its share: together they are what the block was launched with)
            reg_inc<kTcSoftmaxRegs>();
            const int stream = warp / 4, r = int(threadIdx.x) & 127;
            const uint32_t lanes = uint32_t(warp & 3) * 32u << 16;           // this warp's quarter of tensor memory
            const uint32_t s_tmem = tmem + lanes + S::kS + uint32_t(stream) * 128u;
            const uint32_t o_tmem = tmem + lanes + S::kO + uint32_t(stream) * 128u;
            uint32_t s_count = 0;
            while (true) {
                const int t0 = w.tile, t1 = min(w.a.tiles, t0 + (x_end - x0));
                const int tiles = t1 - t0;
                const int unit_rows = min(S::kRows, w.a.r.n * p.group - w.block * S::kRows);
                const int row = w.block * S::kRows + (kBlocks == 2 ? stream * 128 : 0) + r;
                const bool live = row - w.block * S::kRows < unit_rows;
                const int tok = live ? row / p.group : 0, hq = w.head * p.group + (live ? row % p.group : 0);
                const bool active = kBlocks == 2 ? stream * 128 < unit_rows : stream < tiles;
                float fac = p.scale_log2;
                {
                    // this row of q, converted, into the operand tile (all of the row's loads in flight at once)
                    uint4 q[kDim / 8];
                    const uint4* src = reinterpret_cast<const uint4*>(p.q + int64_t(w.a.r.first + tok) * p.q_stride + int64_t(hq) * kDim);
#pragma unroll
                    for (int c = 0; c < kDim / 8; ++c) q[c] = __ldg(src + c);
                    float mul = 1.0f;
                    if (!kBf16) {
                        uint32_t top = 0;
#pragma unroll
                        for (int c = 0; c < kDim / 8; ++c) {
                            const uint32_t u[4] = {q[c].x, q[c].y, q[c].z, q[c].w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) top = __vmaxu2(top, u[i] & 0x7fff7fffu);       // two bf16 patterns at a time
                        }
                        const int e = int(max(top & 0xffffu, top >> 16) >> 7);
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
                            if (!live) v = make_uint4(0, 0, 0, 0);
                            *reinterpret_cast<uint4*>(dst + (c / 8) * S::kAtomBytes + (((c % 8) ^ (r & 7)) << 4)) = v;
                        }
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_full);

                // In the loop thread (g, t) holds rows g + 8h (h = 0..3) of its warp's 32 and columns 2t, 2t + 1 of every 8: the
                // four threads of a row share it, and a column's scales are fetched by the eight threads that need them.
                const int g = lane >> 2, t4 = lane & 3;
                float m[4], l[4], fac4[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    m[h] = kTcNoMax;
                    l[h] = 0.0f;
                    fac4[h] = __shfl_sync(0xffffffffu, fac, g + 8 * h);
                }
                // from there to one row per thread, for O
                auto to_row = [&](const float (&v)[4]) -> float {
                    float r0 = __shfl_sync(0xffffffffu, v[0], (lane & 7) * 4), r1 = __shfl_sync(0xffffffffu, v[1], (lane & 7) * 4);
                    float r2 = __shfl_sync(0xffffffffu, v[2], (lane & 7) * 4), r3 = __shfl_sync(0xffffffffu, v[3], (lane & 7) * 4);
                    r0 = lane & 8 ? r1 : r0;
                    r2 = lane & 8 ? r3 : r2;
                    return lane & 16 ? r2 : r0;
                };
                bool odd = false;
                // A stream without rows or tiles here keeps step with the other: ahead by two units, its arrivals alone would
                // complete the barrier for queries that are not in place.
                if (!active) {
                    alive = warp_wait(&bars.q_full, unit & 1u);
                    if (!alive) break;
                }
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
                    if (kFmt != TL_KV_INT8) odd |= *reinterpret_cast<const uint64_t*>(bars.odd[at]) != 0;
                    const int pos0 = (t0 + n) * kTcTile;
                    const bool edge = pos0 + kTcTile > w.a.r.start || meta != 0;
                    const float* const ks = scales + at * 3 * kTcTile + 2 * t4;
                    // bit i: this thread's row sees position pos0 + 32 c + i
                    auto sees32 = [&](int c) -> uint32_t {
                        const int pos = pos0 + c * 32;
                        if (pos >= w.a.r.len) return 0u;
                        uint32_t see = w.a.r.len - pos >= 32 ? 0xffffffffu : (1u << (w.a.r.len - pos)) - 1u;
                        if (meta & (1u << (2 * c))) see &= 0xffff0000u;
                        if (meta & (2u << (2 * c))) see &= 0x0000ffffu;
                        const int j = pos - w.a.r.start;                     // the step's token at bit 0
                        if (j + 31 < 0) return see;
                        auto word = [&](int k) -> uint32_t {                 // tokens 32 k .. 32 k + 31
                            if (k < 0) return 0xffffffffu;
                            if (p.mask) return k < p.mask_words ? p.mask[int64_t(w.a.r.first + tok) * p.mask_words + k] : 0u;
                            const int d = tok - k * 32;
                            return d >= 31 ? 0xffffffffu : d < 0 ? 0u : (2u << d) - 1u;
                        };
                        const int k = j >> 5;
                        return see & __funnelshift_r(word(k), word(k + 1), uint32_t(j & 31));
                    };
                    // The tile goes by in four pieces of 32 columns; the weights of a piece take the place of scores that have been
                    // read (16-bit values: half the columns).
                    F2 sum[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) sum[h] = F2{0.0f, 0.0f};
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        // scores in log2 units: d[h][i] are columns 32 c + 8 i + 2t + {0, 1} of row g + 8h
                        F2 d[4][4];
                        const float* const kc = ks + c * 32;
                        {
                            uint32_t v[2][16];
                            tmem_ld_16x256b_x4(s_tmem + uint32_t(c) * 32u, v[0]);
                            tmem_ld_16x256b_x4(s_tmem + (16u << 16) + uint32_t(c) * 32u, v[1]);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                F2 k2 = {1.0f, 1.0f}, v2 = {0.0f, 0.0f};
                                if (!kBf16) {
                                    k2 = *reinterpret_cast<const F2*>(kc + i * 8);
                                    v2 = *reinterpret_cast<const F2*>(kc + kTcTile + i * 8);
                                }
#pragma unroll
                                for (int h = 0; h < 4; ++h) {
                                    const F2 a = {__uint_as_float(v[h >> 1][4 * i + 2 * (h & 1)]), __uint_as_float(v[h >> 1][4 * i + 2 * (h & 1) + 1])};
                                    const F2 f = {fac4[h], fac4[h]};
                                    d[h][i] = kBf16 ? f2_mul(a, f) : f2_fma(f2_mul(a, k2), f, v2);
                                }
                            }
                        }
                        if (edge) {
                            const uint32_t see = sees32(c);
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                const uint32_t s4 = __shfl_sync(0xffffffffu, see, g + 8 * h) >> (2 * t4);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    if (!(s4 >> (8 * i) & 1u)) d[h][i].x = -INFINITY;
                                    if (!(s4 >> (8 * i) & 2u)) d[h][i].y = -INFINITY;
                                }
                            }
                        }
                        float top[4], over = kTcNoMax;                       // how far a score lies above its row's maximum
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            top[h] = fmaxf(fmaxf(d[h][0].x, d[h][0].y), fmaxf(d[h][1].x, d[h][1].y));
                            top[h] = fmaxf(top[h], fmaxf(fmaxf(d[h][2].x, d[h][2].y), fmaxf(d[h][3].x, d[h][3].y)));
                            over = fmaxf(over, top[h] - m[h]);
                        }
                        if (__any_sync(0xffffffffu, over > kLag + kHead)) {
                            // A new reference: what was taken against the old one is rescaled, by a whole power of two, so that weights that
                            // are rounded already are not rounded again.
                            float f[4];
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
                                top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
                                const bool up = top[h] > m[h] + (kLag + kHead);        // (by the row's own scores)
                                const float to = floorf(top[h]) - kHead;
                                f[h] = up ? ex2(m[h] - to) : 1.0f;
                                m[h] = up ? to : m[h];
                                l[h] *= f[h];
                                sum[h] = f2_mul(sum[h], F2{f[h], f[h]});
                            }
                            tmem_st_wait();
#pragma unroll 1
                            for (int k = 0; k < 2 * c; ++k) {                // this tile's weights so far
                                const uint32_t at_p = s_tmem + uint32_t(k & 1) * (16u << 16) + uint32_t(k >> 1) * 16u;
                                uint32_t pv[8];
                                tmem_ld_16x128b_x4(at_p, pv);
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const float fh = k & 1 ? (i & 1 ? f[3] : f[2]) : (i & 1 ? f[1] : f[0]);
                                    if (kBf16) {
                                        pv[i] = pack_bf16(__uint_as_float(pv[i] << 16) * fh, __uint_as_float(pv[i] & 0xffff0000u) * fh);
                                    } else {
                                        const float2 e = __half22float2(*reinterpret_cast<const __half2*>(&pv[i]));
                                        pv[i] = pack_f16(e.x * fh, e.y * fh);
                                    }
                                }
                                tmem_st_16x128b_x4(at_p, pv);
                            }
                            if (!first) {
                                // (S of this tile was issued after the previous O += P V had completed)
                                const float fr = to_row(f);
#pragma unroll 1
                                for (int k = 0; k < kDim / 16; ++k) {
                                    uint32_t o[16];
                                    tmem_ld_32x32b_x16(o_tmem + uint32_t(k) * 16u, o);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fr);
                                    tmem_st_32x32b_x16(o_tmem + uint32_t(k) * 16u, o);
                                }
                            }
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t pw[8];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                F2 r2 = {1.0f, 1.0f};
                                if (!kBf16) r2 = *reinterpret_cast<const F2*>(kc + 2 * kTcTile + i * 8);
#pragma unroll
                                for (int hh = 0; hh < 2; ++hh) {
                                    const int h = half * 2 + hh;
                                    const F2 x = f2_add(d[h][i], F2{-m[h], -m[h]});
                                    const F2 e = {ex2(x.x), ex2(x.y)};
                                    sum[h] = kBf16 ? f2_add(sum[h], e) : f2_fma(e, r2, sum[h]);
                                    pw[2 * i + hh] = kBf16 ? pack_bf16(e.x, e.y) : pack_f16(e.x, e.y);
                                }
                            }
                            tmem_st_16x128b_x4(s_tmem + uint32_t(half) * (16u << 16) + uint32_t(c) * 16u, pw);
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 4; ++h) l[h] += sum[h].x + sum[h].y;
                    tmem_st_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.p_full[stream]);
                }
                if (!alive) break;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
                    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
                }
                const float m_row = to_row(m), l_row = to_row(l);
                // the last product of this stream
                if (active) {
                    alive = warp_wait(&bars.pv_done[stream], (s_count - 1) & 1u);
                    if (!alive) break;
                    tc_fence_after_sync();
                }
                float f_own = 1.0f, f_other = 0.0f, m_all = m_row, l_all = l_row;
                bool odd_all = odd;
                if (kBlocks == 1) {
                    stats[stream * kTcTile + r] = make_float4(m_row, l_row, odd ? 1.0f : 0.0f, 0.0f);
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.exchange);
                    alive = warp_wait(&bars.exchange, unit & 1u);
                    if (!alive) break;
                    tc_fence_after_sync();
                    const float4 o = stats[(stream ^ 1) * kTcTile + r];
                    m_all = fmaxf(m_row, o.x);
                    const float use = m_all == -INFINITY ? 0.0f : m_all;
                    f_own = ex2(m_row - use);
                    f_other = ex2(o.x - use);
                    l_all = l_row * f_own + o.y * f_other;
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
                            const int from = max(w.a.r.start, t0 * kTcTile), to = min(w.a.r.len, t1 * kTcTile);
                            for (int pos = from; pos < to; ++pos) {
                                if (!attend_sees(p, w.a.r.first + tok, tok, pos - w.a.r.start)) continue;
                                const int page = p.batch.page_table[int64_t(w.b) * p.batch.table_stride + (pos >> p.cache.page_shift)];
                                if (page < 0 || page >= p.cache.pages) continue;
                                const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                                    p.cache.base[1] + int64_t(page) * p.cache.page_stride + int64_t(w.head) * p.cache.head_stride +
                                    int64_t(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride) + c * 32;
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
                    if (kFmt == TL_KV_E4M3 && odd_all && live) {
                        // NaN codes alike: what this row sees of them, over what has just been written
                        const int from = max(w.a.r.start, t0 * kTcTile), to = min(w.a.r.len, t1 * kTcTile);
#pragma unroll 1
                        for (int pos = from; pos < to; ++pos) {
                            if (!attend_sees(p, w.a.r.first + tok, tok, pos - w.a.r.start)) continue;
                            const int page = p.batch.page_table[int64_t(w.b) * p.batch.table_stride + (pos >> p.cache.page_shift)];
                            if (page < 0 || page >= p.cache.pages) continue;
                            const char* const codes = p.cache.base[1] + int64_t(page) * p.cache.page_stride + int64_t(w.head) * p.cache.head_stride +
                                                      int64_t(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride;
#pragma unroll 1
                            for (int i = c_from * 32; i < c_to * 32; ++i) {
                                if ((codes[i] & 0x7f) != 0x7f) continue;
                                if (whole) p.out[int64_t(w.a.r.first + tok) * p.out_stride + int64_t(hq) * kDim + i] = __ushort_as_bfloat16(0x7fff);
                                else p.part[(slot * S::kRows + prow) * kDim + i] = __uint_as_float(0x7fc00000u);
                            }
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
            leave();
            return;
        } else if (warp < kTcMmaWarp) {
            // ============================================================ producers
            reg_dec<kTcProducerRegs>();
            const int pt = int(threadIdx.x) - kTcProducerWarp * 32;
            uint32_t bad_any = 0;
            while (true) {
                const int t0 = w.tile, t1 = min(w.a.tiles, t0 + (x_end - x0));
                const int tiles = t1 - t0;
                const int32_t* const table = p.batch.page_table + int64_t(w.b) * p.batch.table_stride;
                const int len = w.a.r.len;
                const int pos_mask = (1 << p.cache.page_shift) - 1;
                const char* const head_base[2] = {p.cache.base[0] + int64_t(w.head) * p.cache.head_stride,
                                                  p.cache.base[1] + int64_t(w.head) * p.cache.head_stride};
                // Page numbers of four tiles, one group of 16 positions per lane (-1: no page), and the next four on the way.
                // (Entries are checked when their turn comes: here they would be waited for.)
                auto there = [&](int n) { return n + (lane >> 3) < tiles && (t0 + n) * kTcTile + lane * 16 < len; };
                auto load_pages = [&](int n) -> int { return __ldg(table + (there(n) ? ((t0 + n) * kTcTile + lane * 16) >> p.cache.page_shift : 0)); };
                int pages = 0, pages_next = load_pages(0);
                int64_t place = 0;                                           // byte offset of the lane's group in the pool
                auto turn_to = [&](int n) {                                  // tile n (one after the other)
                    if ((n & 3) != 0) return;
                    pages = there(n) && pages_next >= 0 && pages_next < p.cache.pages ? pages_next : -1;
                    pages_next = load_pages(n + 4);
                    place = pages < 0 ? -1 : int64_t(pages) * p.cache.page_stride + int64_t(((t0 + n) * kTcTile + lane * 16) & pos_mask) * p.cache.token_stride;
                };
                auto page_of = [&](int n, int group) { return __shfl_sync(0xffffffffu, pages, (n & 3) * 8 + group); };
                auto place_of = [&](int n, int group) { return __shfl_sync(0xffffffffu, place, (n & 3) * 8 + group); };
                // groups of tile n without a page, as far as the sequence reaches
                auto bad_groups = [&](int n) -> uint32_t {
                    const bool bad = pages < 0 && (t0 + (n & ~3)) * kTcTile + lane * 16 < len;
                    return (__ballot_sync(0xffffffffu, bad) >> ((n & 3) * 8)) & 255u;
                };
                if (!kBf16) {
                    constexpr int kPieces = kDim / 16;                       // 16-byte pieces of a row of codes
                    constexpr int kRowsPer = kTcProducerThreads / kPieces;   // rows one round of the threads covers
                    constexpr int kRounds = S::kRounds;
                    static_assert(kRounds * kRowsPer == kTcTile, "rounds");
                    char* const raw_gen = smem + S::kOffRaw + pt * 16;
                    const uint32_t raw_mem = smem_u32(raw_gen);
                    // Eight neighbouring lanes cover four pieces of two rows: their stores of the swizzled halves fall on
                    // different banks (the two 64-dimension atoms of a row lie on the same ones).
                    const int piece = kPieces == 8 ? (lane & 3) | (lane >> 4) << 2 : lane & 3;
                    const int row0 = kPieces == 8 ? (pt >> 5) * 4 + ((lane >> 2) & 3) : pt >> 2;
                    const uint32_t within = uint32_t(row0 & 15) * uint32_t(p.cache.token_stride) + uint32_t(piece) * 16u;
                    const int scale_row = pt & 127, scale_of = pt >> 7;      // half of the threads fetch keys' scales, half values'
                    uint4 last = make_uint4(0, 0, 0, 0);                     // the values' last round
                    float sc = 0.0f;
                    bool sc_lack = false;
                    bool lack = false;                                       // its row does not exist
                    // (Whole warp; the tile that `pages` has been turned to.)  Codes wait in shared memory, in slots that only this
                    // thread uses (a load's destination there takes no line of the first-level cache, which is small beside
                    // this kernel's shared memory); the last round, for which there is no slot, waits in registers.  Positions
                    // without a row are filled with zeros.
                    int64_t from[kRounds];                                   // of tile n + 1: byte offset in the pool, -1 without a row
                    auto locate = [&](int n) {
                        const int pos0 = (t0 + n) * kTcTile;
#pragma unroll
                        for (int i = 0; i < kRounds; ++i) {
                            const int row = row0 + i * kRowsPer;
                            const int64_t at = place_of(n, row >> 4);
                            from[i] = at >= 0 && pos0 + row < len ? at + within : -1;
                        }
                    };
                    auto fetch = [&](int which) {
#pragma unroll
                        for (int i = 0; i < kRounds; ++i) {
                            const bool in = from[i] >= 0;
                            const char* const src = head_base[which] + (in ? from[i] : 0);
                            if (which * kRounds + i < S::kRawSlots) {
                                cp_async_16(raw_mem + uint32_t(which * kRounds + i) * 4096u, src, in);
                            } else {
                                last = __ldg(reinterpret_cast<const uint4*>(src));
                                lack = !in;
                            }
                        }
                        cp_async_commit();
                    };
                    auto fetch_scale = [&](int n) {
                        const int pos = (t0 + n) * kTcTile + scale_row;
                        const int page = page_of(n, scale_row >> 4);
                        const bool in = page >= 0 && pos < len;
                        sc = __ldg(p.cache.scale[scale_of] + int64_t(in ? page : 0) * p.cache.scale_page_stride + int64_t(w.head) * p.cache.scale_head_stride +
                                   (in ? pos & pos_mask : 0));
                        sc_lack = !in;                                       // (zeroed at its use: here it would be waited for)
                    };
                    // Values of a tile whose rows from own_from on are the step's own tokens.  Query rows differ in what they see of those,
                    // so an E4M3 NaN stays out of the product (a weight of 0 would not keep it out).  True: there was one.
                    auto take_nan_out = [&](int own_from) -> bool {
                        auto clean = [](uint4& v) -> bool {
                            if (__builtin_expect((e4m3_nan_bits(v.x) | e4m3_nan_bits(v.y) | e4m3_nan_bits(v.z) | e4m3_nan_bits(v.w)) == 0, 1)) return false;
                            v = make_uint4(v.x & ~e4m3_nan_bytes(v.x), v.y & ~e4m3_nan_bytes(v.y), v.z & ~e4m3_nan_bytes(v.z), v.w & ~e4m3_nan_bytes(v.w));
                            return true;
                        };
                        bool odd = row0 + (kRounds - 1) * kRowsPer >= own_from && !lack && clean(last);
#pragma unroll 1
                        for (int i = 0; i < kRounds - 1; ++i)
                            if (row0 + i * kRowsPer >= own_from) odd |= clean(*reinterpret_cast<uint4*>(raw_gen + (kRounds + i) * 4096));
                        return odd;
                    };
                    auto store = [&](int which, char* base) {
                        const int c = (piece & 3) * 2;
                        char* const at0 = base + (piece >> 2) * S::kAtomBytes + row0 * 128 + ((c ^ (row0 & 7)) << 4);
                        char* const at1 = base + (piece >> 2) * S::kAtomBytes + row0 * 128 + (((c + 1) ^ (row0 & 7)) << 4);
#pragma unroll
                        for (int i = 0; i < kRounds; ++i) {
                            uint4 raw;
                            if (which * kRounds + i < S::kRawSlots) raw = *reinterpret_cast<const uint4*>(raw_gen + (which * kRounds + i) * 4096);
                            else raw = lack ? make_uint4(0, 0, 0, 0) : last;
                            uint32_t h[8];
                            codes4_to_f16<kFmt>(raw.x, h[0], h[1]);
                            codes4_to_f16<kFmt>(raw.y, h[2], h[3]);
                            codes4_to_f16<kFmt>(raw.z, h[4], h[5]);
                            codes4_to_f16<kFmt>(raw.w, h[6], h[7]);
                            *reinterpret_cast<uint4*>(at0 + i * kRowsPer * 128) = make_uint4(h[0], h[1], h[2], h[3]);      // (kRowsPer: a multiple of 8)
                            *reinterpret_cast<uint4*>(at1 + i * kRowsPer * 128) = make_uint4(h[4], h[5], h[6], h[7]);
                        }
                    };
                    // one round ahead: tile n + 1 is asked for while tile n is stored
#pragma unroll 1
                    for (int n = -1; n < tiles; ++n) {
                        const uint32_t at = tiles_before + n;
                        const uint32_t ki = at % S::kKStages, vi = at % S::kVStages;
                        const bool more = n + 1 < tiles;
                        uint32_t bad = 0;
                        if (n >= 0) {
                            bad = bad_groups(n);
                            alive = warp_wait(&bars.k_empty[ki], ((at / S::kKStages) & 1u) ^ 1u);
                            if (!alive) break;
                            cp_async_wait<1>();                              // (the keys were asked for before the values)
                            store(0, smem + S::kOffK + ki * S::kOperand);
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0 && !(tp.stall && blockIdx.x == 0 && pt == 0 && at == 0)) mbar_arrive(&bars.k_full[ki]);
                        }
                        if (more) {
                            turn_to(n + 1);
                            locate(n + 1);
                            fetch(0);
                        } else {
                            cp_async_commit();
                        }
                        if (n >= 0) {
                            alive = warp_wait(&bars.v_empty[vi], ((at / S::kVStages) & 1u) ^ 1u);
                            if (!alive) break;
                            cp_async_wait<1>();
                            const int own_from = w.a.r.start - (t0 + n) * kTcTile;
                            const bool odd = kFmt == TL_KV_E4M3 && own_from < kTcTile && take_nan_out(own_from);
                            store(1, smem + S::kOffV + vi * S::kOperand);
                            float* const to = scales + vi * 3 * kTcTile + scale_row;
                            const float s_now = sc_lack ? 0.0f : sc;
                            if (scale_of == 0) {
                                to[0] = s_now;
                            } else {
                                const float v = s_now >= kScaleFloor ? s_now : kScaleFloor;    // a row of zero values keeps its weight in the sum
                                to[kTcTile] = fmaf(s_now, 0.0f, lg2(v));             // a NaN scale reaches the score alone
                                to[2 * kTcTile] = __fdividef(1.0f, v);
                            }
                            if (pt == 0) bars.meta[vi] = bad;
                            bad_any |= bad;
                            const bool any_odd = kFmt == TL_KV_E4M3 && __any_sync(0xffffffffu, odd) != 0;
                            if (kFmt == TL_KV_E4M3 && lane == 0) bars.odd[vi][warp - kTcProducerWarp] = any_odd;
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&bars.v_full[vi]);
                        }
                        if (more) {
                            fetch(1);
                            fetch_scale(n + 1);                              // (behind the use of the last one: a copy of it would be waited for)
                        }
                    }
                } else {
#pragma unroll 1
                    for (int n = 0; n < tiles; ++n) {
                        const uint32_t at = tiles_before + n;
                        const int pos0 = (t0 + n) * kTcTile;
                        const uint32_t ki = at % S::kKStages, vi = at % S::kVStages;
                        turn_to(n);
                        const uint32_t bad = bad_groups(n);
                        bad_any |= bad;
                        const bool plain = bad == 0 && pos0 + kTcTile <= w.a.r.start;     // whole, and the context's alone
#pragma unroll 1
                        for (int which = 0; which < 2; ++which) {
                            uint64_t* const full = which ? &bars.v_full[vi] : &bars.k_full[ki];
                            char* const dst = smem + (which ? S::kOffV + vi * S::kOperand : S::kOffK + ki * S::kOperand);
                            alive = which ? warp_wait(&bars.v_empty[vi], ((at / S::kVStages) & 1u) ^ 1u)
                                          : warp_wait(&bars.k_empty[ki], ((at / S::kKStages) & 1u) ^ 1u);
                            if (!alive) break;
                            bool odd = false;
                            if (plain) {
                                // one box per lane, spread over the warps: an instruction holds its thread for some 100 clocks
                                if (pt == 0) {
                                    if (which) bars.meta[vi] = 0, bars.odd[vi][0] = 0;   // (ahead of this thread's arrival)
                                    mbar_arrive_expect_tx(full, S::kOperand);
                                }
                                const int k = lane * kTcProducers + warp - kTcProducerWarp;
                                const int t = k / S::kAtoms * 16, a = k % S::kAtoms;
                                const int page = page_of(n, (t >> 4) & 7);
                                if (t < kTcTile && (t & (tp.box_tokens - 1)) == 0)
                                    tma_load_4d(smem_u32(dst + a * S::kAtomBytes + t * 128), &tp.map[which], full, a * 64, (pos0 + t) & pos_mask, w.head, page);
                            } else {
                                constexpr int kPieces = kDim / 8;
                                const int piece = pt % kPieces;
#pragma unroll 4
                                for (int row = pt / kPieces; row < kTcTile; row += kTcProducerThreads / kPieces) {
                                    const int pos = pos0 + row;
                                    const int64_t at = place_of(n, row >> 4);
                                    const bool in = at >= 0 && pos < len;
                                    const int64_t off = in ? at + uint32_t(row & 15) * uint32_t(p.cache.token_stride) : 0;
                                    uint4 v = __ldg(reinterpret_cast<const uint4*>(head_base[which] + off + piece * 16));
                                    if (!in) v = make_uint4(0, 0, 0, 0);
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
                                fence_proxy_async_smem();
                            }
                            const bool any_odd = __any_sync(0xffffffffu, odd) != 0;
                            if (which && pt == 0 && !plain) bars.meta[vi] = bad;
                            if (which && lane == 0 && !(plain && pt == 0)) bars.odd[vi][warp - kTcProducerWarp] = any_odd;
                            __syncwarp();
                            if (lane == 0 && !(plain && pt == 0) && !(tp.stall && blockIdx.x == 0 && pt == 32 && at == 0 && which == 0)) mbar_arrive(full);
                        }
                        if (!alive) break;
                    }
                }
                if (w.a.r.n > w.a.r.len - w.a.r.start) bad_any |= 1u;
                if (!alive) break;
                x0 += tiles;
                if (x0 >= x_end) break;
                tiles_before += tiles;
                attend_next_unit(p, w);
            }
            if (bad_any && pt == 0) atomicCAS(p.status, 0u, kBadPage);
            if (!kBf16) cp_async_wait<0>();
            if (kBf16 && !alive) {                             // gave up: wait (with a limit) for the copies in flight
                const uint64_t since = global_timer_ns();
                while (global_timer_ns() - since < 2000000ull) {}
            }
            leave();
            return;
        } else {
            // ============================================================ matrix instructions
            reg_dec<kTcMmaRegs>();
            if (warp == kTcMmaWarp && lane == 0) {
            constexpr uint32_t kind = kBf16 ? (1u << 7) | (1u << 10) : 0u;
            constexpr uint32_t idesc_s = (1u << 4) | kind | ((128u >> 3) << 17) | ((128u >> 4) << 24);
            constexpr uint32_t idesc_o = (1u << 4) | kind | (1u << 16) | ((uint32_t(kDim) >> 3) << 17) | ((128u >> 4) << 24);
            // Operand descriptors in halves: the issuing thread is alone in its warp and every instruction between two
            // products costs it several clocks, so a step adds a constant to a word that is otherwise ready.
            // (128-byte swizzle, descriptor version 1; 8-row groups 1024 bytes apart; V's 64-column atoms kAtomBytes apart)
            constexpr uint32_t kHi = (1024u >> 4) | 1u << 14 | 2u << 29;
            constexpr uint32_t kStep = uint32_t(S::kOperand) >> 4;
            const uint32_t q_lo = (smem_u32(smem) >> 4) | 1u << 16, k_lo = (smem_u32(smem + S::kOffK) >> 4) | 1u << 16;
            const uint32_t v_lo = (smem_u32(smem + S::kOffV) >> 4) | uint32_t(S::kAtomBytes >> 4) << 16;
            uint32_t p_phase = 0;                            // bit x: parity of stream x's next product
            auto scores = [&](int x, uint32_t stage) {
                const uint32_t q = q_lo + (kBlocks == 2 ? uint32_t(x) * kStep : 0u), k = k_lo + stage * kStep, to = tmem + S::kS + uint32_t(x) * 128u;
#pragma unroll
                for (int j = 0; j < kDim / 16; ++j) {
                    constexpr uint32_t kAtom = uint32_t(S::kAtomBytes) >> 4;
                    const uint32_t off = uint32_t(j >> 2) * kAtom + uint32_t(j & 3) * 2u;
                    umma_split<false>(to, q + off, kHi, k + off, kHi, idesc_s, j > 0);
                }
                umma_commit(&bars.s_full[x]);
            };
            auto values = [&](int x, uint32_t stage, uint32_t go_on) {
                const uint32_t v = v_lo + stage * kStep, to = tmem + S::kO + uint32_t(x) * 128u, from = tmem + S::kS + uint32_t(x) * 128u;
#pragma unroll
                for (int j = 0; j < kTcTile / 16; ++j)
                    umma_ts(to, from + uint32_t(j) * 8u, v + uint32_t(j) * (2048u >> 4), kHi, idesc_o, j > 0 ? 1u : go_on);
                umma_commit(&bars.pv_done[x]);
            };
            auto k_wait = [&](uint32_t at) { return wait(&bars.k_full[at % S::kKStages], uint32_t(at / S::kKStages) & 1u); };
            auto v_wait = [&](uint32_t at) { return wait(&bars.v_full[at % S::kVStages], uint32_t(at / S::kVStages) & 1u); };
            while (true) {
                const int t0 = w.tile, t1 = min(w.a.tiles, t0 + (x_end - x0));
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
                        values(x, vi, n >= (kBlocks == 2 ? 1 : 2));
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
            leave();
            return;
        }
    }
    leave();
}

#endif  // __CUDACC__

}  // namespace tl
