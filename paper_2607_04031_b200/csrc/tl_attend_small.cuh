// Attention for few query rows per key/value head (decoding, short chains, small trees).
//
// One pass over the cache with a running maximum and sum.  Every warp owns 16 positions of a tile and all rows of the
// unit (16 or 32), so each cache element is fetched and converted by exactly one thread of the machine and no barrier
// stands inside the loop; the warps' sums are joined once per unit.
//
// Operands reach the matrix instruction without a trip through a shared layout.  The contraction index of q k^T (the
// head dimension) may be permuted as long as q is permuted alike, and so may the output columns of p v: thread
// (g = lane / 4, t = lane % 4) therefore loads whole 16-byte pieces of the rows it needs (tokens g and g + 8 for
// q k^T, tokens 2t, 2t+1, 2t+8, 2t+9 for p v) with cp.async into slots that only it reads, several tiles ahead, and
// its registers are the instruction's B fragments after the conversion:
//   q k^T: 4 consecutive codes of a token are the fragment of one 16-deep step;
//   p v:   codes of two tokens at the same dimensions, interleaved bytewise, are one fragment pair each.
// 8-bit codes become f16 (exact for both formats), q becomes f16 scaled by a power of two per row (exact but for
// elements 2^-31 below the row's largest).  The key's scale multiplies the score.  The value's scale goes into the
// exponent, w_j = 2^(s_j + log2 vs_j - m), with m following the maximum of s_j + log2 vs_j (attend_head): w is as exact as f16
// can be where the contribution w_j v_j is large, and the softmax sum is that of w_j / vs_j.  The second product
// takes w rounded to f16 (11 bits) with 8-bit caches, and as two bf16 terms (16 bits) with bf16 caches, whose eight bits
// alone would put as much error into the result as its own rounding does; the sum takes w in fp32.
//
// What bounds it: the floor is one reading of the cache.  32 requests of one token (8 rows a head) over 4100 positions, E4M3:
// 61.2 us, 3.4 TB/s, 0.53 of a plain copy; every byte is read once, the issue slots are 37 % in use and DRAM 43 %: the chain
// from scores over maximum and exponential to the second product, with the 12 warps per SM that its registers allow.
#pragma once

#include "tl_attend.cuh"

namespace tl {

struct SmallYes { static constexpr bool value = true; };
struct SmallNo { static constexpr bool value = false; };

template <int kDim, int kFmt, int kMT>
struct SmallShape {
    static constexpr bool kBf16 = kFmt == TL_KV_BF16;
    static constexpr int kItem = kBf16 ? 2 : 1;
    static constexpr float kHead = attend_head(kFmt);
    static constexpr int kRowBytes = kDim * kItem;
    static constexpr int kCtasPerSm = kMT == 1 && kRowBytes == 128 ? 3 : kMT == 1 && kRowBytes < 128 ? 2 : 1;
    static constexpr int kWarps = kDim == 256 || kCtasPerSm == 3 ? 4 : 8;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kRows = kMT * 16;
    static constexpr int kTile = kWarps * 16;
    static constexpr int kSteps = kDim / 16;                       // 16-deep steps of q k^T
    static constexpr int kKChunks = kRowBytes / 64;                // 16-byte pieces of a token per thread (4 threads a row)
    static constexpr int kVBytes = kRowBytes / 8 < 16 ? kRowBytes / 8 : 16;
    static constexpr int kVChunks = kRowBytes / 8 / kVBytes;       // pieces of a token per thread (8 threads a row)
    static constexpr int kNTiles = kDim / 8;                       // 8-wide column tiles of p v
    static constexpr int kStageBytes = 32 * kRowBytes + 128;       // one warp's 16 tokens, keys and values, and the scales
    static constexpr int kSub = kMT == 1 && kRowBytes <= 128 ? 2 : 1;   // sub-tiles a warp takes at a time
    static constexpr int kQBytes = kMT * kSteps * 512;
    static constexpr int kStatBytes = (kWarps * kRows * 2 + kRows * 4) * 4;
    static constexpr int kLimit = (kCtasPerSm == 3 ? 74 : kCtasPerSm == 2 ? 112 : 225) * 1024;
    static constexpr int kBudget = kLimit - kQBytes - kStatBytes;
    static constexpr int kStagesFit = kBudget / (kWarps * kStageBytes);
    static constexpr int kStages = kStagesFit > 6 ? 6 : kStagesFit;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kJoin = kWarps * kRows * kDim * 4;
    static constexpr int kUnion = kRing > kJoin ? kRing : kJoin;   // the ring's memory also serves the join
    static constexpr int kSmem = kUnion + kQBytes + kStatBytes;
    static_assert(kStages >= 2 * kSub, "no room for the stages ahead");
    static_assert(kSmem <= kLimit, "shared memory");
};

template <int kDim, int kFmt, int kMT>
__global__ void __launch_bounds__(SmallShape<kDim, kFmt, kMT>::kThreads, SmallShape<kDim, kFmt, kMT>::kCtasPerSm)
attend_kernel(const AttendParams p) {
    using S = SmallShape<kDim, kFmt, kMT>;
    constexpr bool kBf16 = S::kBf16;
    extern __shared__ __align__(128) char smem[];
    float* const join = reinterpret_cast<float*>(smem);
    uint4* const q_frag = reinterpret_cast<uint4*>(smem + S::kUnion);                 // [mt][step][lane]
    float* const stat_m = reinterpret_cast<float*>(smem + S::kUnion + S::kQBytes);    // [warp][row]
    float* const stat_l = stat_m + S::kWarps * S::kRows;
    float* const row_fac = stat_l + S::kWarps * S::kRows;                             // [row]
    float* const row_m = row_fac + S::kRows;                                          // [row] joined maximum and sum
    float* const row_l = row_m + S::kRows;
    float* const nan_taken = row_l + S::kRows;                                        // E4M3: not 0 when NaN codes were taken out
    const int lane = int(lane_id()), warp = int(threadIdx.x) / 32, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + uint32_t(warp * S::kStages * S::kStageBytes);
    const char* const ring_gen = smem + warp * S::kStages * S::kStageBytes;

    pdl_wait();
    pdl_launch_dependents();
    int per, x = 0, x_end = 0;
    AttendPlace w;
    const bool work = attend_range(p, int(blockIdx.x), &per, &x, &x_end, &w);
    if (!work) return;

    while (true) {
        const int t0 = w.tile, t1 = min(w.a.tiles, t0 + (x_end - x));
        const int rows = min(S::kRows, w.a.r.n * p.group - w.block * S::kRows);
        const int32_t* const table = p.batch.page_table + int64_t(w.b) * p.batch.table_stride;
        const char* const k_head = p.cache.base[0] + int64_t(w.head) * p.cache.head_stride;
        const char* const v_head = p.cache.base[1] + int64_t(w.head) * p.cache.head_stride;
        const int len = w.a.r.len, start = w.a.r.start;
        const int pos_mask = (1 << p.cache.page_shift) - 1;

        // this warp's sub-tiles: positions (t0 + i) * kTile + warp * 16, for i = 0 .. count - 1 (those that begin inside)
        const int pos_first = t0 * S::kTile + warp * 16;
        int count = t1 - t0;
        if (pos_first + (count - 1) * S::kTile >= len) --count;          // only the unit's last tile can begin past the end
        // Page numbers of 32 sub-tiles, one per lane, and the next 32 on the way (checked when their turn comes: where they
        // are asked for they would be waited for).
        auto load_page = [&](int i) -> int { return __ldg(table + (i < count ? (pos_first + i * S::kTile) >> p.cache.page_shift : 0)); };
        auto checked = [&](int page, int i) { return i < count && page >= 0 && page < p.cache.pages ? page : -1; };
        int pages = load_page(lane), pages_next = load_page(lane + 32);
        pages = checked(pages, lane);
        uint32_t bad_any = 0;
        // (offsets within a sub-tile fit 32 bits: the host bounds the token stride)
        const uint32_t ts = uint32_t(p.cache.token_stride);
        const uint32_t k_off = uint32_t(g) * ts + uint32_t(t) * 16u, v_off = uint32_t(2 * t) * ts + uint32_t(g) * uint32_t(S::kVBytes);
        auto issue = [&](int i) {                                        // starts the copies of sub-tile i (whole warp, i upwards)
            if (i < count) {
                if (i > 0 && (i & 31) == 0) {
                    pages = checked(pages_next, i + lane);
                    pages_next = load_page(i + 32 + lane);
                }
                const int page = __shfl_sync(0xffffffffu, pages, i & 31);
                const bool ok = page >= 0;
                bad_any |= ok ? 0u : 1u;
                const int pos = pos_first + i * S::kTile;
                const int line = pos & pos_mask;
                const int left = ok ? len - pos : 0;
                const int64_t at = ok ? int64_t(page) * p.cache.page_stride + int64_t(line) * p.cache.token_stride : 0;
                const char* const k_at = k_head + at;
                const char* const v_at = v_head + at;
                const uint32_t dst = ring + uint32_t((i % S::kStages) * S::kStageBytes);
                auto copy = [&](auto whole) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool in = decltype(whole)::value || g + 8 * h < left;
                        const char* src = in ? k_at + (k_off + uint32_t(8 * h) * ts) : k_head;
#pragma unroll
                        for (int c = 0; c < S::kKChunks; ++c)
                            cp_async_16(dst + uint32_t((h * S::kKChunks + c) * 512 + lane * 16), src + c * 64, in);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int more = (k & 1) + 8 * (k >> 1);
                        const bool in = decltype(whole)::value || 2 * t + more < left;
                        const char* src = in ? v_at + (v_off + uint32_t(more) * ts) : v_head;
#pragma unroll
                        for (int c = 0; c < S::kVChunks; ++c) {
                            const uint32_t to = dst + uint32_t(16 * S::kRowBytes + (k * S::kVChunks + c) * 32 * S::kVBytes + lane * S::kVBytes);
                            if (S::kVBytes == 16) cp_async_16(to, src + c * 128, in);
                            else cp_async_8(to, src, in);
                        }
                    }
                };
                if (left >= 16) copy(SmallYes{});
                else copy(SmallNo{});
                if (!kBf16 && lane < 8) {
                    // (the scales of a page's 16 tokens are read whole; those past the end belong to masked positions)
                    const float* sc = p.cache.scale[lane >> 2] + (ok ? int64_t(page) * p.cache.scale_page_stride + int64_t(w.head) * p.cache.scale_head_stride + line : 0);
                    cp_async_16(dst + uint32_t(32 * S::kRowBytes + lane * 16), sc + (ok ? (lane & 3) * 4 : 0), ok);
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < S::kStages - S::kSub; ++i) issue(i);

        if (kFmt == TL_KV_E4M3 && threadIdx.x == 0) *nan_taken = 0.0f;
        // the query rows as A fragments: warp by warp, one row at a time
        for (int r = warp; r < S::kRows; r += S::kWarps) {
            const int row = w.block * S::kRows + r;
            constexpr int kPer = kDim / 32;
            float v[kPer];
            if (r < rows) {
                const int tok = row / p.group, hq = w.head * p.group + row % p.group;
                const __nv_bfloat16* src = p.q + int64_t(w.a.r.first + tok) * p.q_stride + int64_t(hq) * kDim + lane * kPer;
                const uint32_t* s32 = reinterpret_cast<const uint32_t*>(src);
#pragma unroll
                for (int i = 0; i < kPer / 2; ++i) {
                    const uint32_t u = s32[i];
                    v[2 * i] = __uint_as_float(u << 16);
                    v[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[i] = 0.0f;
            }
            float fac = p.scale_log2, mul = 1.0f;
            if (!kBf16) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
                top = __reduce_max_sync(0xffffffffu, top);
                // largest element to [2^14, 2^15); rows of zeros, infinities or NaN stay as they are
                const int e = int(top >> 23);
                const int up = e == 0 || e == 255 ? 0 : min(127 + 14 - e, 100);
                mul = __uint_as_float(uint32_t(127 + up) << 23);
                fac *= __uint_as_float(uint32_t(127 - up) << 23);
            }
            if (lane == 0) row_fac[r] = fac;
            __half* const frag16 = reinterpret_cast<__half*>(q_frag);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int d = lane * kPer + i;
                constexpr int kPiece = kBf16 ? 8 : 16;                 // elements of a 16-byte piece of the cache row
                const int c = d / (4 * kPiece), tt = d / kPiece % 4, ii = d % kPiece;
                const int step = c * (kPiece / 4) + ii / 4, reg = (r % 16 >= 8 ? 1 : 0) + 2 * (ii % 4 / 2);
                const int at = (((r / 16) * S::kSteps + step) * 32 + (r % 8) * 4 + tt) * 8 + reg * 2 + (ii & 1);
                if (kBf16) reinterpret_cast<__nv_bfloat16*>(frag16)[at] = __float2bfloat16_rn(v[i]);
                else frag16[at] = __float2half_rn(v[i] * mul);
            }
        }
        __syncthreads();

        float o[kMT][S::kNTiles][4];
        float m[kMT][2], l[kMT][2], fac[kMT][2];
        int tok_of[kMT][2];
#pragma unroll
        for (int mt = 0; mt < kMT; ++mt) {
#pragma unroll
            for (int j = 0; j < S::kNTiles; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][j][e] = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = mt * 16 + h * 8 + g;
                m[mt][h] = -INFINITY;
                l[mt][h] = 0.0f;
                fac[mt][h] = row_fac[r];
                tok_of[mt][h] = (w.block * S::kRows + min(r, rows - 1)) / p.group;
            }
        }

        for (int i = 0; i < count; i += S::kSub) {
            // stages i .. i + kSub - 1 have landed; the slots of the last turn are free
            cp_async_wait<S::kStages - 2 * S::kSub>();
            __syncwarp();
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) issue(i + S::kStages - S::kSub + u);
            const char* st[S::kSub];
            bool here[S::kSub];                                        // (at an odd end the last turn has one sub-tile less)
            float s[S::kSub][kMT][2][4];
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                here[u] = u == 0 || i + u < count;
                st[u] = ring_gen + ((i + u) % S::kStages) * S::kStageBytes;
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[u][mt][nt][e] = 0.0f;
            }
#pragma unroll
            for (int c = 0; c < S::kKChunks; ++c) {
                constexpr int kStepsPer = kBf16 ? 2 : 4;
                uint32_t a0[S::kSub][4], a1[S::kSub][4];
#pragma unroll
                for (int u = 0; u < S::kSub; ++u) {
                    const uint4 k0 = *reinterpret_cast<const uint4*>(st[u] + c * 512 + lane * 16);
                    const uint4 k1 = *reinterpret_cast<const uint4*>(st[u] + (S::kKChunks + c) * 512 + lane * 16);
                    a0[u][0] = k0.x, a0[u][1] = k0.y, a0[u][2] = k0.z, a0[u][3] = k0.w;
                    a1[u][0] = k1.x, a1[u][1] = k1.y, a1[u][2] = k1.z, a1[u][3] = k1.w;
                }
#pragma unroll
                for (int q = 0; q < kStepsPer; ++q) {
                    uint32_t f4[kMT][4];
#pragma unroll
                    for (int mt = 0; mt < kMT; ++mt) {
                        const uint4 f = q_frag[(mt * S::kSteps + c * kStepsPer + q) * 32 + lane];
                        f4[mt][0] = f.x, f4[mt][1] = f.y, f4[mt][2] = f.z, f4[mt][3] = f.w;
                    }
#pragma unroll
                    for (int u = 0; u < S::kSub; ++u) {
                        uint32_t b00, b01, b10, b11;
                        if (kBf16) {
                            b00 = a0[u][(2 * q) & 3], b01 = a0[u][(2 * q + 1) & 3];
                            b10 = a1[u][(2 * q) & 3], b11 = a1[u][(2 * q + 1) & 3];
                        } else {
                            codes4_to_f16<kFmt>(a0[u][q & 3], b00, b01);
                            codes4_to_f16<kFmt>(a1[u][q & 3], b10, b11);
                        }
#pragma unroll
                        for (int mt = 0; mt < kMT; ++mt) {
                            mma_16816<kBf16>(s[u][mt][0], f4[mt], b00, b01);
                            mma_16816<kBf16>(s[u][mt][1], f4[mt], b10, b11);
                        }
                    }
                }
            }
            // scores in log2 units; the thread's positions: nt * 8 + 2t + {0, 1} of each sub-tile
            float rvs[S::kSub][2][2];
            uint32_t seen[S::kSub];                                    // bit ((mt * 2 + h) * 4 + nt * 2 + e)
            bool edge[S::kSub];
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                if (!kBf16) {
                    const float* sc = reinterpret_cast<const float*>(st[u] + 32 * S::kRowBytes);
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        const float2 ks = *reinterpret_cast<const float2*>(sc + nt * 8 + 2 * t);
                        const float2 vs = *reinterpret_cast<const float2*>(sc + 16 + nt * 8 + 2 * t);
                        // A row of zero values has scale 0: the floor in its place gives it its share of the sum.  A NaN
                        // scale reaches the score alone (the product with 0), which a mask can still replace.
                        const float v0 = vs.x >= kScaleFloor ? vs.x : kScaleFloor, v1 = vs.y >= kScaleFloor ? vs.y : kScaleFloor;
                        const float lv0 = fmaf(vs.x, 0.0f, lg2(v0)), lv1 = fmaf(vs.y, 0.0f, lg2(v1));
                        rvs[u][nt][0] = __fdividef(1.0f, v0);
                        rvs[u][nt][1] = __fdividef(1.0f, v1);
#pragma unroll
                        for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                s[u][mt][nt][2 * h] = fmaf(s[u][mt][nt][2 * h], fac[mt][h] * ks.x, lv0);
                                s[u][mt][nt][2 * h + 1] = fmaf(s[u][mt][nt][2 * h + 1], fac[mt][h] * ks.y, lv1);
                            }
                    }
                } else {
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                s[u][mt][nt][2 * h] *= fac[mt][h];
                                s[u][mt][nt][2 * h + 1] *= fac[mt][h];
                            }
                }
                const int pos0 = pos_first + (i + u) * S::kTile;
                edge[u] = pos0 + 16 > start;                           // the step's own tokens, or past the end
                seen[u] = 0xffffffffu;
                if (edge[u] || bad_any || !here[u]) {
                    seen[u] = 0;
                    bool ok = here[u];
                    if (ok) {
                        const int page = table[pos0 >> p.cache.page_shift];
                        ok = page >= 0 && page < p.cache.pages;
                    }
#pragma unroll
                    for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int pos = pos0 + (e >> 1) * 8 + 2 * t + (e & 1);
                                const bool vis = ok && pos < len && attend_sees(p, w.a.r.first + tok_of[mt][h], tok_of[mt][h], pos - start);
                                if (vis) seen[u] |= 1u << ((mt * 2 + h) * 4 + e);
                                else s[u][mt][e >> 1][2 * h + (e & 1)] = -INFINITY;
                            }
                    if (!kBf16 && !here[u]) rvs[u][0][0] = rvs[u][0][1] = rvs[u][1][0] = rvs[u][1][1] = 0.0f;   // (never loaded)
                }
            }
            // The reference may lag by up to 2^8, which f16 and the sums have room for: the rescaling of O, half of all turns with an
            // exact maximum, becomes rare.
            float top[kMT][2];
            bool grew = false;
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = -INFINITY;
#pragma unroll
                    for (int u = 0; u < S::kSub; ++u)
                        x = fmaxf(x, fmaxf(fmaxf(s[u][mt][0][2 * h], s[u][mt][0][2 * h + 1]), fmaxf(s[u][mt][1][2 * h], s[u][mt][1][2 * h + 1])));
                    top[mt][h] = x;
                    grew |= x > m[mt][h] + (kLag + S::kHead);
                }
            if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x = fmaxf(top[mt][h], __shfl_xor_sync(0xffffffffu, top[mt][h], 1));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                        // (by the row's own scores: what other rows see leaves its bits alone)
                        const bool up = x > m[mt][h] + (kLag + S::kHead);
                        const float to = x - S::kHead, f = up ? ex2(m[mt][h] - to) : 1.0f;
                        m[mt][h] = up ? to : m[mt][h];
                        l[mt][h] *= f;
#pragma unroll
                        for (int j = 0; j < S::kNTiles; ++j) {
                            o[mt][j][2 * h] *= f;
                            o[mt][j][2 * h + 1] *= f;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                if (u > 0 && !here[u]) break;
                uint32_t a[kMT][4], a_low[kMT][4];
                float pf[kMT][2][4];
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // (a row that has seen nothing yet has maximum -inf: any finite number serves in its place)
                        const float m_use = m[mt][h] == -INFINITY ? 0.0f : m[mt][h];
                        float sum = 0.0f;
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float e2 = ex2(s[u][mt][nt][2 * h + e] - m_use);
                                pf[mt][nt][2 * h + e] = e2;
                                sum = kBf16 ? sum + e2 : fmaf(e2, rvs[u][nt][e], sum);
                            }
                        l[mt][h] += sum;
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const float lo = pf[mt][nt][2 * h], hi = pf[mt][nt][2 * h + 1];
                            a[mt][nt * 2 + h] = kBf16 ? pack_bf16(lo, hi) : pack_f16(lo, hi);
                            // what the rounding to bf16 left over
                            if (kBf16) a_low[mt][nt * 2 + h] = pack_bf16(lo - __uint_as_float(a[mt][nt * 2 + h] << 16), hi - __uint_as_float(a[mt][nt * 2 + h] & 0xffff0000u));
                        }
                    }
                const char* const vst = st[u] + 16 * S::kRowBytes;
                if (kBf16 && edge[u]) {
                    // A value may be infinite or NaN for a token that other rows see: its product with a masked weight of 0
                    // must not reach this row.  (Positions past the end were filled with 0; INT8 codes are always finite.)
                    bool odd = false;
#pragma unroll
                    for (int k = 0; k < 4 * S::kVChunks; ++k) {
                        const uint4 v = *reinterpret_cast<const uint4*>(vst + k * 512 + lane * 16);
                        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) odd |= (x[q] & 0x7f80u) == 0x7f80u || (x[q] & 0x7f800000u) == 0x7f800000u;
                    }
                    if (__any_sync(0xffffffffu, odd)) {
                        for (int tok = 0; tok < 16; ++tok) {
                            const int from = g * 4 + (tok % 8) / 2, k = (tok >> 3) * 2 + (tok & 1);
#pragma unroll
                            for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const float own0 = tok & 1 ? pf[mt][0][2 * h + 1] : pf[mt][0][2 * h];
                                    const float own1 = tok & 1 ? pf[mt][1][2 * h + 1] : pf[mt][1][2 * h];
                                    const float pw = __shfl_sync(0xffffffffu, tok >> 3 ? own1 : own0, from);
                                    const uint32_t vis = __shfl_sync(0xffffffffu, seen[u], from) >> ((mt * 2 + h) * 4 + (tok >> 3) * 2 + (tok & 1)) & 1u;
                                    if (!vis) continue;
#pragma unroll
                                    for (int j = 0; j < S::kNTiles; ++j)
#pragma unroll
                                        for (int e = 0; e < 2; ++e) {
                                            const char* v = vst + (k * S::kVChunks + j / 8) * 512 + ((2 * t + e) * 4 + (tok % 8) / 2) * 16 + (j % 8) * 2;
                                            o[mt][j][2 * h + e] += pw * __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(v));
                                        }
                                }
                        }
                        continue;
                    }
                }
#pragma unroll
                for (int c = 0; c < S::kVChunks; ++c) {
                    constexpr int kWords = S::kVBytes / 4;
                    uint32_t v[4][kWords];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const char* src = vst + (k * S::kVChunks + c) * 32 * S::kVBytes + lane * S::kVBytes;
                        if (S::kVBytes == 16) {
                            const uint4 x = *reinterpret_cast<const uint4*>(src);
                            v[k][0] = x.x, v[k][1 % kWords] = x.y, v[k][2 % kWords] = x.z, v[k][3 % kWords] = x.w;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2*>(src);
                            v[k][0] = x.x, v[k][1 % kWords] = x.y;
                        }
                    }
                    if (kFmt == TL_KV_E4M3 && edge[u]) {
                        // Among the step's own tokens, of which rows see different ones: a NaN code stays out of the product (a weight
                        // of 0 would not keep it out), and the rows that see it get theirs when the warps are joined.
                        uint32_t any = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int q = 0; q < kWords; ++q) any |= e4m3_nan_bits(v[k][q]);
                        if (__builtin_expect(any != 0, 0)) {
                            *nan_taken = 1.0f;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
#pragma unroll
                                for (int q = 0; q < kWords; ++q) v[k][q] &= ~e4m3_nan_bytes(v[k][q]);
                        }
                    }
#pragma unroll
                    for (int q = 0; q < kWords; ++q) {
                        if (kBf16) {
                            const uint32_t b[4] = {__byte_perm(v[0][q], v[1][q], 0x5410), __byte_perm(v[2][q], v[3][q], 0x5410),
                                                   __byte_perm(v[0][q], v[1][q], 0x7632), __byte_perm(v[2][q], v[3][q], 0x7632)};
#pragma unroll
                            for (int mt = 0; mt < kMT; ++mt) {
                                mma_16816<true>(o[mt][(c * kWords + q) * 2], a[mt], b[0], b[1]);
                                mma_16816<true>(o[mt][(c * kWords + q) * 2 + 1], a[mt], b[2], b[3]);
                                mma_16816<true>(o[mt][(c * kWords + q) * 2], a_low[mt], b[0], b[1]);
                                mma_16816<true>(o[mt][(c * kWords + q) * 2 + 1], a_low[mt], b[2], b[3]);
                            }
                        } else {
                            uint32_t lo[4], hi[4];
                            codes4_to_f16<kFmt>(__byte_perm(v[0][q], v[1][q], 0x5140), lo[0], lo[1]);
                            codes4_to_f16<kFmt>(__byte_perm(v[0][q], v[1][q], 0x7362), lo[2], lo[3]);
                            codes4_to_f16<kFmt>(__byte_perm(v[2][q], v[3][q], 0x5140), hi[0], hi[1]);
                            codes4_to_f16<kFmt>(__byte_perm(v[2][q], v[3][q], 0x7362), hi[2], hi[3]);
#pragma unroll
                            for (int z = 0; z < 4; ++z)
#pragma unroll
                                for (int mt = 0; mt < kMT; ++mt)
                                    mma_16816<false>(o[mt][(c * kWords + q) * 4 + z], a[mt], lo[z], hi[z]);
                        }
                    }
                }
            }
        }
        cp_async_wait<0>();
        if (bad_any && lane == 0) atomicCAS(p.status, 0u, kBadPage);
        if (w.a.r.n > len - start && threadIdx.x == 0) atomicCAS(p.status, 0u, kBadPage);

        // join the warps: a common maximum per row, then the sums
#pragma unroll
        for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float sum = l[mt][h];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if (t == 0) {
                    stat_m[warp * S::kRows + mt * 16 + h * 8 + g] = m[mt][h];
                    stat_l[warp * S::kRows + mt * 16 + h * 8 + g] = sum;
                }
            }
        __syncthreads();                                               // (also: every warp is done with the ring)
        if (int(threadIdx.x) < S::kRows) {
            float top = -INFINITY, sum = 0.0f;
            for (int k = 0; k < S::kWarps; ++k) top = fmaxf(top, stat_m[k * S::kRows + threadIdx.x]);
            const float use = top == -INFINITY ? 0.0f : top;
            for (int k = 0; k < S::kWarps; ++k) sum += stat_l[k * S::kRows + threadIdx.x] * ex2(stat_m[k * S::kRows + threadIdx.x] - use);
            row_m[threadIdx.x] = top;
            row_l[threadIdx.x] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = mt * 16 + h * 8 + g;
                if (r >= rows) continue;
                const float top = row_m[r];
                const float f = ex2(m[mt][h] - (top == -INFINITY ? 0.0f : top));
                float* const dst = join + (warp * S::kRows + r) * kDim;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < S::kNTiles; j += 4) {
                        // columns of tile j .. j + 3 are consecutive dimensions within this thread's piece
                        constexpr int kPiece = kBf16 ? 8 : S::kVBytes;
                        const int d = (j / kPiece) * 8 * kPiece + (2 * t + e) * kPiece + j % kPiece;
                        *reinterpret_cast<float4*>(dst + d) = make_float4(o[mt][j][2 * h + e] * f, o[mt][j + 1][2 * h + e] * f,
                                                                          o[mt][j + 2][2 * h + e] * f, o[mt][j + 3][2 * h + e] * f);
                    }
            }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == w.a.tiles;
        const int slot = int(blockIdx.x) * 2 + (t0 > 0 ? 0 : 1);
        for (int e = threadIdx.x; e < rows * (kDim / 4); e += S::kThreads) {
            const int r = e / (kDim / 4), d = e % (kDim / 4) * 4;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < S::kWarps; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(join + (k * S::kRows + r) * kDim + d);
                sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
            }
            if (whole) {
                const int row = w.block * S::kRows + r, tok = row / p.group, hq = w.head * p.group + row % p.group;
                const float ll = row_l[r], inv = ll == 0.0f ? 0.0f : 1.0f / ll;
                *reinterpret_cast<uint2*>(p.out + int64_t(w.a.r.first + tok) * p.out_stride + int64_t(hq) * kDim + d) =
                    make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
                if (p.lse && d == 0) p.lse[int64_t(w.a.r.first + tok) * p.q_heads + hq] = ll == 0.0f ? -INFINITY : (row_m[r] + log2f(ll)) * 0.69314718055994531f;
            } else {
                *reinterpret_cast<float4*>(p.part + (int64_t(slot) * S::kRows + r) * kDim + d) = sum;
                if (d == 0) p.part_ml[int64_t(slot) * S::kRows + r] = make_float2(row_m[r], row_l[r]);
            }
        }
        if (kFmt == TL_KV_E4M3 && *nan_taken != 0.0f) {
            // what the rows see of the NaN codes that were taken out, over what this thread has just written
            for (int e = threadIdx.x; e < rows * (kDim / 4); e += S::kThreads) {
                const int r = e / (kDim / 4), d = e % (kDim / 4) * 4, row = w.block * S::kRows + r, tok = row / p.group;
                uint32_t bad = 0;
                for (int pos = max(start & ~15, t0 * S::kTile); pos < min(len, t1 * S::kTile); ++pos) {   // (whole groups of 16)
                    const int page = table[pos >> p.cache.page_shift];
                    if (page < 0 || page >= p.cache.pages || !attend_sees(p, w.a.r.first + tok, tok, pos - start)) continue;
                    bad |= e4m3_nan_bits(*reinterpret_cast<const uint32_t*>(v_head + int64_t(page) * p.cache.page_stride +
                                                                            int64_t(pos & pos_mask) * p.cache.token_stride + d));
                }
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    if (!(bad >> (8 * i) & 0x80u)) continue;
                    if (whole) p.out[int64_t(w.a.r.first + tok) * p.out_stride + int64_t(w.head * p.group + row % p.group) * kDim + d + i] = __ushort_as_bfloat16(0x7fff);
                    else p.part[(int64_t(slot) * S::kRows + r) * kDim + d + i] = __uint_as_float(0x7fc00000u);
                }
            }
        }
        x += t1 - t0;
        if (x >= x_end) break;
        attend_next_unit(p, w);
        __syncthreads();                                               // the join's memory becomes the ring again
    }
}

template <int kDim, int kFmt, int kMT>
int launch_attend_small(const AttendParams& p, int ctas, cudaStream_t stream) {
    using S = SmallShape<kDim, kFmt, kMT>;
    const void* kernel = reinterpret_cast<const void*>(attend_kernel<kDim, kFmt, kMT>);
    if (int rc = ensure_smem_attr(kernel, S::kSmem)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas));
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = opt(TL_OPT_PDL) != 0 ? 1 : 0;
    return check_cuda(cudaLaunchKernelEx(&cfg, attend_kernel<kDim, kFmt, kMT>, p));
}

}  // namespace tl
