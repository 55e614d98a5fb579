// Attention for few query rows per key/value head over a 4-bit cache (decoding, short chains, small trees).
//
// One pass over the cache with a running maximum and sum, as in the kernel for the wider formats: every warp owns 16 positions of a
// tile and all rows of the unit, each cache element is fetched and converted by exactly one thread of the machine, no barrier stands
// inside the loop, and the warps' sums are joined once per unit.  With 4 bits a byte of the cache costs twice the instructions, and
// instructions are what bounds it, so the products are turned round: the cache is the operand with 16 rows of the instruction and the
// queries the one with 8 columns,
//     S^T (16 tokens x 8 rows) = K q^T,     O^T (16 dimensions x 8 rows) += V^T P^T.
// Decoding with up to 8 query heads per key/value head then leaves no half of an instruction, of the scores or of the accumulators
// unused (a 16-row query operand leaves half): 16 products, 4 scores per thread and 32 accumulators for 16 tokens of 128 dimensions.
// Thread (g = lane / 4, t = lane % 4) holds
//   K      tokens g, g + 8; the contraction index may be permuted as long as q is, so its share is a contiguous piece of the row;
//   q^T    row g, the same piece, in shared memory for the whole unit;
//   S^T    tokens g, g + 8 of rows 2t, 2t + 1.  P^T as the second product wants it (row g, tokens 2t, 2t + 1) is that transposed
//          8 x 8 by 8 x 8, one movmatrix each;
//   V^T    tokens 2t, 2t + 1, 2t + 8, 2t + 9 of a contiguous piece of dimensions; the codes of two tokens at one dimension are put
//          side by side by half bytes and converted together.
// Codes become f16 by one conversion per pair, times their group scales (kGroupUnit): exact.  Scales, weights, references and what
// masked positions may hold: as over an 8-bit cache; no code or group scale reads as infinite or NaN, so positions past the end need
// no zeros in their place.
//
// Measured choices.  Queries in registers took as long with one block of 8 rows and 2 to 12 % longer with two and four.  CTAs per SM and
// sub-tiles a turn with the queries where they are (64 query and 8 key/value heads of 128, contexts of half the length to all of it, us as
// it is / one sub-tile a turn / three CTAs / five CTAs): 1 request of one token over 4100 14.9 / 14.4 / 14.4 / 16.7, 4 over 4100 17.0 / 16.2 /
// 17.5 / 20.5, 32 over 4100 40.8 / 40.4 / 40.1 / 49.5, 64 over 2000 43.2 / 41.6 / 44.6 / 49.3; 1 over 407 (32 / 4 heads) 9.8 / 9.3 / 9.8 / 10.2.
// (While queries lay in registers two sub-tiles took 48 us for 32 over 4100 where one took 54; now they make no odds, or 1 to 5 % the wrong
// way.)  With 64 accumulators two CTAs / three: 32 requests of one token over 4100, heads of 256, 65.3 / 60.7; two tokens each, 64 over 2000
// 57.6 / 54.8, 16 over 4100 32.9 / 33.2; heads of 64, four tokens each, 4 over 4100 20.8 / 21.7, 16 32.8 / 34.7, 64 over 2000 57.5 / 56.9.
//
// What bounds it: 32 requests of one token over 4100 (64 query and 8 key/value heads of 128, 122 MB): 41 us, floor 18.6.  8.6 us pass
// outside of the loop (launch, ranges, queries, joins; as 29 below from copies of an earlier form); 20 million warp instructions keep the ALUs, which run unpacking and softmax at half
// rate, busy for 48 % and the issue slots for 58 % of the time with four warps per scheduler; the copies alone (no arithmetic)
// take 29.  Bulk copies in place of cp.async: as fast issued by each warp, 62 us by a warp of their own.
#pragma once

#include "tl_attend.cuh"

namespace tl {

template <int kDim, int kNT>
struct FourShape {
    static constexpr int kRowBytes = kDim / 2, kGroups = kDim / 16, kRows = kNT * 8;
    static constexpr int kWarps = 4, kThreads = kWarps * 32, kTile = kWarps * 16;
    static constexpr int kAcc = kDim / 4 * kNT;                    // accumulators of a thread
    static constexpr int kCtasPerSm = kAcc <= 32 ? 4 : 2;
    static constexpr int kSub = kAcc <= 32 && kDim <= 128 ? 2 : 1;                // sub-tiles of 16 tokens a warp takes at a time
    static constexpr int kKBytes = kRowBytes / 4 < 16 ? kRowBytes / 4 : 16, kKChunks = kRowBytes / 4 / kKBytes, kKPiece = 2 * kKBytes;
    static constexpr int kVBytes = kRowBytes / 8, kVPiece = 2 * kVBytes;
    static constexpr int kSteps = kDim / 16, kTiles = kDim / 16;   // 16-deep steps of K q^T, 16-row tiles of V^T P^T
    static constexpr int kValueAt = 16 * kRowBytes, kScaleAt = 32 * kRowBytes, kGroupAt = kScaleAt + 128;
    static constexpr int kStageBytes = kGroupAt + 32 * kGroups;
    static constexpr int kQBytes = kNT * kSteps * 256;
    static constexpr int kStatBytes = (kWarps * kRows * 2 + kRows * 3) * 4;
    static constexpr int kBudget = 225 * 1024 / kCtasPerSm - 1024 - kQBytes - kStatBytes;
    static constexpr int kStagesFit = kBudget / (kWarps * kStageBytes);
    static constexpr int kStages = kStagesFit > 6 ? 6 : kStagesFit;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kJoinRow = kDim + 4;                      // floats: rows of a join on different banks
    static constexpr int kJoin = kWarps * kRows * kJoinRow * 4;
    static constexpr int kUnion = kRing > kJoin ? kRing : kJoin;   // the ring's memory also serves the join
    static constexpr int kSmem = kUnion + kQBytes + kStatBytes;
    static_assert(kStages >= 2 * kSub, "no room for the stages ahead");
    static_assert(kSmem <= 225 * 1024 / kCtasPerSm, "shared memory");
};

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Where a token's values lie in a stage: rows 2t and 2t + 1, which four threads read together, on different banks.
template <int kDim>
__device__ __forceinline__ int four_value_row(int token) { return (token >> 1 & 3) | (token & 1) << 2 | (token & 8); }
template <int kDim>
__device__ __forceinline__ int four_value_swap(int row) { return kDim == 256 ? (row & 3) * 2 : kDim == 128 ? (row >> 1 & 1) * 2 : 0; }
template <int kDim>
__device__ __forceinline__ int four_key_swap(int token) { return kDim == 256 ? (token & 1) * 4 : 0; }

constexpr float kFourNoMax = -3.0e38f;   // in place of a maximum while a row has seen nothing

template <int kDim, int kNT>
__global__ void __launch_bounds__(FourShape<kDim, kNT>::kThreads, FourShape<kDim, kNT>::kCtasPerSm)
attend_four_kernel(const AttendParams p) {
    using S = FourShape<kDim, kNT>;
    constexpr float kHead = attend_head(TL_KV_E2M1);
    extern __shared__ __align__(128) char smem[];
    float* const join = reinterpret_cast<float*>(smem);
    uint2* const q_frag = reinterpret_cast<uint2*>(smem + S::kUnion);                 // [nt][step][lane]
    float* const stat_m = reinterpret_cast<float*>(smem + S::kUnion + S::kQBytes);    // [warp][row]
    float* const stat_l = stat_m + S::kWarps * S::kRows;
    float* const row_fac = stat_l + S::kWarps * S::kRows;                             // [row]
    float* const row_m = row_fac + S::kRows;                                          // [row] joined maximum and sum
    float* const row_l = row_m + S::kRows;
    const int lane = int(lane_id()), warp = int(threadIdx.x) / 32, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + uint32_t(warp * S::kStages * S::kStageBytes);
    const char* const ring_gen = smem + warp * S::kStages * S::kStageBytes;

    pdl_wait();
    pdl_launch_dependents();
    int per, x = 0, x_end = 0;
    AttendPlace w;
    const bool work = attend_range(p, int(blockIdx.x), &per, &x, &x_end, &w);
    if (!work) return;

    // the 16-byte pieces of 16 rows that this lane copies: token lane / kChunks and every kPerCopy-th after it, piece lane % kChunks
    constexpr int kChunks = S::kRowBytes / 16, kPerCopy = 32 / kChunks, kCopies = 16 / kPerCopy;
    const uint32_t ts = uint32_t(p.cache.token_stride);
    const uint32_t lane_off = uint32_t(lane / kChunks) * ts + uint32_t(lane % kChunks) * 16u;

    while (true) {
        const int t0 = w.tile, t1 = min(w.a.tiles, t0 + (x_end - x));
        const int rows = min(S::kRows, w.a.r.n * p.group - w.block * S::kRows);
        const int32_t* const table = p.batch.page_table + int64_t(w.b) * p.batch.table_stride;
        const char* const k_lane = p.cache.base[0] + int64_t(w.head) * p.cache.head_stride + lane_off;
        const char* const v_lane = p.cache.base[1] + int64_t(w.head) * p.cache.head_stride + lane_off;
        const int len = w.a.r.len, start = w.a.r.start;
        const int pos_mask = (1 << p.cache.page_shift) - 1;
        // scales (8 pieces) and group scales, a run each: what this lane copies of them
        constexpr int kExtra = 8 + 2 * S::kGroups, kExtraCopies = (kExtra + 31) / 32;
        const char* extra[kExtraCopies];
        int64_t extra_page[kExtraCopies];
#pragma unroll
        for (int r = 0; r < kExtraCopies; ++r) {
            const int id = lane + 32 * r, gid = id - 8;
            if (id < 8) {
                extra[r] = reinterpret_cast<const char*>(p.cache.scale[id >> 2] + int64_t(w.head) * p.cache.scale_head_stride + (id & 3) * 4);
                extra_page[r] = p.cache.scale_page_stride * 4;
            } else {
                extra[r] = p.cache.group[gid / S::kGroups & 1] + int64_t(w.head) * p.cache.group_head_stride + gid % S::kGroups * 16;
                extra_page[r] = p.cache.group_page_stride;
            }
        }

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
        uint32_t fill_at = 0, use_at = 0;                                // offsets of the next stage to fill and to use
        auto issue = [&](int i) {                                        // starts the copies of sub-tile i (whole warp, i upwards)
            if (i < count) {
                if (i > 0 && (i & 31) == 0) {
                    pages = checked(pages_next, i + lane);
                    pages_next = load_page(i + 32 + lane);
                }
                const int found = __shfl_sync(0xffffffffu, pages, i & 31);
                const bool ok = found >= 0;
                const int page = ok ? found : 0;
                bad_any |= ok ? 0u : 1u;
                const int line = (pos_first + i * S::kTile) & pos_mask;
                const int64_t at = int64_t(page) * p.cache.page_stride + int64_t(uint32_t(line)) * ts;
                const uint32_t dst = ring + fill_at;
                fill_at = fill_at == (S::kStages - 1) * S::kStageBytes ? 0 : fill_at + S::kStageBytes;
#pragma unroll
                for (int r = 0; r < kCopies; ++r) {
                    const int tok = lane / kChunks + r * kPerCopy, c = lane % kChunks, row = four_value_row<kDim>(tok);
                    cp_async_16(dst + uint32_t(tok * S::kRowBytes + (c ^ four_key_swap<kDim>(tok)) * 16), k_lane + at + uint32_t(r * kPerCopy) * ts, ok);
                    cp_async_16(dst + uint32_t(S::kValueAt + row * S::kRowBytes + (c ^ four_value_swap<kDim>(row)) * 16), v_lane + at + uint32_t(r * kPerCopy) * ts, ok);
                }
#pragma unroll
                for (int r = 0; r < kExtraCopies; ++r) {
                    const int id = lane + 32 * r;
                    if (id < kExtra)
                        cp_async_16(dst + uint32_t(S::kScaleAt + id * 16), extra[r] + int64_t(page) * extra_page[r] + uint32_t(line) * uint32_t(id < 8 ? 4 : S::kGroups), ok);
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < S::kStages - S::kSub; ++i) issue(i);

        // The queries, a block of 8 rows per warp: thread (g, t) takes its piece of row nt * 8 + g, scaled to f16 by a power of two of the row's own.
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            if (nt % S::kWarps != warp) continue;
            const int r = nt * 8 + g, row = w.block * S::kRows + r;
            uint32_t u[S::kSteps][2];
            if (r < rows) {
                const int tok = row / p.group, hq = w.head * p.group + row % p.group;
                const __nv_bfloat16* src = p.q + int64_t(w.a.r.first + tok) * p.q_stride + int64_t(hq) * kDim + t * S::kKPiece;
#pragma unroll
                for (int i = 0; i < S::kSteps / 2; ++i) {                // 8 elements: two steps' shares
                    constexpr int kPer = S::kKPiece / 8;
                    const uint4 v = *reinterpret_cast<const uint4*>(src + i / kPer * 4 * S::kKPiece + i % kPer * 8);
                    u[2 * i][0] = v.x, u[2 * i][1] = v.y, u[2 * i + 1][0] = v.z, u[2 * i + 1][1] = v.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < S::kSteps; ++i) u[i][0] = u[i][1] = 0;
            }
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i) top = __vmaxu2(top, __vmaxu2(u[i][0] & 0x7fff7fffu, u[i][1] & 0x7fff7fffu));
            top = max(top & 0xffffu, top >> 16);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // largest element to [2^14, 2^15); rows of zeros, infinities or NaN stay as they are
            const int e = int(top >> 7);
            const int up = e == 0 || e == 255 ? 0 : min(127 + 14 - e, 100);
            const float mul = __uint_as_float(uint32_t(127 + up) << 23);
            const float f = p.scale_log2 * __uint_as_float(uint32_t(127 - up) << 23) * kGroupUnit;
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) u[i][k] = pack_f16(__uint_as_float(u[i][k] << 16) * mul, __uint_as_float(u[i][k] & 0xffff0000u) * mul);
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i) q_frag[(nt * S::kSteps + i) * 32 + lane] = make_uint2(u[i][0], u[i][1]);
            if (t == 0) row_fac[r] = f;
        }
        __syncthreads();
        float fac[kNT][2];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) fac[nt][0] = row_fac[nt * 8 + 2 * t], fac[nt][1] = row_fac[nt * 8 + 2 * t + 1];

        // o[nt][j]: dimensions 2j, 2j + 1 of the thread's piece ([0], [2]) of row nt * 8 + 2t, and ([1], [3]) of row + 1
        float o[kNT][S::kTiles][4];
        float m[kNT][2], l[kNT][2];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
#pragma unroll
            for (int j = 0; j < S::kTiles; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][j][e] = 0.0f;
            m[nt][0] = m[nt][1] = kFourNoMax;
            l[nt][0] = l[nt][1] = 0.0f;
        }
        const int tiles_n = (rows + 7) / 8;                              // of 8 rows

        for (int i = 0; i < count; i += S::kSub) {
            // stages i .. i + kSub - 1 have landed; the slots of the last turn are free
            cp_async_wait<S::kStages - 2 * S::kSub>();
            __syncwarp();
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) issue(i + S::kStages - S::kSub + u);
            const char* st[S::kSub];
            bool here[S::kSub];                                        // (at an odd end the last turn has one sub-tile less)
            float s[S::kSub][kNT][4];                                  // tokens g, g, g + 8, g + 8 of rows 2t, 2t + 1 in turn
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                here[u] = u == 0 || i + u < count;
                st[u] = ring_gen + use_at;
                use_at = use_at == (S::kStages - 1) * S::kStageBytes ? 0 : use_at + S::kStageBytes;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][nt][e] = 0.0f;
            }
#pragma unroll
            for (int c = 0; c < S::kKChunks; ++c) {
#pragma unroll
                for (int u = 0; u < S::kSub; ++u) {
                    uint32_t w0[4], w1[4], g0[2], g1[2];
                    const int at = kDim == 64 ? t * 8 : ((c * 4 + t) ^ four_key_swap<kDim>(g)) * 16;
                    load_words<S::kKBytes>(st[u] + g * S::kRowBytes + at, w0);
                    load_words<S::kKBytes>(st[u] + (g + 8) * S::kRowBytes + at, w1);
                    const char* const gr = st[u] + S::kGroupAt + g * S::kGroups + (c * 4 + t) * (S::kKPiece / 16);
                    const uint32_t x0 = S::kKPiece == 32 ? *reinterpret_cast<const uint16_t*>(gr) : uint8_t(*gr);
                    const uint32_t x1 = S::kKPiece == 32 ? *reinterpret_cast<const uint16_t*>(gr + 8 * S::kGroups) : uint8_t(gr[8 * S::kGroups]);
                    g0[0] = group_f16x2(x0, 0, 0, 0), g0[1] = group_f16x2(x0, 0, 1, 1);
                    g1[0] = group_f16x2(x1, 0, 0, 0), g1[1] = group_f16x2(x1, 0, 1, 1);
#pragma unroll
                    for (int k = 0; k < S::kKBytes / 4; ++k) {         // a word: eight codes, two steps
                        uint32_t h0[4], h1[4];
                        e2m1x8_to_f16(w0[k], g0[k / 2], h0);
                        e2m1x8_to_f16(w1[k], g1[k / 2], h1);
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int step = c * (S::kKPiece / 4) + 2 * k + z;
                            const uint32_t a[4] = {h0[2 * z], h1[2 * z], h0[2 * z + 1], h1[2 * z + 1]};
#pragma unroll
                            for (int nt = 0; nt < kNT; ++nt) {
                                if (kNT > 2 && nt >= tiles_n) continue;
                                const uint2 b = q_frag[(nt * S::kSteps + step) * 32 + lane];
                                mma_16816<false>(s[u][nt], a, b.x, b.y);
                            }
                        }
                    }
                }
            }
            // scores in log2 units
            float rvs[S::kSub][2];
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                const float* const sc = reinterpret_cast<const float*>(st[u] + S::kScaleAt);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float ks = sc[g + 8 * h], vs = sc[16 + g + 8 * h] * kGroupUnit;
                    // A row of zero values has scale 0: the floor in its place (and in a NaN's) gives it its share of the sum.  A NaN
                    // scale reaches the score alone (the product with 0), which a mask can still replace.
                    const float v = fmaxf(vs, kScaleFloor);
                    const float lv = fmaf(vs, 0.0f, lg2(v));
                    rvs[u][h] = __fdividef(1.0f, v);
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) s[u][nt][2 * h + e] = fmaf(s[u][nt][2 * h + e], fac[nt][e] * ks, lv);
                }
                const int pos0 = pos_first + (i + u) * S::kTile;
                if (pos0 + 16 > start || bad_any || !here[u]) {        // the step's own tokens, or past the end
                    bool ok = here[u];
                    if (ok) {
                        const int page = table[pos0 >> p.cache.page_shift];
                        ok = page >= 0 && page < p.cache.pages;
                    }
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int tok = (w.block * S::kRows + min(nt * 8 + 2 * t + e, rows - 1)) / p.group;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int pos = pos0 + g + 8 * h;
                                if (!(ok && pos < len && attend_sees(p, w.a.r.first + tok, tok, pos - start))) s[u][nt][2 * h + e] = -INFINITY;
                            }
                        }
                    if (!here[u]) rvs[u][0] = rvs[u][1] = 0.0f;        // (never loaded)
                }
            }
            // The reference may lag by up to 2^8, which f16 and the sums have room for: the rescaling of O becomes rare.
            float top[kNT][2];
            bool grew = false;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float y = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
                    for (int u = 1; u < S::kSub; ++u) y = fmaxf(y, fmaxf(s[u][nt][e], s[u][nt][2 + e]));
                    top[nt][e] = y;
                    grew |= y > m[nt][e] + (kLag + kHead);
                }
            if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float y = top[nt][e];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, d));
                        // (by the row's own scores: what other rows see leaves its bits alone)
                        const bool up = y > m[nt][e] + (kLag + kHead);
                        const float to = y - kHead, f = up ? ex2(m[nt][e] - to) : 1.0f;
                        m[nt][e] = up ? to : m[nt][e];
                        l[nt][e] *= f;
#pragma unroll
                        for (int j = 0; j < S::kTiles; ++j) {
                            o[nt][j][e] *= f;
                            o[nt][j][2 + e] *= f;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                if (u > 0 && !here[u]) break;
                uint32_t b[kNT][2];
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float e0 = ex2(s[u][nt][2 * h] - m[nt][0]), e1 = ex2(s[u][nt][2 * h + 1] - m[nt][1]);
                        l[nt][0] = fmaf(e0, rvs[u][h], l[nt][0]);
                        l[nt][1] = fmaf(e1, rvs[u][h], l[nt][1]);
                        b[nt][h] = transpose_8x8(pack_f16(e0, e1));
                    }
                }
                // values of the thread's piece: tokens 2t, 2t + 1 (k = 0, 1), 2t + 8, 2t + 9 (2, 3)
                uint32_t v[4][4], x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = t + (k & 1) * 4 + (k >> 1) * 8, byte = g * S::kVBytes;
                    load_words<S::kVBytes>(st[u] + S::kValueAt + row * S::kRowBytes + (((byte >> 4) ^ four_value_swap<kDim>(row)) << 4) + (byte & 15), v[k]);
                    const char* const at = st[u] + S::kGroupAt + (16 + 2 * t + (k & 1) + 8 * (k >> 1)) * S::kGroups + g * S::kVPiece / 16;
                    x[k] = S::kVPiece == 32 ? *reinterpret_cast<const uint16_t*>(at) : uint8_t(*at);
                }
#pragma unroll
                for (int k = 0; k < S::kVBytes / 4; ++k) {             // eight dimensions
                    constexpr uint32_t kLow = 0x0f0f0f0fu;
                    const uint32_t g01 = group_f16x2(x[0], x[1], k / 2, 4 + k / 2), g89 = group_f16x2(x[2], x[3], k / 2, 4 + k / 2);
                    uint32_t a0[4], a1[4], a2[4], a3[4];
                    e2m1x8_to_f16((v[0][k] & kLow) | (v[1][k] << 4 & ~kLow), g01, a0);
                    e2m1x8_to_f16((v[0][k] >> 4 & kLow) | (v[1][k] & ~kLow), g01, a1);
                    e2m1x8_to_f16((v[2][k] & kLow) | (v[3][k] << 4 & ~kLow), g89, a2);
                    e2m1x8_to_f16((v[2][k] >> 4 & kLow) | (v[3][k] & ~kLow), g89, a3);
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const uint32_t a[4] = {a0[z], a1[z], a2[z], a3[z]};
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            if (kNT > 2 && nt >= tiles_n) continue;
                            mma_16816<false>(o[nt][k * 4 + z], a, b[nt][0], b[nt][1]);
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
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (g == 0) {
                    stat_m[warp * S::kRows + nt * 8 + 2 * t + e] = m[nt][e];
                    stat_l[warp * S::kRows + nt * 8 + 2 * t + e] = sum;
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
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nt * 8 + 2 * t + e;
                if (r >= rows) continue;
                const float top = row_m[r];
                const float f = ex2(m[nt][e] - (top == -INFINITY ? 0.0f : top));
                float* const dst = join + (warp * S::kRows + r) * S::kJoinRow + g * S::kVPiece;
#pragma unroll
                for (int j = 0; j < S::kTiles; j += 2)
                    *reinterpret_cast<float4*>(dst + 2 * j) = make_float4(o[nt][j][e] * f, o[nt][j][2 + e] * f, o[nt][j + 1][e] * f, o[nt][j + 1][2 + e] * f);
            }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == w.a.tiles;
        const int slot = int(blockIdx.x) * 2 + (t0 > 0 ? 0 : 1);
        for (int e = threadIdx.x; e < rows * (kDim / 4); e += S::kThreads) {
            const int r = e / (kDim / 4), d = e % (kDim / 4) * 4;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < S::kWarps; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(join + (k * S::kRows + r) * S::kJoinRow + d);
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
        x += t1 - t0;
        if (x >= x_end) break;
        attend_next_unit(p, w);
        __syncthreads();                                               // the join's memory becomes the ring again
    }
}

template <int kDim, int kNT>
int attend_four_one(bool launch, int* tile, int* per_sm, const AttendParams* p, int ctas, cudaStream_t stream) {
    using S = FourShape<kDim, kNT>;
    if (!launch) {
        *tile = S::kTile;
        *per_sm = S::kCtasPerSm;
        return TL_OK;
    }
    if (int rc = ensure_smem_attr(reinterpret_cast<const void*>(attend_four_kernel<kDim, kNT>), S::kSmem)) return rc;
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
    return check_cuda(cudaLaunchKernelEx(&cfg, attend_four_kernel<kDim, kNT>, *p));
}

}  // namespace tl
