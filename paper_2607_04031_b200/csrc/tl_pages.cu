// Whose pages are whose: reserving, releasing, forking, compacting, and the copies that follow.
//
// The bookkeeping calls are integer work on tables that live on the device, so what they decide must not depend on the order in which
// threads arrive: fresh pages are the lowest free ones in the order of requests and entries, ranks come from prefix sums, and the
// atomics used (counts and minima of integers) give the same result in any order.  reserve, fork and compact run as one cluster of
// kCtas CTAs, each with a share of the pool and of the requests; what the CTAs tell one another goes through the workspace, between
// barriers of the cluster.
#include "tl_kv_rows.cuh"

#include <algorithm>

namespace tl {

struct PageView {
    int32_t* table;
    int32_t* held;
    int32_t* holders;
    int64_t table_stride;
    int requests, pages, page_shift;
};

constexpr int kPageCtas = 8, kPageThreads = 1024, kPageWarps = kPageThreads / 32;

// What a reserving call keeps per page it may take from somebody (written before it is read).
struct PageClaim {
    unsigned long long first;            // lowest (request, entry) that is to write the page
    uint32_t here;                       // how many are to
    uint32_t pad;
};

// Orders everything the cluster's threads have done before, global memory included.
__device__ __forceinline__ void page_sync() {
    __syncwarp();                                             // (loops in front of it may end lane by lane)
    cluster_sync();
}

// Sum of one number per thread in front of the thread, and of all (whole CTA).
template <typename T>
__device__ __forceinline__ T block_scan(T x, T* shared, T* total) {
    const int lane = int(lane_id()), warp = int(threadIdx.x) / 32;
    T run = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, run, d);
        if (lane >= d) run += up;
    }
    __syncthreads();                                          // (the last scan's sums have been read)
    if (lane == 31) shared[warp] = run;
    __syncthreads();
    T sums = shared[lane];                                    // kPageWarps == 32
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T up = __shfl_up_sync(0xffffffffu, sums, d);
        if (lane >= d) sums += up;
    }
    *total = __shfl_sync(0xffffffffu, sums, 31);
    const T before = __shfl_sync(0xffffffffu, sums, (warp + 31) & 31);
    return (warp ? before : 0) + run - x;
}
static_assert(kPageWarps == 32, "block_scan");

// The CTA's share of the pool: a multiple of four pages, in order.
__device__ __forceinline__ void pool_share(int pages, int rank, int* from, int* to) {
    const int64_t each = ((int64_t(pages) + kPageCtas - 1) / kPageCtas + 3) / 4 * 4;
    *from = int(min(int64_t(pages), rank * each));
    *to = int(min(int64_t(pages), (rank + 1) * each));
}

struct ReserveParams {
    PageView t;
    const int32_t* start;
    const int32_t* tokens;
    int32_t* moves;
    int32_t* n_moves;
    int32_t* missing;
    PageClaim* claims;                   // [pages]
    int32_t* fresh;                      // [requests]: fresh pages it needs, then how many the requests in front of it need
    int32_t* copies;                     // [requests]: likewise pages to copy
    int32_t* free_list;                  // [pages]: the pages to be taken, then those given up for them (-1: none)
    int32_t* cta_free;                   // [kPageCtas]
    uint32_t* status;
};

struct ReserveRange {
    int have, need;                      // pages held and wanted
    int first, last;                     // entries to be written among those held
    int start;
};
__device__ __forceinline__ ReserveRange reserve_range(const ReserveParams& p, int b, bool* clipped) {
    ReserveRange r;
    const int tokens = p.tokens[b];
    r.start = max(p.start[b], 0);
    r.have = int(min(int64_t(max(p.t.held[b], 0)), p.t.table_stride));
    const int64_t need = tokens < 0 ? 0 : (int64_t(tokens) + (1 << p.t.page_shift) - 1) >> p.t.page_shift;
    if (need > p.t.table_stride) *clipped = true;
    r.need = int(min(need, p.t.table_stride));
    r.first = r.start >> p.t.page_shift;
    r.last = tokens > r.start ? min(r.need, r.have) : 0;
    return r;
}
// Whether an entry's page has other holders.
__device__ __forceinline__ bool entry_shared(const PageView& t, int page) { return page >= 0 && page < t.pages && t.holders[page] > 1; }
// Whether the entry gives its shared page up (another of those that are to write it keeps it, or somebody who is not).
__device__ __forceinline__ bool entry_leaves(const ReserveParams& p, int b, int e, int page) {
    const PageClaim c = p.claims[page];
    return !(int64_t(c.here) == p.t.holders[page] && c.first == (static_cast<unsigned long long>(b) << 32 | uint32_t(e)));
}

__global__ void __cluster_dims__(kPageCtas, 1, 1) __launch_bounds__(kPageThreads) page_reserve_kernel(const ReserveParams p) {
    __shared__ int64_t sums_wide[kPageWarps];
    __shared__ int sums[kPageWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = int(cluster_cta_rank()), lane = int(lane_id()), warp = rank * kPageWarps + int(threadIdx.x) / 32;
    constexpr int kWarps = kPageCtas * kPageWarps;
    bool clipped = false, bad = false;
    // claims on shared pages: cleared, then counted
    for (int b = warp; b < p.t.requests; b += kWarps) {
        const ReserveRange r = reserve_range(p, b, &clipped);
        for (int e = r.first + lane; e < r.last; e += 32) {
            const int page = p.t.table[int64_t(b) * p.t.table_stride + e];
            bad |= page < 0 || page >= p.t.pages;
            if (entry_shared(p.t, page)) p.claims[page] = PageClaim{~0ull, 0u, 0u};
        }
    }
    page_sync();
    for (int b = warp; b < p.t.requests; b += kWarps) {
        const ReserveRange r = reserve_range(p, b, &clipped);
        for (int e = r.first + lane; e < r.last; e += 32) {
            const int page = p.t.table[int64_t(b) * p.t.table_stride + e];
            if (!entry_shared(p.t, page)) continue;
            atomicAdd(&p.claims[page].here, 1u);
            atomicMin(&p.claims[page].first, static_cast<unsigned long long>(b) << 32 | uint32_t(e));
        }
    }
    // free pages of this CTA's share
    int from, to;
    pool_share(p.t.pages, rank, &from, &to);
    int mine = 0;
    for (int i = from + int(threadIdx.x); i < to; i += kPageThreads) mine += p.t.holders[i] == 0;
    int found;
    block_scan(mine, sums, &found);
    if (threadIdx.x == 0) p.cta_free[rank] = found;
    page_sync();
    // what every request needs
    for (int b = warp; b < p.t.requests; b += kWarps) {
        const ReserveRange r = reserve_range(p, b, &clipped);
        int leaves = 0;
        bool copy = false;
        for (int e = r.first + lane; e < r.last; e += 32) {
            const int page = p.t.table[int64_t(b) * p.t.table_stride + e];
            if (!entry_shared(p.t, page) || !entry_leaves(p, b, e, page)) continue;
            ++leaves;
            copy |= e == r.first && (r.start & ((1 << p.t.page_shift) - 1)) != 0;
        }
        leaves = __reduce_add_sync(0xffffffffu, leaves);
        copy = __any_sync(0xffffffffu, copy);
        if (lane == 0) {
            p.fresh[b] = leaves + max(0, r.need - r.have);
            p.copies[b] = copy;
        }
    }
    page_sync();
    // sums in front of each request (every CTA for itself; the first one keeps them), the lowest free pages in order
    int64_t total = 0;                                        // (what is asked for may be more than there can be)
    int copies = 0;
    for (int b0 = 0; b0 < p.t.requests; b0 += kPageThreads) {
        const int b = b0 + int(threadIdx.x);
        const int64_t n = b < p.t.requests ? p.fresh[b] : 0;
        const int c = b < p.t.requests ? p.copies[b] : 0;
        int64_t all;
        int all_c;
        const int64_t before = total + block_scan(n, sums_wide, &all);
        const int before_c = copies + block_scan(c, sums, &all_c);
        total += all;
        copies += all_c;
        page_sync();                                       // (every CTA has read this part)
        if (rank == 0 && b < p.t.requests) p.fresh[b] = int(min(before, int64_t(INT32_MAX))), p.copies[b] = before_c;
    }
    int at = 0, there = 0;
    for (int c = 0; c < kPageCtas; ++c) {
        const int f = p.cta_free[c];
        if (c < rank) at += f;
        there += f;
    }
    const bool enough = there >= total;
    for (int i0 = from; enough && i0 < to && at < total; i0 += kPageThreads) {
        const int i = i0 + int(threadIdx.x);
        const int f = i < to && p.t.holders[i] == 0;
        int all;
        const int place = at + block_scan(f, sums, &all);
        if (f && place < total) p.free_list[place] = i;
        at += all;
    }
    page_sync();
    if (rank == 0 && threadIdx.x == 0) {
        *p.missing = enough ? 0 : int(min(total - there, int64_t(INT32_MAX)));
        *p.n_moves = enough ? copies : 0;
    }
    // (nothing above has changed the tables; holders of shared pages change when all entries have been decided on)
    for (int b = warp; enough && b < p.t.requests; b += kWarps) {
        const ReserveRange r = reserve_range(p, b, &clipped);
        int place = p.fresh[b];
        int32_t* const row = p.t.table + int64_t(b) * p.t.table_stride;
        for (int e0 = min(r.first, r.have); e0 < r.need; e0 += 32) {
            const int e = e0 + lane;
            bool leave = false;
            int page = -1;
            if (e >= r.first && e < r.last) {
                page = row[e];
                leave = page >= 0 && page < p.t.pages && p.t.holders[page] > 1 && entry_leaves(p, b, e, page);
            }
            const bool take = leave || (e >= r.have && e < r.need);
            const uint32_t who = __ballot_sync(0xffffffffu, take);
            if (take) {
                int32_t* const line = p.free_list + place + __popc(who & ((1u << lane) - 1u));
                const int to_page = *line;
                *line = leave ? page : -1;
                if (leave && e == r.first && (r.start & ((1 << p.t.page_shift) - 1)) != 0) {
                    int32_t* const m = p.moves + int64_t(p.copies[b]) * 3;
                    m[0] = page, m[1] = to_page, m[2] = r.start & ((1 << p.t.page_shift) - 1);
                }
                row[e] = to_page;
                p.t.holders[to_page] = 1;
            }
            place += __popc(who);
        }
        __syncwarp();
        if (lane == 0 && p.t.held[b] < r.need) p.t.held[b] = r.need;
    }
    page_sync();
    for (int i = rank * kPageThreads + int(threadIdx.x); enough && i < total; i += kPageCtas * kPageThreads)
        if (p.free_list[i] >= 0) atomicSub(&p.t.holders[p.free_list[i]], 1);
    if (clipped || bad) atomicCAS(p.status, 0u, kBadPage);
}

// A warp per request: the entries behind those it keeps.
__global__ void __launch_bounds__(256) page_release_kernel(const PageView t, const int32_t* tokens, uint32_t* status) {
    pdl_wait();
    pdl_launch_dependents();
    const int b = int(blockIdx.x) * 8 + int(threadIdx.x) / 32;
    if (b >= t.requests) return;
    const int have = int(min(int64_t(max(t.held[b], 0)), t.table_stride)), keep = tokens ? tokens[b] : 0;
    if (keep < 0) return;
    const int kept = int(min((int64_t(keep) + (1 << t.page_shift) - 1) >> t.page_shift, int64_t(have)));
    int32_t* const row = t.table + int64_t(b) * t.table_stride;
    bool bad = false;
    for (int e = kept + int(lane_id()); e < have; e += 32) {
        const int page = row[e];
        row[e] = -1;
        if (page < 0 || page >= t.pages) bad = true;
        else if (atomicSub(&t.holders[page], 1) <= 0) atomicAdd(&t.holders[page], 1), bad = true;
    }
    __syncwarp();
    if (lane_id() == 0) t.held[b] = kept;
    if (bad) atomicCAS(status, 0u, kBadPage);
}

struct ForkParams {
    PageView t;
    const int32_t* from;
    const int32_t* to;
    const int32_t* tokens;
    int32_t* entries;                    // [forks]: pages to share, -1: the fork is left out
    int forks;
    uint32_t* status;
};
__global__ void __cluster_dims__(kPageCtas, 1, 1) __launch_bounds__(kPageThreads) page_fork_kernel(const ForkParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int rank = int(cluster_cta_rank()), lane = int(lane_id());
    constexpr int kAll = kPageCtas * kPageThreads;
    const int thread = rank * kPageThreads + int(threadIdx.x), warp = thread / 32;
    bool refused = false, bad = false;
    for (int f = thread; f < p.forks; f += kAll) {
        const int from = p.from[f], to = p.to[f];
        int n = -1;
        if (from >= 0 && from < p.t.requests && to >= 0 && to < p.t.requests && p.t.held[to] == 0) {
            const int64_t want = (int64_t(max(p.tokens[f], 0)) + (1 << p.t.page_shift) - 1) >> p.t.page_shift;
            n = int(min(want, min(int64_t(max(p.t.held[from], 0)), p.t.table_stride)));
        }
        p.entries[f] = n;
    }
    page_sync();
    // of several forks to one request the first has it: the lowest of their marks, which are negative
    for (int f = thread; f < p.forks; f += kAll)
        if (p.entries[f] >= 0) atomicMin(&p.t.held[p.to[f]], f - p.forks);
    page_sync();
    for (int f = thread; f < p.forks; f += kAll) {
        if (p.entries[f] >= 0 && p.t.held[p.to[f]] != f - p.forks) p.entries[f] = -1;
        refused |= p.entries[f] < 0;
    }
    page_sync();
    // (a request that is forked to holds nothing, so no row is read that is written here)
    for (int f = warp; f < p.forks; f += kAll / 32) {
        const int n = p.entries[f];
        if (n < 0) continue;
        const int32_t* const src = p.t.table + int64_t(p.from[f]) * p.t.table_stride;
        int32_t* const dst = p.t.table + int64_t(p.to[f]) * p.t.table_stride;
        for (int e = lane; e < n; e += 32) {
            const int page = src[e];
            dst[e] = page;
            if (page < 0 || page >= p.t.pages) bad = true;
            else atomicAdd(&p.t.holders[page], 1);
        }
        if (lane == 0) p.t.held[p.to[f]] = n;
    }
    if (refused) atomicCAS(p.status, 0u, kBadFork);
    if (bad) atomicCAS(p.status, 0u, kBadPage);
}

struct CompactParams {
    PageView t;
    int32_t* moves;
    int32_t* n_moves;
    int32_t* in_use;
    int32_t* went;                       // [pages]: where a page behind the last one in use went (itself: nowhere)
    int32_t* cta_live;                   // [kPageCtas]: pages in use in each CTA's share; then the moves, then all pages in use
    int most;
    uint32_t* status;
};
__global__ void __cluster_dims__(kPageCtas, 1, 1) __launch_bounds__(kPageThreads) page_compact_kernel(const CompactParams p) {
    __shared__ int sums[kPageWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = int(cluster_cta_rank());
    int from, to;
    pool_share(p.t.pages, rank, &from, &to);
    int mine = 0;
    for (int i = from + int(threadIdx.x); i < to; i += kPageThreads) mine += p.t.holders[i] > 0;
    int found;
    block_scan(mine, sums, &found);
    if (threadIdx.x == 0) p.cta_live[rank] = found;
    page_sync();
    int live = 0, before = 0;
    for (int c = 0; c < kPageCtas; ++c) {
        const int n = p.cta_live[c];
        if (c < rank) before += n;
        live += n;
    }
    // Pages in use from `live` on, the highest first, and free places in front of it, the lowest first: as many of one as of the
    // other.
    for (int i0 = from; i0 < to; i0 += kPageThreads) {
        const int i = i0 + int(threadIdx.x);
        const int used = i < to && p.t.holders[i] > 0;
        int all;
        const int in_front = before + block_scan(used, sums, &all);
        before += all;
        if (i >= to) continue;
        if (i == live - 1) p.cta_live[kPageCtas] = live - in_front - used;       // places in front of `live` that are free
        if (i < live && !used) {
            const int r = i - in_front;
            if (r < p.most) p.moves[int64_t(r) * 3 + 1] = i;
        } else if (i >= live) {
            const int r = live - 1 - in_front;
            if (used && r < p.most) p.moves[int64_t(r) * 3] = i;
            p.went[i] = i;
        }
    }
    page_sync();
    const int moves = min(live == 0 ? 0 : p.cta_live[kPageCtas], p.most);
    for (int r = rank * kPageThreads + int(threadIdx.x); r < moves; r += kPageCtas * kPageThreads) {
        const int a = p.moves[int64_t(r) * 3], b = p.moves[int64_t(r) * 3 + 1];
        p.moves[int64_t(r) * 3 + 2] = 1 << p.t.page_shift;
        p.went[a] = b;
        p.t.holders[b] = p.t.holders[a];
        p.t.holders[a] = 0;
    }
    if (rank == 0 && threadIdx.x == 0) {
        *p.n_moves = moves;
        *p.in_use = live;
        p.cta_live[kPageCtas + 1] = live;
    }
}

// The tables after the moves.  A warp per request.
__global__ void __launch_bounds__(256) page_rename_kernel(const PageView t, const int32_t* went, const int32_t* live, uint32_t* status) {
    pdl_wait();
    pdl_launch_dependents();
    const int from = *live;
    bool bad = false;
    const int b = int(blockIdx.x) * 8 + int(threadIdx.x) / 32;
    if (b >= t.requests) return;
    const int have = int(min(int64_t(max(t.held[b], 0)), t.table_stride));
    int32_t* const row = t.table + int64_t(b) * t.table_stride;
    for (int e = int(lane_id()); e < have; e += 32) {
        const int page = row[e];
        if (page < 0 || page >= t.pages) bad = true;
        else if (page >= from) row[e] = went[page];
    }
    if (bad) atomicCAS(status, 0u, kBadPage);
}

struct PageCopyParams {
    KvView from, to;
    const int32_t* moves;
    const int32_t* n_moves;
    int most;
    int piece_shift;                     // 16-byte pieces of a token's row, as a shift
    int group_shift;                     // 4-byte words of its group scales, as a shift; -1: it has none
    uint32_t* status;
};
constexpr int kPageCopyThreads = 256, kPageCopyAhead = 8;

// A warp takes one head's keys or values of one page: its rows in 16-byte pieces, several in flight, then their scales.
__global__ void __launch_bounds__(kPageCopyThreads) page_copy_kernel(const PageCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int n = p.n_moves ? min(max(*p.n_moves, 0), p.most) : p.most;
    const int lane = int(lane_id()), each = 2 * p.from.heads, page_tokens = 1 << p.from.page_shift;
    const int64_t items = int64_t(n) * each;
    for (int64_t item = blockIdx.x * int64_t(kPageCopyThreads / 32) + threadIdx.x / 32; item < items; item += int64_t(gridDim.x) * (kPageCopyThreads / 32)) {
        const int64_t move = item / each;
        const int rest = int(item - move * each), which = rest & 1, head = rest >> 1;
        const int64_t a = p.moves[move * 3], b = p.moves[move * 3 + 1];
        const int rows = min(max(p.moves[move * 3 + 2], 0), page_tokens);
        if (a < 0 || a >= p.from.pages || b < 0 || b >= p.to.pages) {
            if (lane == 0) atomicCAS(p.status, 0u, kBadPage);
            continue;
        }
        const char* const src = p.from.base[which] + a * p.from.page_stride + int64_t(head) * p.from.head_stride;
        char* const dst = p.to.base[which] + b * p.to.page_stride + int64_t(head) * p.to.head_stride;
        const int pieces = rows << p.piece_shift;
        for (int i0 = lane; i0 < pieces; i0 += 32 * kPageCopyAhead) {
            uint4 v[kPageCopyAhead];
#pragma unroll
            for (int k = 0; k < kPageCopyAhead; ++k) {
                const int i = i0 + 32 * k;
                if (i < pieces) v[k] = *reinterpret_cast<const uint4*>(src + int64_t(i >> p.piece_shift) * p.from.token_stride + (i & ((1 << p.piece_shift) - 1)) * 16);
            }
#pragma unroll
            for (int k = 0; k < kPageCopyAhead; ++k) {
                const int i = i0 + 32 * k;
                if (i < pieces) *reinterpret_cast<uint4*>(dst + int64_t(i >> p.piece_shift) * p.to.token_stride + (i & ((1 << p.piece_shift) - 1)) * 16) = v[k];
            }
        }
        if (p.from.scale[0]) {
            const float* const s = p.from.scale[which] + a * p.from.scale_page_stride + int64_t(head) * p.from.scale_head_stride;
            float* const d = p.to.scale[which] + b * p.to.scale_page_stride + int64_t(head) * p.to.scale_head_stride;
            for (int i = lane; i < rows; i += 32) d[i] = s[i];
        }
        if (p.group_shift >= 0) {
            const uint32_t* const s = reinterpret_cast<const uint32_t*>(p.from.group[which] + a * p.from.group_page_stride + int64_t(head) * p.from.group_head_stride);
            uint32_t* const d = reinterpret_cast<uint32_t*>(p.to.group[which] + b * p.to.group_page_stride + int64_t(head) * p.to.group_head_stride);
            for (int i = lane; i < rows << p.group_shift; i += 32) d[i] = s[i];
        }
    }
}

static int page_view(const tl_page_tables* t, PageView* out) {
    if (!t || t->requests < 0 || t->pages < 1 || t->page_tokens < 1) return TL_ERR_INVALID_ARG;
    if (!t->holders || (t->requests > 0 && (!t->page_table || !t->held || t->table_stride < 1))) return TL_ERR_INVALID_ARG;
    if (!is_pow2(t->page_tokens) || t->page_tokens < 16 || t->page_tokens > 1024) return TL_ERR_UNSUPPORTED;
    if (t->pages > (1 << 30) || t->table_stride > (int64_t(1) << 30)) return TL_ERR_UNSUPPORTED;
    if (!words_aligned(t->page_table, t->held, t->holders)) return TL_ERR_ALIGNMENT;
    out->table = t->page_table;
    out->held = t->held;
    out->holders = t->holders;
    out->table_stride = t->table_stride;
    out->requests = t->requests;
    out->pages = t->pages;
    out->page_shift = 0;
    while ((1 << out->page_shift) < t->page_tokens) ++out->page_shift;
    return TL_OK;
}

static size_t up16(size_t n) { return (n + 15) / 16 * 16; }
static size_t page_workspace(const PageView& t, int forks) {
    const size_t reserve = up16(size_t(t.pages) * sizeof(PageClaim)) + up16(size_t(t.requests) * 4) * 2 + up16(size_t(t.pages) * 4) + 256;
    return std::max(reserve, up16(size_t(forks) * 4));        // (compacting takes less than reserving)
}

}  // namespace tl

extern "C" {

size_t tl_page_workspace_bytes(const tl_page_tables* tables, int forks) {
    using namespace tl;
    PageView t;
    if (page_view(tables, &t) || forks < 0) return 0;
    return page_workspace(t, forks);
}

int tl_page_reserve(const tl_page_tables* tables, const int32_t* d_start, const int32_t* d_tokens, int32_t* d_moves, int32_t* d_n_moves,
                    int32_t* d_missing, void* cuda_stream) {
    using namespace tl;
    ReserveParams p = {};
    if (int rc = page_view(tables, &p.t)) return rc;
    if (!d_n_moves || !d_missing || (p.t.requests > 0 && (!d_start || !d_tokens || !d_moves))) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_start, d_tokens, d_moves, d_n_moves, d_missing)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    void* ws = nullptr;
    if (int rc = get_workspace(page_workspace(p.t, 0), &ws, stream)) return rc;
    char* at = static_cast<char*>(ws);
    p.claims = reinterpret_cast<PageClaim*>(at), at += up16(size_t(p.t.pages) * sizeof(PageClaim));
    p.fresh = reinterpret_cast<int32_t*>(at), at += up16(size_t(p.t.requests) * 4);
    p.copies = reinterpret_cast<int32_t*>(at), at += up16(size_t(p.t.requests) * 4);
    p.free_list = reinterpret_cast<int32_t*>(at), at += up16(size_t(p.t.pages) * 4);
    p.cta_free = reinterpret_cast<int32_t*>(at);
    p.start = d_start;
    p.tokens = d_tokens;
    p.moves = d_moves;
    p.n_moves = d_n_moves;
    p.missing = d_missing;
    p.status = dev().ctl.d_status;
    return kv_launch(page_reserve_kernel, dim3(kPageCtas), kPageThreads, stream, p);
}

int tl_page_release(const tl_page_tables* tables, const int32_t* d_tokens, void* cuda_stream) {
    using namespace tl;
    PageView t;
    if (int rc = page_view(tables, &t)) return rc;
    if (!words_aligned(d_tokens)) return TL_ERR_ALIGNMENT;
    if (t.requests == 0) return TL_OK;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    return kv_launch(page_release_kernel, dim3(unsigned(ceil_div(t.requests, 8))), 256, static_cast<cudaStream_t>(cuda_stream), t, d_tokens,
                     dev().ctl.d_status);
}

int tl_page_fork(const tl_page_tables* tables, const int32_t* d_from, const int32_t* d_to, const int32_t* d_tokens, int forks,
                 void* cuda_stream) {
    using namespace tl;
    ForkParams p = {};
    if (int rc = page_view(tables, &p.t)) return rc;
    if (forks < 0 || (forks > 0 && (!d_from || !d_to || !d_tokens))) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_from, d_to, d_tokens)) return TL_ERR_ALIGNMENT;
    if (forks == 0) return TL_OK;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    void* ws = nullptr;
    if (int rc = get_workspace(page_workspace(p.t, forks), &ws, stream)) return rc;
    p.from = d_from;
    p.to = d_to;
    p.tokens = d_tokens;
    p.entries = static_cast<int32_t*>(ws);
    p.forks = forks;
    p.status = dev().ctl.d_status;
    return kv_launch(page_fork_kernel, dim3(kPageCtas), kPageThreads, stream, p);
}

int tl_page_compact(const tl_page_tables* tables, int32_t* d_moves, int most, int32_t* d_n_moves, int32_t* d_in_use, void* cuda_stream) {
    using namespace tl;
    CompactParams p = {};
    if (int rc = page_view(tables, &p.t)) return rc;
    if (most < 0 || (most > 0 && !d_moves) || !d_n_moves || !d_in_use) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_moves, d_n_moves, d_in_use)) return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    void* ws = nullptr;
    if (int rc = get_workspace(page_workspace(p.t, 0), &ws, stream)) return rc;
    p.went = static_cast<int32_t*>(ws);
    p.cta_live = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + up16(size_t(p.t.pages) * 4));
    p.moves = d_moves;
    p.n_moves = d_n_moves;
    p.in_use = d_in_use;
    p.most = most;
    p.status = dev().ctl.d_status;
    if (int rc = kv_launch(page_compact_kernel, dim3(kPageCtas), kPageThreads, stream, p)) return rc;
    if (p.t.requests == 0) return TL_OK;
    return kv_launch(page_rename_kernel, dim3(unsigned(ceil_div(p.t.requests, 8))), 256, stream, p.t, const_cast<const int32_t*>(p.went),
                     const_cast<const int32_t*>(p.cta_live + kPageCtas + 1), p.status);
}

int tl_page_copy(const tl_kv_cache* from, const tl_kv_cache* to, const int32_t* d_moves, const int32_t* d_n_moves, int most,
                 void* cuda_stream) {
    using namespace tl;
    PageCopyParams p = {};
    if (int rc = kv_view(from, &p.from)) return rc;
    if (int rc = kv_view(to, &p.to)) return rc;
    if (from->format != to->format || from->heads != to->heads || from->head_dim != to->head_dim || from->page_tokens != to->page_tokens)
        return TL_ERR_INVALID_ARG;
    if (most < 0 || (most > 0 && !d_moves)) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_moves, d_n_moves)) return TL_ERR_ALIGNMENT;
    if (most == 0) return TL_OK;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_control()) return rc;
    p.moves = d_moves;
    p.n_moves = d_n_moves;
    p.most = most;
    p.status = dev().ctl.d_status;
    const int64_t pieces = kv_bytes(from->format, from->head_dim) / 16;
    while ((1 << p.piece_shift) < pieces) ++p.piece_shift;
    p.group_shift = -1;
    if (from->format == TL_KV_E2M1) p.group_shift = from->head_dim == 64 ? 0 : from->head_dim == 128 ? 1 : 2;
    const int64_t items = int64_t(most) * 2 * from->heads;
    const int64_t blocks = std::min<int64_t>(ceil_div(items, kPageCopyThreads / 32), int64_t(dev().sm_count) * 8);
    return kv_launch(page_copy_kernel, dim3(unsigned(blocks)), kPageCopyThreads, static_cast<cudaStream_t>(cuda_stream), p);
}

}  // extern "C"
