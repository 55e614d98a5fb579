// Whose pages are whose: reserving, releasing, forking, compacting, and the copies that follow.
//
// The bookkeeping calls are integer work on tables that live on the device, so what they decide must not depend on the order in which
// threads arrive: fresh pages are the lowest free ones in the order of requests and entries, ranks come from prefix sums, and the
// atomics used (counts and minima of integers) give the same result in any order.  reserve and compact look through the whole pool,
// 32 pages per thread, in one CTA or (a large pool) one cluster; what threads tell one another goes through the workspace, between
// barriers.
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

constexpr int kPageThreads = 1024, kPageWarps = kPageThreads / 32;
// CTAs that look through a pool: one, whose barriers cost little, or (larger pools) a cluster of eight.  us per call, one CTA / cluster, 512
// requests, calls back to back:
//   reserve (nothing to take)     32768 pages 6.1 (the host's call) / 11.7, 65536 8.6 / 11.6, 131072 14.2 / 11.8, 2^20 92 / 18.6
//   compact (nothing to move)     16384 pages 11.5 / 14.2, 32768 13.0 / 14.9, 65536 28 / 16.3, 131072 57 / 16.7, 2^20 469 / 73
// One turn of one CTA is 32768 pages; compacting touches every page of a turn, reserving only as many as it takes.
constexpr int kPageCtas = 8, kReserveOfOne = 1 << 16, kCompactOfOne = 1 << 15;

// What a reserving call keeps per page it may take from somebody (written before it is read).
struct PageClaim {
    unsigned long long first;            // lowest (request, entry) that is to write the page
    uint32_t here;                       // how many are to
    uint32_t pad;
};

// Orders everything the threads have done before, global memory included.
template <int kCtas>
__device__ __forceinline__ void page_sync() {
    __syncwarp();                                             // (loops in front of it may end lane by lane)
    if (kCtas > 1) cluster_sync();
    else __syncthreads();
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

// The pool is looked through 32 pages per thread at a time, in the order of turns, CTAs and threads.  Bit i: page first + i is free
// (or, used: is in use); pages past the end are neither.  Whole warp (of consecutive threads): a load of 32 neighbouring pages gives
// one thread its word.
__device__ __forceinline__ uint32_t page_bits(const PageView& t, int64_t first, bool used) {
    const int lane = int(lane_id());
    const int64_t base = first - int64_t(lane) * 32;
    uint32_t bits = 0;
    int v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const int64_t i = base + j * 32 + lane;
        v[j] = i < t.pages ? t.holders[i] : used ? 0 : 1;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const uint32_t word = __ballot_sync(0xffffffffu, (v[j] == 0) != used);
        if (lane == j) bits = word;
    }
    return bits;
}
// Sum of the first n numbers of a list, by a whole warp.
__device__ __forceinline__ int64_t warp_sum(const int32_t* list, int n) {
    int64_t sum = 0;
    for (int i = int(lane_id()); i < n; i += 32) sum += list[i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum;
}

struct ReserveParams {
    PageView t;
    const int32_t* start;
    const int32_t* tokens;
    int32_t* moves;
    int32_t* n_moves;
    int32_t* missing;
    PageClaim* claims;                   // [pages]
    int32_t* free_list;                  // [pages]: the pages to be taken, then those given up for them (-1: none)
    int32_t* counts;                     // (cluster) [turns of the pool * CTAs]: free pages
    int32_t* fresh;                      // (cluster) [turns of the requests * CTAs]: pages to be taken, one CTA's (at most INT32_MAX)
    int32_t* copies;                     // (cluster) likewise pages to copy
    uint32_t* status;
};

struct ReserveRange {
    int have, need;                      // pages held and wanted
    int first, last;                     // entries to be written among those held
    int line;                            // rows of entry `first` in front of the position it is written from
};
__device__ __forceinline__ ReserveRange reserve_range(const ReserveParams& p, int b, bool* clipped) {
    ReserveRange r = {0, 0, 0, 0, 0};
    if (b >= p.t.requests) return r;
    const int tokens = p.tokens[b], start = max(p.start[b], 0);
    r.have = int(min(int64_t(max(p.t.held[b], 0)), p.t.table_stride));
    const int64_t need = tokens < 0 ? 0 : (int64_t(tokens) + (1 << p.t.page_shift) - 1) >> p.t.page_shift;
    if (need > p.t.table_stride) *clipped = true;
    r.need = int(min(need, p.t.table_stride));
    r.first = start >> p.t.page_shift;
    r.last = tokens > start ? min(r.need, r.have) : 0;
    r.line = start & ((1 << p.t.page_shift) - 1);
    return r;
}
// Calls f(request, entry, page) for every entry to be written, a request per lane; f's result (0 or 1) is added up for the request.
// Few entries are their lane's, a long range is taken by the whole warp.
template <typename F>
__device__ __forceinline__ int for_entries(const PageView& t, int b, const ReserveRange& r, F f) {
    constexpr int kFew = 2;
    const int n = max(r.last - r.first, 0);
    int sum = 0;
    if (n <= kFew)
        for (int e = r.first; e < r.last; ++e) sum += f(b, e, t.table[int64_t(b) * t.table_stride + e]);
    __syncwarp();
    for (uint32_t many = __ballot_sync(0xffffffffu, n > kFew); many; many &= many - 1) {
        const int l = __ffs(int(many)) - 1, b1 = __shfl_sync(0xffffffffu, b, l);
        const int first = __shfl_sync(0xffffffffu, r.first, l), last = __shfl_sync(0xffffffffu, r.last, l);
        int part = 0;
        for (int e = first + int(lane_id()); e < last; e += 32) part += f(b1, e, t.table[int64_t(b1) * t.table_stride + e]);
        part = __reduce_add_sync(0xffffffffu, part);
        if (int(lane_id()) == l) sum = part;
    }
    return sum;
}

template <int kCtas>
__global__ void __launch_bounds__(kPageThreads) page_reserve_kernel(const ReserveParams p) {
    __shared__ int64_t sums_wide[kPageWarps];
    __shared__ int sums[kPageWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = kCtas > 1 ? int(cluster_cta_rank()) : 0, lane = int(lane_id());
    constexpr int kAll = kCtas * kPageThreads;
    const int thread = rank * kPageThreads + int(threadIdx.x);
    const int turns = int((int64_t(p.t.pages) + kAll * 32 - 1) / (kAll * 32)), rounds = (p.t.requests + kAll - 1) / kAll;
    bool clipped = false, bad = false;
    const ReserveRange mine = reserve_range(p, thread, &clipped);
    auto range = [&](int round) { return round == 0 ? mine : reserve_range(p, thread + round * kAll, &clipped); };
    auto shared = [&](int page) { return page >= 0 && page < p.t.pages && p.t.holders[page] > 1; };
    auto order = [](int b, int e) { return static_cast<unsigned long long>(b) << 32 | uint32_t(e); };
    // whether an entry gives its shared page up: another of those that are to write it keeps it, or somebody who is not
    auto leaves = [&](int b, int e, int page) {
        const PageClaim c = p.claims[page];
        return !(int64_t(c.here) == p.t.holders[page] && c.first == order(b, e));
    };

    // free pages
    uint32_t bits0 = 0;
    int64_t there = 0, total = 0;                             // free pages, pages to be taken (cluster: added up below)
    int copies = 0;
    int place_first = 0;                                      // free pages of the first turn in front of the thread's, in its CTA
    for (int k = 0; k < turns; ++k) {
        const uint32_t bits = page_bits(p.t, (int64_t(k) * kAll + thread) * 32, false);
        int found;
        const int before = block_scan(__popc(bits), sums, &found);
        if (k == 0) bits0 = bits, place_first = before;
        there += found;
        if (kCtas > 1 && threadIdx.x == 0) p.counts[k * kCtas + rank] = found;
    }
    // claims on shared pages: cleared, then counted
    int any = 0;
    for (int k = 0; k < rounds; ++k)
        any |= for_entries(p.t, thread + k * kAll, range(k), [&](int, int, int page) {
            bad |= page < 0 || page >= p.t.pages;
            if (!shared(page)) return 0;
            p.claims[page] = PageClaim{~0ull, 0u, 0u};
            return 1;
        });
    // (without shared pages, as in most steps, there is nothing to count)
    const bool claims = kCtas > 1 || __syncthreads_or(any) != 0;
    if (claims) {
        page_sync<kCtas>();
        for (int k = 0; k < rounds; ++k)
            for_entries(p.t, thread + k * kAll, range(k), [&](int b, int e, int page) {
                if (!shared(page)) return 0;
                atomicAdd(&p.claims[page].here, 1u);
                atomicMin(&p.claims[page].first, order(b, e));
                return 0;
            });
        page_sync<kCtas>();
    }
    // what every request needs, and the sums of it
    int fresh0 = 0, copies0 = 0;                              // of the thread's first request
    auto needs = [&](int k, int* copy) {
        const ReserveRange r = range(k);
        int first_leaves = 0;
        const int gone = !claims ? 0 : for_entries(p.t, thread + k * kAll, r, [&](int b, int e, int page) { return int(shared(page) && leaves(b, e, page)); });
        if (gone && r.line != 0) {
            const int b = thread + k * kAll, page = p.t.table[int64_t(b) * p.t.table_stride + r.first];
            first_leaves = shared(page) && leaves(b, r.first, page);
        }
        *copy = first_leaves;
        return gone + max(0, r.need - r.have);
    };
    for (int k = 0; k < rounds; ++k) {
        int copy, all_c;
        const int64_t n = needs(k, &copy);
        int64_t all;
        const int64_t before = block_scan(n, sums_wide, &all);
        const int before_c = block_scan(copy, sums, &all_c);
        if (k == 0) fresh0 = int(min(before, int64_t(INT32_MAX))), copies0 = before_c;
        total += all;
        copies += all_c;
        if (kCtas > 1 && threadIdx.x == 0) {
            p.fresh[k * kCtas + rank] = int(min(all, int64_t(INT32_MAX)));
            p.copies[k * kCtas + rank] = all_c;
        }
    }
    if (kCtas > 1) {
        page_sync<kCtas>();
        total = warp_sum(p.fresh, rounds * kCtas), there = warp_sum(p.counts, turns * kCtas);
        copies = int(warp_sum(p.copies, rounds * kCtas));
    }
    const bool enough = there >= total;
    if (thread == 0) {
        *p.missing = enough ? 0 : int(min(total - there, int64_t(INT32_MAX)));
        *p.n_moves = enough ? copies : 0;
    }
    // the lowest free pages, in order
    int64_t passed = 0;                                       // free pages of the turns gone by (one CTA)
    for (int k = 0; enough && k < turns; ++k) {
        const int64_t base = kCtas > 1 ? warp_sum(p.counts, k * kCtas + rank) : passed;
        if (base >= total) break;                             // (the same for the whole CTA)
        const int64_t first = (int64_t(k) * kAll + thread) * 32;
        uint32_t bits = bits0;
        int64_t place = base + place_first;
        if (k > 0 || turns > 1) {
            int all;
            if (k > 0) bits = page_bits(p.t, first, false);
            place = base + block_scan(__popc(bits), sums, &all);
            passed += all;
        }
        for (; bits && place < total; bits &= bits - 1) p.free_list[place++] = int(first) + __ffs(int(bits)) - 1;
    }
    page_sync<kCtas>();
    // (nothing above has changed the tables; holders of shared pages change when all entries have been decided on)
    int64_t taken_before = 0;                                 // by the rounds gone by (one CTA)
    int copied_before = 0;
    for (int k = 0; enough && k < rounds; ++k) {
        const ReserveRange r = range(k);
        int copy = 0;
        int64_t before = fresh0;
        int before_c = copies0;
        int64_t place0 = 0;
        int move0 = 0;
        if (kCtas > 1) place0 = warp_sum(p.fresh, k * kCtas + rank), move0 = int(warp_sum(p.copies, k * kCtas + rank));
        else place0 = taken_before, move0 = copied_before;
        if (k > 0 || rounds > 1) {
            int all_c;
            int64_t all;
            const int64_t n = needs(k, &copy);
            before = block_scan(n, sums_wide, &all);
            before_c = block_scan(copy, sums, &all_c);
            taken_before += all;
            copied_before += all_c;
        }
        place0 += before;
        move0 += before_c;
        // one entry after the other by its request's lane, or (a prompt's pages) by the whole warp
        const int b = thread + k * kAll, from = claims ? min(r.first, r.have) : r.have, n = max(r.need - from, 0);
        auto take = [&](int b1, int e, int first, int last, int have, int64_t place, int page, bool leave, int line, int move) {
            int32_t* const slot = p.free_list + place;
            const int to = *slot;
            *slot = leave ? page : -1;
            if (leave && e == first && line != 0) {
                int32_t* const m = p.moves + int64_t(move) * 3;
                m[0] = page, m[1] = to, m[2] = line;
            }
            p.t.table[int64_t(b1) * p.t.table_stride + e] = to;
            p.t.holders[to] = 1;
        };
        auto leaving = [&](int b1, int e, int first, int last, int* page) {
            if (!claims || e < first || e >= last) return false;
            *page = p.t.table[int64_t(b1) * p.t.table_stride + e];
            return shared(*page) && leaves(b1, e, *page);
        };
        constexpr int kFew = 2;
        if (n <= kFew) {
            int64_t place = place0;
            for (int e = from; e < r.need; ++e) {
                int page = -1;
                const bool leave = leaving(b, e, r.first, r.last, &page);
                if (leave || e >= r.have) take(b, e, r.first, r.last, r.have, place++, page, leave, r.line, move0);
            }
        }
        __syncwarp();
        for (uint32_t many = __ballot_sync(0xffffffffu, n > kFew); many; many &= many - 1) {
            const int l = __ffs(int(many)) - 1, b1 = __shfl_sync(0xffffffffu, b, l), need = __shfl_sync(0xffffffffu, r.need, l);
            const int first = __shfl_sync(0xffffffffu, r.first, l), last = __shfl_sync(0xffffffffu, r.last, l);
            const int have = __shfl_sync(0xffffffffu, r.have, l), line = __shfl_sync(0xffffffffu, r.line, l);
            const int move = __shfl_sync(0xffffffffu, move0, l);
            int64_t place = __shfl_sync(0xffffffffu, place0, l);
            for (int e0 = __shfl_sync(0xffffffffu, from, l); e0 < need; e0 += 32) {
                const int e = e0 + lane;
                int page = -1;
                const bool leave = leaving(b1, e, first, last, &page), taken = leave || (e >= have && e < need);
                const uint32_t who = __ballot_sync(0xffffffffu, taken);
                if (taken) take(b1, e, first, last, have, place + __popc(who & ((1u << lane) - 1u)), page, leave, line, move);
                place += __popc(who);
            }
        }
        if (r.need > r.have) p.t.held[b] = r.need;
    }
    if (claims) {
        page_sync<kCtas>();
        for (int64_t i = thread; enough && i < total; i += kAll)
            if (p.free_list[i] >= 0) atomicSub(&p.t.holders[p.free_list[i]], 1);
    }
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
    constexpr int kAhead = 4;
    for (int e0 = kept + int(lane_id()); e0 < have; e0 += 32 * kAhead) {
        int page[kAhead], had[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) page[k] = e0 + 32 * k < have ? row[e0 + 32 * k] : 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            had[k] = 1;
            if (e0 + 32 * k >= have) continue;
            row[e0 + 32 * k] = -1;
            if (page[k] < 0 || page[k] >= t.pages) bad = true;
            else had[k] = atomicSub(&t.holders[page[k]], 1);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (had[k] <= 0) atomicAdd(&t.holders[page[k]], 1), bad = true;           // (it had no holder)
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
// Which forks are made, and how many pages each shares; `held` is that after the call.  One CTA: every count is read before one is
// written.
__global__ void __launch_bounds__(kPageThreads) page_fork_kernel(const ForkParams p) {
    pdl_wait();
    pdl_launch_dependents();
    bool refused = false;
    for (int f = int(threadIdx.x); f < p.forks; f += kPageThreads) {
        const int from = p.from[f], to = p.to[f];
        int n = -1;
        if (from >= 0 && from < p.t.requests && to >= 0 && to < p.t.requests && p.t.held[to] == 0) {
            const int64_t want = (int64_t(max(p.tokens[f], 0)) + (1 << p.t.page_shift) - 1) >> p.t.page_shift;
            n = int(min(want, min(int64_t(max(p.t.held[from], 0)), p.t.table_stride)));
        }
        p.entries[f] = n;
    }
    __syncthreads();
    // of several forks to one request the first has it: the lowest of their marks, which are negative
    for (int f = int(threadIdx.x); f < p.forks; f += kPageThreads)
        if (p.entries[f] >= 0) atomicMin(&p.t.held[p.to[f]], f - p.forks);
    __syncthreads();
    for (int f = int(threadIdx.x); f < p.forks; f += kPageThreads) {
        if (p.entries[f] >= 0 && *static_cast<volatile int32_t*>(&p.t.held[p.to[f]]) != f - p.forks) p.entries[f] = -1;
        refused |= p.entries[f] < 0;
    }
    __syncthreads();
    for (int f = int(threadIdx.x); f < p.forks; f += kPageThreads)
        if (p.entries[f] >= 0) p.t.held[p.to[f]] = p.entries[f];
    if (refused) atomicCAS(p.status, 0u, kBadFork);
}
// A warp per fork.  (A request that is forked to held nothing, so no row is read that is written here.)
__global__ void __launch_bounds__(256) page_share_kernel(const ForkParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int f = int(blockIdx.x) * 8 + int(threadIdx.x) / 32;
    if (f >= p.forks) return;
    const int n = p.entries[f];
    if (n <= 0) return;
    const int32_t* const src = p.t.table + int64_t(p.from[f]) * p.t.table_stride;
    int32_t* const dst = p.t.table + int64_t(p.to[f]) * p.t.table_stride;
    bool bad = false;
    for (int e = int(lane_id()); e < n; e += 32) {
        const int page = src[e];
        dst[e] = page;
        if (page < 0 || page >= p.t.pages) bad = true;
        else atomicAdd(&p.t.holders[page], 1);
    }
    if (bad) atomicCAS(p.status, 0u, kBadPage);
}

struct CompactParams {
    PageView t;
    int32_t* moves;
    int32_t* n_moves;
    int32_t* in_use;
    int32_t* went;                       // [pages]: where a page behind the last one in use went (itself: nowhere)
    int32_t* counts;                     // [turns of the pool * CTAs]: pages in use
    int32_t* sums;                       // [2]: pages in use, free places in front of that number
    int most;
    uint32_t* status;
};
template <int kCtas>
__global__ void __launch_bounds__(kPageThreads) page_compact_kernel(const CompactParams p) {
    __shared__ int sums[kPageWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = kCtas > 1 ? int(cluster_cta_rank()) : 0;
    constexpr int kAll = kCtas * kPageThreads;
    const int thread = rank * kPageThreads + int(threadIdx.x);
    const int turns = int((int64_t(p.t.pages) + kAll * 32 - 1) / (kAll * 32));
    uint32_t bits0 = 0;
    int live = 0, passed = 0;
    for (int k = 0; k < turns; ++k) {
        const uint32_t bits = page_bits(p.t, (int64_t(k) * kAll + thread) * 32, true);
        if (k == 0) bits0 = bits;
        int found;
        block_scan(__popc(bits), sums, &found);
        live += found;
        if (kCtas > 1 && threadIdx.x == 0) p.counts[k * kCtas + rank] = found;
    }
    if (kCtas > 1) {
        page_sync<kCtas>();
        live = int(warp_sum(p.counts, turns * kCtas));
    }
    // Pages in use from `live` on, the highest first, and free places in front of it, the lowest first: as many of one as of the
    // other.
    if (live == 0 && thread == 0) p.sums[1] = 0;
    for (int k = 0; k < turns; ++k) {
        const int64_t first = (int64_t(k) * kAll + thread) * 32;
        const uint32_t bits = k == 0 ? bits0 : page_bits(p.t, first, true);
        int all;
        const int before = (kCtas > 1 ? int(warp_sum(p.counts, k * kCtas + rank)) : passed) + block_scan(__popc(bits), sums, &all);
        passed += all;
        const int lane = int(lane_id());
        const int64_t base = first - int64_t(lane) * 32;
        for (int j = 0; j < 32 && base + j * 32 < p.t.pages; ++j) {             // one thread's pages side by side
            const uint32_t word = __shfl_sync(0xffffffffu, bits, j);
            const int in_front = __shfl_sync(0xffffffffu, before, j) + __popc(word & ((1u << lane) - 1u));
            if (base + j * 32 + lane >= p.t.pages) continue;
            const int i = int(base) + j * 32 + lane;
            const int used = int(word >> lane & 1u);
            if (i < live && !used) {
                const int r = i - in_front;
                if (r < p.most) p.moves[int64_t(r) * 3 + 1] = i;
            } else if (i >= live) {
                const int r = live - 1 - in_front;
                if (used && r < p.most) p.moves[int64_t(r) * 3] = i;
                p.went[i] = i;
            }
            if (i == live - 1) p.sums[1] = live - in_front - used;
        }
        __syncwarp();
    }
    page_sync<kCtas>();
    const int moves = min(p.sums[1], p.most);
    for (int r = thread; r < moves; r += kAll) {
        const int a = p.moves[int64_t(r) * 3], b = p.moves[int64_t(r) * 3 + 1];
        p.moves[int64_t(r) * 3 + 2] = 1 << p.t.page_shift;
        p.went[a] = b;
        p.t.holders[b] = p.t.holders[a];
        p.t.holders[a] = 0;
    }
    if (thread == 0) {
        *p.n_moves = moves;
        *p.in_use = live;
        p.sums[0] = live;
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
// Sizes of the lists that reserving and compacting keep per CTA and turn (those of the cluster are the longer ones).
static size_t page_turns(int64_t n, int64_t each) { return up16(size_t(ceil_div(n, kPageThreads * each)) * 4 + kPageCtas * 4); }
static size_t page_workspace(const PageView& t, int forks) {
    const size_t reserve = up16(size_t(t.pages) * sizeof(PageClaim)) + up16(size_t(t.pages) * 4) + page_turns(t.pages, 32) + 2 * page_turns(t.requests, 1);
    const size_t compact = up16(size_t(t.pages) * 4) + page_turns(t.pages, 32) + 16;
    return std::max(std::max(reserve, compact), up16(size_t(forks) * 4));
}

// A kernel that looks through the pool: one CTA up to `of_one` pages, or a cluster.
template <typename P>
static int page_launch(const PageView& t, int of_one, void (*one)(P), void (*cluster)(P), const P& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    const bool single = t.pages <= of_one;
    cfg.gridDim = dim3(single ? 1 : kPageCtas);
    cfg.blockDim = dim3(kPageThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (!single) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = kPageCtas, attr[n].val.clusterDim.y = 1, attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (opt(TL_OPT_PDL) != 0) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = unsigned(n);
    return check_cuda(cudaLaunchKernelEx(&cfg, single ? one : cluster, p));
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
    p.free_list = reinterpret_cast<int32_t*>(at), at += up16(size_t(p.t.pages) * 4);
    p.counts = reinterpret_cast<int32_t*>(at), at += page_turns(p.t.pages, 32);
    p.fresh = reinterpret_cast<int32_t*>(at), at += page_turns(p.t.requests, 1);
    p.copies = reinterpret_cast<int32_t*>(at);
    p.start = d_start;
    p.tokens = d_tokens;
    p.moves = d_moves;
    p.n_moves = d_n_moves;
    p.missing = d_missing;
    p.status = dev().ctl.d_status;
    return page_launch(p.t, kReserveOfOne, page_reserve_kernel<1>, page_reserve_kernel<kPageCtas>, p, stream);
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
    if (int rc = kv_launch(page_fork_kernel, dim3(1), kPageThreads, stream, p)) return rc;
    return kv_launch(page_share_kernel, dim3(unsigned(ceil_div(forks, 8))), 256, stream, p);
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
    p.counts = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + up16(size_t(p.t.pages) * 4));
    p.sums = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(p.counts) + page_turns(p.t.pages, 32));
    p.moves = d_moves;
    p.n_moves = d_n_moves;
    p.in_use = d_in_use;
    p.most = most;
    p.status = dev().ctl.d_status;
    if (int rc = page_launch(p.t, kCompactOfOne, page_compact_kernel<1>, page_compact_kernel<kPageCtas>, p, stream)) return rc;
    if (p.t.requests == 0) return TL_OK;
    return kv_launch(page_rename_kernel, dim3(unsigned(ceil_div(p.t.requests, 8))), 256, stream, p.t, const_cast<const int32_t*>(p.went),
                     const_cast<const int32_t*>(p.sums), p.status);
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
