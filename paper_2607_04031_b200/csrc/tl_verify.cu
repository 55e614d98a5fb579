// Verification of draft trees against the target's distribution (tl_tree_verify).
//
// A thread-block cluster owns one request.  The walk from the root needs, per drafted token, its probability under the
// target and under the drafter, at its parent: they are gathered once, all in parallel, into shared memory, and every
// warp then walks the tree by itself (the same numbers, so the same decisions; nothing has to be broadcast).  Only a
// refused draft, and the draw at the end, need whole rows: then each CTA of the cluster sums its slice of the
// vocabulary, the warps' sums stay in shared memory in the order of the ids, and the slices' sums are exchanged through
// distributed shared memory.  Given those sums, the draw looks for the slice, the warp and the id in turn, re-reading
// one warp's part (about V / 128 values with eight CTAs).  Every sum is fp64 in a fixed order: the answer does not
// depend on timing, and differs from exact arithmetic only when a random number falls within 1e-13 of a boundary.
//
// What bounds it: the bytes of the rows p and q at the node where the walk stops (8 V bytes), and for a single request
// the chain of dependent loads (offsets, parents and tokens, gathered probabilities, row, part of the row).  32 trees of 16
// over 128256 ids: 22 to 24 us (1.4 TB/s of those bytes; issue slots 29 % in use, the rest is waiting along the chain and at the
// cluster's barriers); one chain of 5 over 32000: 9.2 to 10.6 us, a launch and that chain.
#include "tl_kv.cuh"

#include <algorithm>

namespace tl {

constexpr int kVerifyThreads = 512, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyRows = 1024;        // rows of a tree whose gathered numbers are kept in shared memory
constexpr int kVerifyTries = 512;        // children of one node that are tried

struct VerifyParams {
    const float* target;
    const float* draft;
    int64_t target_stride, draft_stride, vocab;
    const int32_t *tokens, *parents, *offsets;
    int requests, rows;
    const float *accept, *sample;
    int32_t *accepted, *n_accepted, *next;
    int64_t accepted_stride;
};

struct VerifySmem {
    double total[2][8];                  // [pass parity][rank]: this CTA's copy of the slices' sums
    double part[kVerifyWarps];           // the warps' sums of the last pass
    double row[32];                      // sums of 32 ids each, when the draw looks for its id
    double mass[kVerifyTries];           // S before each refused draft of the node
    int32_t gone[kVerifyTries];          // their tokens
    int32_t parent[kVerifyRows];
    int32_t token[kVerifyRows];
    float u[kVerifyRows], p[kVerifyRows], q[kVerifyRows];
};

__device__ __forceinline__ double positive(float x) { return double(fmaxf(x, 0.0f)); }       // a NaN counts as zero
__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ void st_cluster_f64(uint32_t cluster_addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(cluster_addr), "d"(v) : "memory");
}

template <bool kDraft>
__global__ void __launch_bounds__(kVerifyThreads, 2) tree_verify_kernel(const VerifyParams p, int cluster) {
    __shared__ VerifySmem sm;
    pdl_wait();
    pdl_launch_dependents();
    const int rank = int(blockIdx.x) % cluster, b = int(blockIdx.x) / cluster;
    const int lane = int(lane_id()), warp = threadIdx.x / 32;
    const int first = min(max(p.offsets[b], 0), p.rows);
    const int n = min(max(p.offsets[b + 1], first), p.rows) - first;
    if (n == 0) {                                            // (the same for the whole cluster)
        if (rank == 0) {
            for (int64_t i = threadIdx.x; i < p.accepted_stride; i += kVerifyThreads) p.accepted[b * p.accepted_stride + i] = -1;
            if (threadIdx.x == 0) {
                p.n_accepted[b] = 0;
                p.next[b] = -1;
            }
        }
        return;
    }
    const float* target = p.target + int64_t(first) * p.target_stride;
    const float* draft = kDraft ? p.draft + int64_t(first) * p.draft_stride : nullptr;

    // a drafted token's probabilities at its parent
    auto gather = [&](int i, int parent, int token, float& pp, float& qq) {
        const bool there = parent >= 0 && parent < i && token >= 0 && token < p.vocab;
        pp = there ? target[int64_t(parent) * p.target_stride + token] : 0.0f;
        qq = there ? (kDraft ? draft[int64_t(parent) * p.draft_stride + token] : 1.0f) : 0.0f;
    };
    const int kept_rows = min(n, kVerifyRows);
    for (int i = threadIdx.x; i < kept_rows; i += kVerifyThreads) {
        const int parent = p.parents[first + i], token = p.tokens[first + i];
        sm.parent[i] = i == 0 ? -1 : parent;
        sm.token[i] = token;
        sm.u[i] = p.accept[first + i];
        gather(i, i == 0 ? -1 : parent, token, sm.p[i], sm.q[i]);
    }
    const float u_sample = p.sample[b];
    // (the cluster's CTAs have all started when this returns: their shared memory may be written to)
    __syncwarp();
    if (cluster > 1) cluster_sync();
    else __syncthreads();

    // (ids fit 32 bits with room for the roundings below: the host bounds the vocabulary)
    const int vocab = int(p.vocab);
    const int slice = ((vocab + cluster - 1) / cluster + 3) / 4 * 4;
    const int s0 = min(rank * slice, vocab), s1 = min(s0 + slice, vocab);
    const int per_warp = ((s1 - s0 + kVerifyWarps - 1) / kVerifyWarps + 31) / 32 * 32;
    const int w0 = min(s0 + warp * per_warp, s1), w1 = min(w0 + per_warp, s1);
    int parity = 0, node = 0, length = 1, tries = 0;

    // the residual at id j of the node's rows, after `tries` refused drafts
    auto value = [&](int j, float pj, float qj) -> double {
        double r = positive(pj);
        if (kDraft) {
            const double q = positive(qj);
            for (int k = 0; k < tries; ++k) r = fmax(r - sm.mass[k] * q, 0.0);
        } else {
            for (int k = 0; k < tries; ++k) r = sm.gone[k] == j ? 0.0 : r;
        }
        return r;
    };
    // the sum of the residual over the vocabulary; leaves the warps' sums and the slices' sums in shared memory
    auto pass = [&]() -> double {
        const float* prow = target + int64_t(node) * p.target_stride;
        const float* qrow = kDraft && tries > 0 ? draft + int64_t(node) * p.draft_stride : nullptr;
        // One term of the sum; the common cases (no refused draft, one, none of this warp's ids refused) have loops of their
        // own: the general one costs several times their instructions, and instructions are what a pass is made of.
        double sum = 0.0;
        auto sweep = [&](auto term) {
            int j0 = w0;
            if (((reinterpret_cast<uintptr_t>(prow) | reinterpret_cast<uintptr_t>(qrow)) & 15u) == 0) {
                constexpr int kUnroll = 2;                   // x 4 ids x 32 lanes (w0 is a multiple of 4)
                for (; j0 + 128 * kUnroll <= w1; j0 += 128 * kUnroll) {
                    float4 pj[kUnroll], qj[kUnroll];
#pragma unroll
                    for (int e = 0; e < kUnroll; ++e) {
                        const int j = j0 + e * 128 + lane * 4;
                        pj[e] = *reinterpret_cast<const float4*>(prow + j);
                        qj[e] = qrow ? *reinterpret_cast<const float4*>(qrow + j) : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int e = 0; e < kUnroll; ++e) {
                        const int j = j0 + e * 128 + lane * 4;
                        sum += (term(j, pj[e].x, qj[e].x) + term(j + 1, pj[e].y, qj[e].y)) + (term(j + 2, pj[e].z, qj[e].z) + term(j + 3, pj[e].w, qj[e].w));
                    }
                }
            }
            constexpr int kUnroll = 8;
            for (; j0 + 32 * kUnroll <= w1; j0 += 32 * kUnroll) {
                float pj[kUnroll], qj[kUnroll];
#pragma unroll
                for (int e = 0; e < kUnroll; ++e) {
                    pj[e] = prow[j0 + e * 32 + lane];
                    qj[e] = qrow ? qrow[j0 + e * 32 + lane] : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < kUnroll; ++e) sum += term(j0 + e * 32 + lane, pj[e], qj[e]);
            }
            for (int j = j0 + lane; j < w1; j += 32) sum += term(j, prow[j], qrow ? qrow[j] : 0.0f);
        };
        int special = 0, gone[4] = {-1, -1, -1, -1};         // refused ids among this warp's
        if (!kDraft)
            for (int k = 0; k < tries; ++k) {
                const int id = sm.gone[k];
                if (id < w0 || id >= w1) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) gone[e] = special == e ? id : gone[e];
                ++special;
            }
        if (kDraft ? tries == 0 : special == 0) sweep([](int, float pj, float) { return positive(pj); });
        else if (kDraft && tries == 1)                       // max(p - q, 0), the mass being 1
            sweep([](int, float pj, float qj) {
                const float pz = fmaxf(pj, 0.0f), qz = fmaxf(qj, 0.0f);
                return pz > qz ? double(pz) - double(qz) : 0.0;
            });
        else if (kDraft && tries <= 3) {                     // max(max(max(p - q, 0) - S1 q, 0) - S2 q, 0)
            const double m1 = sm.mass[1], m2 = tries == 3 ? sm.mass[2] : 0.0;
            sweep([&](int, float pj, float qj) {
                const float pz = fmaxf(pj, 0.0f), qz = fmaxf(qj, 0.0f);
                if (pz <= qz) return 0.0;
                const double q = double(qz), r = double(pz) - q - m1 * q, r2 = r - m2 * q;
                return r2 > 0.0 ? r2 : 0.0;                  // (what falls below 0 once stays there: all that follows is subtracted)
            });
        } else if (!kDraft && special <= 4)
            sweep([&](int j, float pj, float) {
                return positive(j == gone[0] || j == gone[1] || j == gone[2] || j == gone[3] ? 0.0f : pj);
            });
        else sweep(value);
        sum = warp_sum_f64(sum);
        __syncthreads();                                     // the last pass's sums have been read
        if (lane == 0) sm.part[warp] = sum;
        __syncthreads();
        double all = 0.0;
        for (int w = 0; w < kVerifyWarps; ++w) all += sm.part[w];
        parity ^= 1;
        if (cluster == 1) {
            if (threadIdx.x == 0) sm.total[parity][0] = all;
            __syncthreads();
            return all;
        }
        if (int(threadIdx.x) < cluster)
            st_cluster_f64(map_to_cta(smem_u32(&sm.total[parity][rank]), threadIdx.x), all);
        __syncwarp();
        cluster_sync();
        double s = 0.0;
        for (int c = 0; c < cluster; ++c) s += sm.total[parity][c];
        return s;
    };

    double total = 0.0;
    bool have_total = false;
    if (rank == 0 && threadIdx.x == 0) p.accepted[b * p.accepted_stride] = 0;
    while (true) {
        int next = -1;
        double mass = 1.0;
        tries = 0;
        have_total = false;
        bool open = length < p.accepted_stride, empty = false;
        for (int i0 = node + 1; open && next < 0 && i0 < n; i0 += 32) {
            const int i = i0 + lane;
            const int parent = i < n ? (i < kVerifyRows ? sm.parent[i] : p.parents[first + i]) : -1;
            uint32_t children = __ballot_sync(0xffffffffu, parent == node);
            while (children && open) {
                const int c = i0 + __ffs(int(children)) - 1;
                children &= children - 1;
                int token;
                float u, pc, qc;
                if (c < kVerifyRows) {
                    token = sm.token[c], u = sm.u[c], pc = sm.p[c], qc = sm.q[c];
                } else {
                    token = p.tokens[first + c], u = p.accept[first + c];
                    gather(c, node, token, pc, qc);
                }
                const double r = value(token, pc, qc), q = positive(qc);
                if (tries < kVerifyTries && double(u) * q * mass < r) {
                    next = c;
                    break;
                }
                // (what is not tried can neither be kept nor changes the residual)
                if (tries == kVerifyTries) {
                    open = false;
                    break;
                }
                __syncthreads();                             // (all warps take this path together)
                if (threadIdx.x == 0) {
                    sm.mass[tries] = mass;
                    sm.gone[tries] = token;
                }
                __syncthreads();
                ++tries;
                if (kDraft) {
                    mass = pass();
                    total = mass;
                    have_total = true;
                } else {
                    mass -= fmin(r, mass);
                }
                empty = !(mass > 0.0);
                open = !empty;
            }
        }
        if (empty) {                                         // nothing is left of the residual: back to the target's row
            tries = 0;
            have_total = false;
        }
        if (next < 0) break;
        node = next;
        if (rank == 0 && threadIdx.x == 0) p.accepted[b * p.accepted_stride + length] = node;
        ++length;
    }
    // draw from the residual; from the target's row where nothing is left of it
    if (!have_total) total = pass();
    if (!(total > 0.0) && tries > 0) {
        tries = 0;
        total = pass();
    }
    if (rank == 0) {
        for (int64_t i = length + threadIdx.x; i < p.accepted_stride; i += kVerifyThreads) p.accepted[b * p.accepted_stride + i] = -1;
        if (threadIdx.x == 0) {
            p.n_accepted[b] = length;
            if (!(total > 0.0)) p.next[b] = -1;
        }
    }
    if (total > 0.0) {
        const double t = double(u_sample) * total;
        // the slice: the first whose running sum exceeds t, the last that holds anything at most
        int owner = -1;
        double before = 0.0, at = 0.0;
        for (int c = 0; c < cluster; ++c) {
            const double s = sm.total[parity][c];
            if (s > 0.0) {
                owner = c;
                at = before;
                if (before + s > t) break;
            }
            before += s;
        }
        if (owner == rank) {
            int w = -1;
            double run = at, from = at;
            for (int k = 0; k < kVerifyWarps; ++k) {
                const double s = sm.part[k];
                if (s > 0.0) {
                    w = k;
                    from = run;
                    if (run + s > t) break;
                }
                run += s;
            }
            // All warps of the CTA look through warp w's ids, 32 rows of 32 at a time, two rows a warp: the rows' sums to shared
            // memory, one scan over them, and one over the row that holds the answer.  (The values are in the second-level
            // cache by now.)
            const float* prow = target + int64_t(node) * p.target_stride;
            const float* qrow = kDraft && tries > 0 ? draft + int64_t(node) * p.draft_stride : nullptr;
            const int f0 = min(s0 + w * per_warp, s1), f1 = min(f0 + per_warp, s1);
            auto scan = [&](double v) {                      // inclusive running sum over the lanes
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const double up = __shfl_up_sync(0xffffffffu, v, d);
                    if (lane >= d) v += up;
                }
                return v;
            };
            double sum = from, row_from = from;
            int row = -1;                                    // the last row with anything in it, or the one that exceeds t
            for (int j0 = f0; j0 < f1; j0 += 1024) {
                float pj[2], qj[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = j0 + (warp + e * kVerifyWarps) * 32 + lane;
                    pj[e] = j < f1 ? prow[j] : 0.0f;
                    qj[e] = kDraft && qrow && j < f1 ? qrow[j] : 0.0f;
                }
                double v[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) v[e] = warp_sum_f64(value(j0 + (warp + e * kVerifyWarps) * 32 + lane, pj[e], qj[e]));
                __syncthreads();                             // the last rows' sums have been read
                if (lane == 0) {
                    sm.row[warp] = v[0];
                    sm.row[warp + kVerifyWarps] = v[1];
                }
                __syncthreads();
                const double mine = sm.row[lane], to = scan(mine);
                const uint32_t some = __ballot_sync(0xffffffffu, mine > 0.0), over = __ballot_sync(0xffffffffu, sum + to > t && mine > 0.0);
                if (some) {
                    const int k = over ? __ffs(int(over)) - 1 : 31 - __clz(int(some));
                    row = j0 + k * 32;
                    row_from = sum + __shfl_sync(0xffffffffu, to - mine, k);
                }
                if (over) break;
                sum += __shfl_sync(0xffffffffu, to, 31);
            }
            if (warp == 0) {
                int found = -1;
                if (row >= 0) {
                    const int j = row + lane;
                    const double r = j < f1 ? value(j, prow[j], kDraft && qrow ? qrow[j] : 0.0f) : 0.0, to = scan(r);
                    const uint32_t hit = __ballot_sync(0xffffffffu, row_from + to > t && r > 0.0), any = __ballot_sync(0xffffffffu, r > 0.0);
                    found = row + (hit ? __ffs(int(hit)) - 1 : 31 - __clz(int(any | 1u)));
                }
                if (lane == 0) p.next[b] = found;
            }
        }
    }
    __syncwarp();
    if (cluster > 1) cluster_sync();                         // no CTA leaves while another may still write to it
}

}  // namespace tl

extern "C" {

int tl_tree_verify(const float* d_target, int64_t target_stride, const float* d_draft, int64_t draft_stride, int64_t vocab,
                   const int32_t* d_tokens, const int32_t* d_parents, const int32_t* d_token_offsets, int requests,
                   int tokens, const float* d_accept, const float* d_sample, int32_t* d_accepted,
                   int64_t accepted_stride, int32_t* d_n_accepted, int32_t* d_next, void* cuda_stream) {
    using namespace tl;
    if (requests < 0 || tokens < 0 || vocab < 1 || vocab > (1 << 30) || accepted_stride < 1) return TL_ERR_INVALID_ARG;
    if (requests == 0) return TL_OK;
    if (!d_token_offsets || !d_accepted || !d_n_accepted || !d_next || !d_sample) return TL_ERR_INVALID_ARG;
    if (tokens > 0 && (!d_target || !d_tokens || !d_parents || !d_accept)) return TL_ERR_INVALID_ARG;
    if (target_stride < vocab || (d_draft && draft_stride < vocab)) return TL_ERR_INVALID_ARG;
    if (!words_aligned(d_target, d_draft, d_tokens, d_parents, d_token_offsets, d_accept, d_sample, d_accepted, d_n_accepted, d_next))
        return TL_ERR_ALIGNMENT;
    if (opt(TL_OPT_PLAN_AS_IF_SMS)) return TL_ERR_INVALID_ARG;
    ApiLock lock;
    if (int rc = ensure_device_info()) return rc;
    VerifyParams p = {};
    p.target = d_target;
    p.draft = d_draft;
    p.target_stride = target_stride;
    p.draft_stride = draft_stride;
    p.vocab = vocab;
    p.tokens = d_tokens;
    p.parents = d_parents;
    p.offsets = d_token_offsets;
    p.requests = requests;
    p.rows = tokens;
    p.accept = d_accept;
    p.sample = d_sample;
    p.accepted = d_accepted;
    p.n_accepted = d_n_accepted;
    p.next = d_next;
    p.accepted_stride = accepted_stride;
    // As many CTAs per request as leave every request resident, at most the eight of a portable cluster, and at least
    // 2048 ids per CTA.  Trees of 8, us with 1 / 2 / 4 / 8 CTAs a request: 1 request over 128256 ids 59 / 39 / 29 / 23, over
    // 2048 14 / 16 / 16 / 16; 32 over 128256 64 / 41 / 31 / 25; 100 over 32000 29 / 25 / 31 / 43; 200 over 8192 18 / 27 / 37 / 70.
    int cluster = 8;
    while (cluster > 1 && (int64_t(requests) * cluster > dev().sm_count * 2 || vocab / cluster < 2048)) cluster /= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(requests) * unsigned(cluster));
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = static_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (opt(TL_OPT_PDL) != 0) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = unsigned(cluster);
        attr[n].val.clusterDim.y = 1;
        attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = unsigned(n);
    return check_cuda(d_draft ? cudaLaunchKernelEx(&cfg, tree_verify_kernel<true>, p, cluster)
                              : cudaLaunchKernelEx(&cfg, tree_verify_kernel<false>, p, cluster));
}

}  // extern "C"
