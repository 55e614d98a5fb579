// Shared by the kernels around the paged key/value cache: device views of tl_kv_cache / tl_kv_batch, the addressing,
// and the conversions between stored codes and the operands of the matrix instructions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tl_common.cuh"

namespace tl {

enum : uint32_t {
    kBadPage = 0xA00,           // a page-table entry outside the cache, or a position past the table's last page
    kBadAccepted = 0xB00        // tl_kv_commit: an accepted index outside the request's tokens
};

// tl_kv_cache as the kernels use it: strides in bytes, page size as a shift.
struct KvView {
    char* base[2];              // keys, values
    float* scale[2];
    int64_t page_stride, head_stride, token_stride;     // bytes
    int64_t scale_page_stride, scale_head_stride;       // floats
    int64_t pages;
    int heads, page_shift;
};
struct KvBatchView {
    const int32_t* page_table;
    const int32_t* start;
    const int32_t* offsets;
    int64_t table_stride;
    int requests, tokens;
};

constexpr int64_t kKvMaxTokens = int64_t(1) << 30;         // of one sequence

// Checks a cache / batch description and turns it into the view (host).
int kv_view(const tl_kv_cache* c, KvView* out);
int kv_batch_view(const tl_kv_batch* b, KvBatchView* out);

// Whether each of the arrays (NULL ones aside) starts on a boundary of its 4-byte elements.
template <typename... P>
inline bool words_aligned(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 3u) == 0; }

inline int kv_item(int format) { return format == TL_KV_BF16 ? 2 : 1; }

#ifdef __CUDACC__

// One request of a batch.  Whatever the offsets on the device hold, the rows stay inside [0, tokens) and the length
// inside what the page table can address.
struct KvRequest {
    int first, n;               // its rows
    int start;                  // tokens in the cache before the step's
    int len;                    // positions that exist: start + n, as far as the page table reaches
};
// Positions the page table of a request can address (at most 2^30: a position fits 32 bits with room to spare).
__device__ __forceinline__ int kv_room(const KvBatchView& bv, int page_shift) {
    return int(min(bv.table_stride << page_shift, int64_t(1) << 30));
}
__device__ __forceinline__ KvRequest kv_request(const KvBatchView& bv, int page_shift, int b) {
    KvRequest r;
    int a = bv.offsets[b], e = bv.offsets[b + 1];
    a = min(max(a, 0), bv.tokens);
    e = min(max(e, a), bv.tokens);
    const int room = kv_room(bv, page_shift);
    r.first = a;
    r.n = e - a;
    r.start = min(max(bv.start[b], 0), room);
    r.len = r.n < room - r.start ? r.start + r.n : room;
    return r;
}

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 31u; }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_8(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

// Two codes (the low 16 bits of x) to two f16 values, both formats exactly: every E4M3 value and every integer up to
// 2048 is an f16 value.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t x) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t x) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(x));
    return r;
}
// Signed bytes: 0x6400 is 1024 in f16, whose last mantissa bit is worth 1, so 0x64 in front of (byte ^ 0x80) reads
// 1024 + 128 + value; the subtraction is exact.
__device__ __forceinline__ uint32_t s8x2_from_biased(uint32_t pair_with_64) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(pair_with_64), "r"(0x64806480u));
    return r;
}
// Four codes of one 32-bit word to two f16x2 registers.
template <int kFmt>
__device__ __forceinline__ void codes4_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if (kFmt == TL_KV_E4M3) {
        lo = e4m3x2_to_f16x2(w);
        hi = e4m3x2_hi_to_f16x2(w);
    } else {
        w ^= 0x80808080u;
        lo = s8x2_from_biased(__byte_perm(w, 0x64646464u, 0x4140));
        hi = s8x2_from_biased(__byte_perm(w, 0x64646464u, 0x4342));
    }
}

// Which bytes hold an E4M3 NaN (0x7f, 0xff): their top bits, and whole bytes.  tl_kv_append writes none: they stand in memory that
// nobody wrote.
__device__ __forceinline__ uint32_t e4m3_nan_bits(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t e4m3_nan_bytes(uint32_t x) { return (e4m3_nan_bits(x) >> 7) * 0xffu; }

// D (fp32 16 x 8) += A (16 x 16) B (16 x 8), operands f16 or bf16.
template <bool kBf16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

#endif  // __CUDACC__

}  // namespace tl
