// What the kernels of the paged key-value cache share (contracts in include/kl.h): the cache and the rows of a call as they see
// them, page look-ups, e4m3 scales and conversions, prefix sums over sequences.
#pragma once

#include "kl_device.cuh"

#include <cuda_fp16.h>

#include <type_traits>

namespace kl {

// A cache and the sequences that live in it, as the kernels see them (strides in bytes).
struct PagedView {
    uint8_t *k, *v;
    uint8_t *ke, *ve;          // e4m3: scale exponents [n_pages][nkv][page]
    __nv_bfloat16* bounds;     // [n_pages][nkv][2][hd] or null
    int64_t page_b, head_b, row_b;
    uint32_t nkv, hd, page, n_pages, fp8;
    const int32_t* positions;
    const int32_t* table;
    int64_t table_stride;
    uint32_t table_pages, n_seqs;
    int32_t* status;           // or null
};

__device__ __forceinline__ void pg_error(const PagedView& c) {
    if (c.status) atomicCAS(c.status, 0, ERR_OUT_OF_RANGE);
}
// Whether an earlier call has set the status word; the same answer for every thread of the block, although another
// block may be setting the word right now.
__device__ __forceinline__ bool pg_stopped(const PagedView& c) {
    return c.status && __syncthreads_or(*(volatile int32_t*)c.status != 0);
}

// Physical page behind logical page `lp` of sequence s, or -1 (and the status word set) when there is none.
__device__ __forceinline__ int32_t pg_physical(const PagedView& c, uint32_t s, uint32_t lp) {
    if (lp < c.table_pages) {
        const int32_t p = c.table[(int64_t)s * c.table_stride + lp];
        if ((uint32_t)p < c.n_pages) return p;
    }
    pg_error(c);
    return -1;
}

// Positions sequence s holds (0 for an empty slot); a position behind the page table sets the status word and is cut off.
__device__ __forceinline__ uint32_t pg_length(const PagedView& c, uint32_t s) {
    const int32_t pos = c.positions[s];
    if (pos < 0) return 0u;
    const uint32_t most = c.table_pages * c.page;
    if ((uint32_t)pos >= most) {
        pg_error(c);
        return most;
    }
    return (uint32_t)pos + 1u;
}

// 64-bit division that is usually a 32-bit one (a 64-bit division is a few hundred cycles of a kernel that may last 5 us).
__device__ __forceinline__ uint64_t pg_div(uint64_t x, uint32_t y) { return (x >> 32) == 0u ? (uint64_t)((uint32_t)x / y) : x / y; }

// 2^(e - 127) of a scale byte, and its inverse for the bytes a row can have (up to 247).
__device__ __forceinline__ float pg_scale(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x00400000u); }
__device__ __forceinline__ float pg_inv_scale(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// Scale byte of a row whose largest finite magnitude has the bits `big`: e + 127 with the smallest e >= -127 with
// magnitude <= 448 * 2^e.  m * 2^k with m in [1, 2): 448 = 1.75 * 2^8, so e = k - 8, or k - 7 where m > 1.75 (the 23 fraction
// bits of 1.75 are 0x600000: adding 0x1fffff to larger ones carries into the exponent).  Numbers below 2^-119 all get -127.
__device__ __forceinline__ uint32_t pg_exponent(uint32_t big) { return (uint32_t)max((int32_t)((big + 0x1fffffu) >> 23) - 8, 0); }

// Four floats to four e4m3 codes (x0 in the low byte), nearest even, saturating.
__device__ __forceinline__ uint32_t pg_to_e4m3x4(float x0, float x1, float x2, float x3) {
    uint32_t r;
    asm("{.reg .b16 a, b; cvt.rn.satfinite.e4m3x2.f32 a, %2, %1; cvt.rn.satfinite.e4m3x2.f32 b, %4, %3; mov.b32 %0, {a, b};}"
        : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    return r;
}
// Two e4m3 codes (low 16 bits) to two halves, exact.
__device__ __forceinline__ uint32_t pg_e4m3x2_to_f16x2(uint32_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}
__device__ __forceinline__ float2 pg_f16x2_to_float2(uint32_t h) {
    const __half2 v = *reinterpret_cast<const __half2*>(&h);
    return __half22float2(v);
}

// Two bf16 at a time: the number of the larger magnitude (its sign means nothing), product, smaller and larger one.  NaN is
// left out where the other number is none.
__device__ __forceinline__ uint32_t pg_larger(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pg_mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pg_min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pg_max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The smallest and the largest of three floats; NaN is left out.
__device__ __forceinline__ float pg_min3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float pg_max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Eight consecutive elements to dst (16-byte aligned).
template <class T>
__device__ __forceinline__ void pg_store8(T* dst, const float (&x)[8]);
template <>
__device__ __forceinline__ void pg_store8<float>(float* dst, const float (&x)[8]) {
    reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <>
__device__ __forceinline__ void pg_store8<__nv_bfloat16>(__nv_bfloat16* dst, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
// Prefix sums of count(s) over the n sequences, for a block of NW warps: pre[t] = sum over the sequences before thread t's
// share (per = ceil(n / threads) sequences each); returns the sum over all of them.
template <int NW, class Count>
__device__ __forceinline__ uint64_t pg_prefix(uint32_t n, uint64_t* pre, uint64_t* wsum, Count&& count) {
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, per = (n + NW * 32u - 1u) / (NW * 32u);
    uint64_t mine = 0;
    for (uint32_t s = tid * per; s < min(n, (tid + 1u) * per); ++s) mine += count(s);
    uint64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31u) wsum[warp] = incl;
    __syncthreads();
    uint64_t all = 0, before = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < (int)warp) before += wsum[w];
        all += wsum[w];
    }
    pre[tid] = before + incl - mine;
    __syncthreads();
    return all;
}
// The largest t with pre[t] <= x (pre[0] = 0): which of 32 groups of NW entries, then which entry.  Whole warps.
template <int NW>
__device__ __forceinline__ uint32_t pg_find(const uint64_t* pre, uint64_t x) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t i = (__popc(__ballot_sync(0xffffffffu, pre[lane * NW] <= x)) - 1) * NW;
    return i + __popc(__ballot_sync(0xffffffffu, lane < (uint32_t)NW && pre[i + lane % NW] <= x)) - 1;
}

// The rows a call brings, and where they lie.
struct PagedRows {
    const int32_t* row_starts;   // [n_seqs + 1], or null: row s belongs to sequence s
    uint32_t n_rows;
    uint8_t *k, *v;
    int64_t k_stride, v_stride;  // bytes
};

__device__ __forceinline__ uint32_t pg_row_start(const PagedView& c, const PagedRows& r, uint32_t s) {   // s in [0, n_seqs]
    if (!r.row_starts) return min(s, r.n_rows);
    const int32_t x = r.row_starts[s];
    return x < 0 ? 0u : min((uint32_t)x, r.n_rows);
}

// An array of row starts that descends or leaves [0, n_rows] is an error (one block of a call looks).
__device__ __forceinline__ void pg_check_starts(const PagedView& c, const PagedRows& r) {
    for (uint32_t s = threadIdx.x; s < c.n_seqs; s += blockDim.x) {
        const int32_t a = r.row_starts[s], b = r.row_starts[s + 1u];
        if (a < 0 || b < a || (uint32_t)b > r.n_rows) pg_error(c);
    }
}

}  // namespace kl
