// Kernels of the paged key-value cache (contracts in include/kl.h): append with quantisation and page bounds, read back,
// page selection by bounds, attention of one new token over pages.
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

// ---- rows in and out

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

constexpr int PG_THREADS = 256;

// An array of row starts that descends or leaves [0, n_rows] is an error (one block of a call looks).
__device__ __forceinline__ void pg_check_starts(const PagedView& c, const PagedRows& r) {
    for (uint32_t s = threadIdx.x; s < c.n_seqs; s += blockDim.x) {
        const int32_t a = r.row_starts[s], b = r.row_starts[s + 1u];
        if (a < 0 || b < a || (uint32_t)b > r.n_rows) pg_error(c);
    }
}

// Append.  One block = the rows of one call that fall into one page, for one kv head, so that the page's bounds have one
// writer and its rows are quantised where they pass by.  Sequence s touches at most rows / page + 2 pages, so block u of
// the grid belongs to the sequence s with base(s) <= u < base(s + 1), base(s) = row_starts[s] / page + 2 s, and is its
// page number u - base(s) (blocks without a page leave).  hd / 8 lanes share a row, eight columns each; half of the
// lane groups take keys, the other half values.
// Per row and head: largest magnitude over the lanes (as whole numbers: the bits of a float; of bf16 rows two at a time in one
// word), the exponent from its bits, one multiplication by a power of two per element (exact), rounding by the conversion
// instruction.
// Measured, 8 kv heads of 128: one bf16 row 2.1 us (launch and a chain of three loads); 8191 bf16 rows to e4m3 12.7 us, 61 % of
// the copy rate.  What bounds it is instructions (some 96 per eight elements on average, half of the time) and a block's chain
// of sequence, page and rows; two rows at a time, bf16 pairs and 32-bit strides took it there from 16.3 us.  Rows requested
// asynchronously through shared memory: 12.1 us at best, not kept for that.  8191 fp32 rows to e4m3 18.2 us (72 %), bf16 rows to a
// bf16 cache 14.8 (70 %), fp32 rows to a bf16 cache 19.0 (82 %).
constexpr int PW_THREADS = 128;   // (before the steps above: 16.3 us; 256 threads 17.6, 64 threads 25.0)
template <class T, int HD, bool FP8>
__global__ void __launch_bounds__(PW_THREADS, 1024 / PW_THREADS) kl_paged_append_kernel(const PagedView c, const PagedRows rows) {
    extern __shared__ float pg_red[];   // [groups of K rows][2][hd] when the cache has bounds
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t u = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    uint32_t s = u, j = 0, r0 = u, r1 = u + 1u;
    int32_t pos;
    if (rows.row_starts) {
        // the last s with base(s) <= u, and its position: all candidates are loaded at once (a search would be a chain of loads)
        __shared__ uint32_t found[5];
        if (u == 0u && h == 0u) pg_check_starts(c, rows);
        if (tid == 0u) found[0] = 0u;
        __syncthreads();
        uint32_t best = 0, b0 = 0, b1 = 0;
        int32_t bp = 0;
        for (uint32_t t = tid; t < c.n_seqs; t += PW_THREADS) {
            const uint32_t x = pg_row_start(c, rows, t), y = pg_row_start(c, rows, t + 1u);
            const int32_t p = c.positions[t];
            if (x / c.page + 2u * t <= u) {
                best = t + 1u;
                b0 = x; b1 = y; bp = p;
            }
        }
        const uint32_t wbest = __reduce_max_sync(0xffffffffu, best);
        if ((tid & 31u) == 0u && wbest) atomicMax(&found[0], wbest);
        __syncthreads();
        if (found[0] == 0u) return;   // base(0) = row_starts[0] / page may lie above u
        if (best == found[0]) {
            found[1] = b0; found[2] = b1; found[3] = (uint32_t)bp;
        }
        __syncthreads();
        s = found[0] - 1u;
        r0 = found[1]; r1 = found[2]; pos = (int32_t)found[3];
        j = u - (r0 / c.page + 2u * s);
    } else {
        pos = c.positions[s];
    }
    if (pos < 0 || r1 <= r0) return;
    const uint64_t n = r1 - r0, p0 = (uint64_t)pos, p1 = p0 + n;            // positions [p0, p1)
    const uint64_t lp = (uint64_t)((uint32_t)pos / c.page) + j, a0 = max(p0, lp * c.page), a1 = min(p1, (lp + 1u) * c.page);
    if (a0 >= a1) return;
    if (lp >= c.table_pages) {
        if (tid == 0u) pg_error(c);
        return;
    }
    const int32_t phys = pg_physical(c, s, (uint32_t)lp);
    if (phys < 0) return;

    constexpr uint32_t LANES = HD / 8, GROUPS = PW_THREADS / LANES / 2;   // lanes per row, rows at a time per side (K, V)
    const uint32_t grp = tid / LANES, lane = tid % LANES, col = lane * 8u;
    const bool is_v = grp >= GROUPS;   // the same for a whole warp
    const uint32_t g = is_v ? grp - GROUPS : grp;
    const uint32_t off0 = (uint32_t)(a0 - lp * c.page), cnt = (uint32_t)(a1 - a0), row0 = r0 + (uint32_t)(a0 - p0);
    const uint32_t src_stride = (uint32_t)(is_v ? rows.v_stride : rows.k_stride), dst_stride = (uint32_t)c.row_b;   // at most 2^31
    const uint8_t* src = (is_v ? rows.v : rows.k) + (uint64_t)row0 * src_stride + ((size_t)h * HD + col) * sizeof(T);
    uint8_t* dst = (is_v ? c.v : c.k) + (int64_t)phys * c.page_b + (int64_t)h * c.head_b + (int64_t)off0 * c.row_b + col * (FP8 ? 1 : 2);
    uint8_t* exps = FP8 ? (is_v ? c.ve : c.ke) + ((int64_t)phys * c.nkv + h) * c.page + off0 : nullptr;
    // the page's bounds so far, requested ahead of the rows: thread t looks after columns t, t + PW_THREADS, ... of [lo | hi]
    __nv_bfloat16* bounds = c.bounds ? c.bounds + ((int64_t)phys * c.nkv + h) * 2 * HD : nullptr;
    const bool bounded = bounds && !is_v;
    constexpr int COLS = 2 * HD / PW_THREADS;
    static_assert(COLS * PW_THREADS == 2 * HD, "columns");
    float old[COLS];
    if (bounds)
#pragma unroll
        for (int i = 0; i < COLS; ++i) {
            const uint32_t t = tid + i * PW_THREADS;
            old[i] = off0 == 0u ? (t >= (uint32_t)HD ? -INFINITY : INFINITY) : __bfloat162float(bounds[t]);
        }
    // bounds of the rows seen: eight columns in 32 bits (e4m3), or two in one word as the cache holds them (bf16)
    float lo[FP8 ? 8 : 1], hi[FP8 ? 8 : 1];
    uint32_t lo2[FP8 ? 1 : 4], hi2[FP8 ? 1 : 4];
#pragma unroll
    for (int i = 0; i < (FP8 ? 8 : 1); ++i) {
        lo[i] = INFINITY;
        hi[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < (FP8 ? 1 : 4); ++i) {
        lo2[i] = 0x7f807f80u;
        hi2[i] = 0xff80ff80u;
    }
    constexpr int U = sizeof(T) == 2 ? 4 : 2;   // rows a lane has in flight (bf16: two 14.3 us, eight 13.1)
    for (uint32_t i0 = 0; i0 < cnt; i0 += GROUPS * U) {   // every lane of a warp takes part in the shuffles
        uint4 raw[U][sizeof(T) / 2];
#pragma unroll
        for (int y = 0; y < U; ++y) {
            const uint32_t i = min(i0 + y * GROUPS + g, cnt - 1u);   // past the end the last row again, which changes no maximum
#pragma unroll
            for (int q = 0; q < (int)sizeof(T) / 2; ++q) raw[y][q] = reinterpret_cast<const uint4*>(src + (uint64_t)i * src_stride)[q];
        }
#pragma unroll
        for (int y = 0; y < U; y += 2) {   // two rows at a time
            if (i0 + y * GROUPS >= cnt) break;   // the same for the whole block
            const uint32_t i[2] = {i0 + y * GROUPS + g, i0 + (y + 1) * GROUPS + g};
            uint32_t w[2][8];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint4 p = raw[y + r][0], p2 = raw[y + r][sizeof(T) / 2 - 1];
                w[r][0] = p.x; w[r][1] = p.y; w[r][2] = p.z; w[r][3] = p.w;
                w[r][4] = p2.x; w[r][5] = p2.y; w[r][6] = p2.z; w[r][7] = p2.w;
            }
            auto element = [&](int r, int q) { return sizeof(T) == 4 ? __uint_as_float(w[r][q]) : q & 1 ? bf_hi(w[r][q / 2]) : bf_lo(w[r][q / 2]); };
            if constexpr (FP8) {
                uint32_t big[2];   // largest magnitudes, as their bits; infinities and NaN do not count
                auto finite = [&](int r) {   // (asked for by whole warps: a branch, not instructions that are skipped one by one)
                    uint32_t b = 0u;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const uint32_t u = __float_as_uint(element(r, q)) & 0x7fffffffu;
                        if (u < 0x7f800000u) b = max(b, u);
                    }
                    return b;
                };
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        big[r] = 0u;
#pragma unroll
                        for (int q = 0; q < 8; ++q) big[r] = max(big[r], w[r][q] & 0x7fffffffu);
                        if (__any_sync(0xffffffffu, big[r] >= 0x7f800000u)) big[r] = finite(r);
#pragma unroll
                        for (uint32_t o = LANES / 2u; o > 0u; o >>= 1) big[r] = max(big[r], __shfl_xor_sync(0xffffffffu, big[r], o));
                    }
                } else {   // both rows in one word: the first in its low half
                    const uint32_t a = pg_larger(pg_larger(w[0][0], w[0][1]), pg_larger(w[0][2], w[0][3]));
                    const uint32_t b = pg_larger(pg_larger(w[1][0], w[1][1]), pg_larger(w[1][2], w[1][3]));
                    uint32_t m = pg_larger(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632)) & 0x7fff7fffu;
                    if (__any_sync(0xffffffffu, (m + 0x00800080u) & 0x80008000u)) m = finite(0) >> 16 | (finite(1) & 0xffff0000u);
#pragma unroll
                    for (uint32_t o = LANES / 2u; o > 0u; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                    big[0] = m << 16;
                    big[1] = m & 0xffff0000u;
                }
                uint32_t code[2][2];
                float scale[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t e = pg_exponent(big[r]);
                    float x[8];
                    if constexpr (sizeof(T) == 2) {   // products by a power of two: exact, or so small that the code is zero
                        const uint32_t inv = (254u - e) * 0x00800080u;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t t = pg_mul_bf16x2(w[r][q], inv);
                            x[2 * q] = bf_lo(t);
                            x[2 * q + 1] = bf_hi(t);
                        }
                    } else {
                        const float inv = pg_inv_scale(e);
#pragma unroll
                        for (int q = 0; q < 8; ++q) x[q] = element(r, q) * inv;
                    }
                    code[r][0] = pg_to_e4m3x4(x[0], x[1], x[2], x[3]);
                    code[r][1] = pg_to_e4m3x4(x[4], x[5], x[6], x[7]);
                    scale[r] = pg_scale(e);
                    if (i[r] < cnt) {
                        *reinterpret_cast<uint2*>(dst + (uint64_t)i[r] * dst_stride) = make_uint2(code[r][0], code[r][1]);
                        if (lane == 0u) exps[i[r]] = (uint8_t)e;
                    }
                }
                if (bounded) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t shift = 16 * (q & 1);
                        const float2 f = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(code[0][q / 2] >> shift & 0xffffu));
                        const float2 h = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(code[1][q / 2] >> shift & 0xffffu));
                        const float x0 = f.x * scale[0], x1 = f.y * scale[0], y0 = h.x * scale[1], y1 = h.y * scale[1];
                        lo[2 * q] = pg_min3(lo[2 * q], x0, y0);
                        hi[2 * q] = pg_max3(hi[2 * q], x0, y0);
                        lo[2 * q + 1] = pg_min3(lo[2 * q + 1], x1, y1);
                        hi[2 * q + 1] = pg_max3(hi[2 * q + 1], x1, y1);
                    }
                }
            } else {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    uint32_t v[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = sizeof(T) == 4 ? pack_bf16(element(r, 2 * q), element(r, 2 * q + 1)) : w[r][q];
                    if (i[r] < cnt) *reinterpret_cast<uint4*>(dst + (uint64_t)i[r] * dst_stride) = make_uint4(v[0], v[1], v[2], v[3]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        lo2[q] = pg_min_bf16x2(lo2[q], v[q]);
                        hi2[q] = pg_max_bf16x2(hi2[q], v[q]);
                    }
                }
            }
        }
    }
    if (!bounds) return;
    if (!is_v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float* to = pg_red + g * 2u * HD + col + 2 * q;
            *reinterpret_cast<float2*>(to) = FP8 ? make_float2(lo[FP8 ? 2 * q : 0], lo[FP8 ? 2 * q + 1 : 0]) : make_float2(bf_lo(lo2[FP8 ? 0 : q]), bf_hi(lo2[FP8 ? 0 : q]));
            *reinterpret_cast<float2*>(to + HD) = FP8 ? make_float2(hi[FP8 ? 2 * q : 0], hi[FP8 ? 2 * q + 1 : 0]) : make_float2(bf_lo(hi2[FP8 ? 0 : q]), bf_hi(hi2[FP8 ? 0 : q]));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
        const uint32_t t = tid + i * PW_THREADS;
        const bool up = t >= (uint32_t)HD;
        float x = old[i];
#pragma unroll
        for (uint32_t k = 0; k < GROUPS; ++k) {
            const float y = pg_red[k * 2u * HD + t];
            x = up ? fmaxf(x, y) : fminf(x, y);
        }
        bounds[t] = up ? __float2bfloat16_ru(x) : __float2bfloat16_rd(x);   // exact but for e4m3 rows of scale bytes 0 .. 2
    }
}

// Sequence a row belongs to: the largest s with row_starts[s] <= row (the last of several that start there).  `starts`:
// the array in shared memory, or null.
__device__ __forceinline__ uint32_t pg_seq_of_row(const PagedView& c, const PagedRows& r, const uint32_t* starts, uint32_t row) {
    if (!r.row_starts) return row;
    uint32_t lo = 0, hi = c.n_seqs;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) / 2u;
        if ((starts ? starts[mid] : pg_row_start(c, r, mid)) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Read back.  A block walks over chunks of R rows (as many as make PR_ITEMS 16-byte pieces).  R threads look up where the rows
// of the next chunk lie -- a chain of dependent loads: sequence, position, page -- while the block copies this chunk's.  hd / 8
// lanes share a (row, head, K or V), eight columns each: 16 bytes of a bf16 output, so that a warp's stores are contiguous
// (16 columns of an e4m3 row per lane, 16-byte loads but 32-byte strides between the stores: 88 instead of 79 us).
// Measured: 65537 e4m3 rows of 8 x 128 to bf16, 404 MB in all, 78.5 us, 80 % of the copy rate (to fp32 144 us, 72 %); 4096 bf16 rows
// 10.0 us (to fp32 20.6).
constexpr int PR_UNROLL = 4;   // pieces a lane has in flight (eight: no faster for e4m3, 13.2 instead of 9.9 us for 4096 bf16 rows)
constexpr uint32_t PR_ITEMS = 4096;
constexpr uint32_t PR_STARTS = 512;   // sequences whose first rows are kept in shared memory
__host__ __device__ constexpr uint32_t pr_rows(uint32_t nkv, uint32_t lanes) {   // rows of a chunk
    return 2u * nkv * lanes >= PR_ITEMS ? 1u : PR_ITEMS / (2u * nkv * lanes) < (uint32_t)PG_THREADS ? PR_ITEMS / (2u * nkv * lanes) : (uint32_t)PG_THREADS;
}
template <class T, int HD, bool FP8>
__global__ void __launch_bounds__(PG_THREADS, 4) kl_paged_read_kernel(const PagedView c, const PagedRows rows) {
    constexpr uint32_t E = 8, LANES = HD / E, GROUPS = PG_THREADS / LANES;
    using Piece = typename std::conditional<FP8, uint2, uint4>::type;   // a lane's columns in the cache
    __shared__ uint32_t starts_s[PR_STARTS + 1];
    __shared__ int64_t at_s[2][PG_THREADS], exp_s[2][PG_THREADS];   // offsets of a chunk's rows (head 0), -1: nothing to copy
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t tid = threadIdx.x, grp = tid / LANES, col = tid % LANES * E;
    const uint32_t R = pr_rows(c.nkv, LANES), per_row = 2u * c.nkv, di = GROUPS % per_row, dr = GROUPS / per_row;
    if (rows.row_starts && blockIdx.x == 0u) pg_check_starts(c, rows);
    const bool kept = rows.row_starts && c.n_seqs <= PR_STARTS;
    if (kept) {
        for (uint32_t s = tid; s <= c.n_seqs; s += PG_THREADS) starts_s[s] = pg_row_start(c, rows, s);
        __syncthreads();
    }
    const uint32_t* starts = kept ? starts_s : nullptr;
    auto look_up = [&](uint64_t row0, int64_t& at, int64_t& ex) {   // row row0 + tid
        at = ex = -1;
        const uint64_t row64 = row0 + tid;
        if (tid >= R || row64 >= rows.n_rows) return;
        const uint32_t row = (uint32_t)row64, s = pg_seq_of_row(c, rows, starts, row);
        const uint32_t r0 = starts ? starts[s] : pg_row_start(c, rows, s), r1 = starts ? starts[s + 1u] : pg_row_start(c, rows, s + 1u);
        const int32_t pos = c.positions[s];
        if (pos < 0 || row < r0 || row >= r1) return;
        const uint64_t p = (uint64_t)pos + (row - r0), lp = pg_div(p, c.page);
        const int32_t phys = lp < c.table_pages ? pg_physical(c, s, (uint32_t)lp) : -1;
        if (phys < 0) {
            pg_error(c);
            return;
        }
        const uint32_t off = (uint32_t)(p - lp * c.page);
        at = (int64_t)phys * c.page_b + (int64_t)off * c.row_b;
        ex = (int64_t)phys * c.nkv * c.page + off;
    };
    const uint32_t head_b = (uint32_t)c.head_b, k_stride = (uint32_t)rows.k_stride, v_stride = (uint32_t)rows.v_stride;   // at most 2^31
    const uint64_t step = (uint64_t)gridDim.x * R;
    uint64_t row0 = (uint64_t)blockIdx.x * R;
    int64_t at, ex;
    look_up(row0, at, ex);
    for (int buf = 0; row0 < rows.n_rows; row0 += step, buf ^= 1) {
        at_s[buf][tid] = at;
        exp_s[buf][tid] = ex;
        __syncthreads();   // (the buffer's previous contents were read before the barrier of the round between)
        look_up(row0 + step, at, ex);
        uint32_t r = grp / per_row, i = grp - r * per_row;   // row of the chunk, head (values: nkv + head)
        while (r < R) {
            Piece x[PR_UNROLL];
            uint32_t e[PR_UNROLL], to_r[PR_UNROLL], to_i[PR_UNROLL];
#pragma unroll
            for (int u = 0; u < PR_UNROLL; ++u) {
                const int64_t from = r < R ? at_s[buf][r] : -1;
                to_r[u] = from >= 0 ? r : 0xffffffffu;
                to_i[u] = i;
                if (from >= 0) {
                    const bool is_v = i >= c.nkv;
                    const uint32_t h = is_v ? i - c.nkv : i;
                    x[u] = *reinterpret_cast<const Piece*>((is_v ? c.v : c.k) + from + (uint64_t)h * head_b + col * (FP8 ? 1 : 2));
                    if (FP8) e[u] = (is_v ? c.ve : c.ke)[exp_s[buf][r] + h * c.page];
                }
                i += di;
                r += dr;
                if (i >= per_row) {
                    i -= per_row;
                    ++r;
                }
            }
#pragma unroll
            for (int u = 0; u < PR_UNROLL; ++u)
                if (to_r[u] != 0xffffffffu) {
                    const bool is_v = to_i[u] >= c.nkv;
                    const uint32_t row = (uint32_t)row0 + to_r[u];
                    T* out = reinterpret_cast<T*>((is_v ? rows.v : rows.k) + (uint64_t)row * (is_v ? v_stride : k_stride)) +
                             (is_v ? to_i[u] - c.nkv : to_i[u]) * HD + col;
                    float f[8];
                    if constexpr (FP8) {
                        const float scale = pg_scale(e[u]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float2 y = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(((q < 2 ? x[u].x : x[u].y) >> (16 * (q & 1))) & 0xffffu));
                            f[2 * q] = y.x * scale;
                            f[2 * q + 1] = y.y * scale;
                        }
                        pg_store8<T>(out, f);
                    } else if constexpr (sizeof(T) == 2) {
                        *reinterpret_cast<uint4*>(out) = x[u];
                    } else {
                        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            f[2 * q] = bf_lo(w[q]);
                            f[2 * q + 1] = bf_hi(w[q]);
                        }
                        pg_store8<T>(out, f);
                    }
                }
        }
    }
}

// 16 (or 4) bytes to shared memory, asynchronously; nothing is read and zeros are written when `ok` is false.
__device__ __forceinline__ void pa_copy16(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pa_copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void pa_copy4(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint4 pa_lds16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 pa_lds8(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}

// D += A * B, one m16n8k16 tile of f16 (e4m3 caches) or bf16 operands.  Not volatile: the compiler may interleave chains.
template <bool FP8>
__device__ __forceinline__ void pa_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (FP8)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// ---- page selection

struct PagedSelect {
    const uint8_t* q;
    int64_t q_stride;      // bytes
    uint32_t q_f32, G;
    uint32_t keep_first, keep_last, n_select;
    int32_t* selected;
    float2* scores;        // [n_seqs][nkv][table_pages]: score, bound of its error
};
__device__ __forceinline__ float pg_q(const uint8_t* row, uint32_t f32, uint32_t i) {
    return f32 ? reinterpret_cast<const float*>(row)[i] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[i]);
}

// A score as a whole number of the same order: at least 2, NaN 1, so that 0 is below every page.
__device__ __forceinline__ uint32_t pg_key(float x) {
    if (isnan(x)) return 1u;
    const uint32_t u = __float_as_uint(x + 0.f);   // -0 becomes +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The exact score of a page, by one warp: sums in 64 bits (the products of a bf16 bound and a query are exact there, and so,
// but for extreme spreads, are their sums), rounded once to 32; the largest over query heads [g0, g1) of kv head h.
__device__ __forceinline__ float ps_exact(const PagedView& c, const PagedSelect& a, uint32_t s, uint32_t h, int32_t phys, uint32_t g0, uint32_t g1) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t* b = reinterpret_cast<const uint32_t*>(c.bounds + ((int64_t)phys * c.nkv + h) * 2 * c.hd);
    const uint8_t* q = a.q + (int64_t)s * a.q_stride;
    uint32_t lo[4], hi[4];   // columns 2 lane + 64 i, + 1
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (64u * i < c.hd) {
            lo[i] = b[lane + 32u * i];
            hi[i] = b[c.hd / 2u + lane + 32u * i];
        }
    float best = __int_as_float(0x7fc00000);   // NaN
#pragma unroll 1
    for (uint32_t g = g0; g < g1; ++g) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (64u * i < c.hd) {
                const uint32_t d = (h * a.G + g) * c.hd + 2u * lane + 64u * i;
                const float x = pg_q(q, a.q_f32, d), y = pg_q(q, a.q_f32, d + 1u);
                sum += (double)x * (double)bf_lo(x >= 0.f ? hi[i] : lo[i]);
                sum += (double)y * (double)bf_hi(y >= 0.f ? hi[i] : lo[i]);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        best = fmaxf(best, (float)sum);        // fmaxf leaves NaN out
    }
    return best;
}

// Scores good to a known bound, on the tensor cores: kl_paged_topk_kernel computes exact ones where the bound leaves the
// choice open, which is a few pages of thousands where pages differ (64-bit scores for every page kept the 64-bit pipe and the
// selects in front of it busy for five times as long as reading the bounds takes).
//   max(q lo, q hi) = min(q, 0) lo + max(q, 0) hi: with the bounds [lo | hi] of a page as a row of 2 hd numbers and
//   [min(q, 0) | max(q, 0)] as columns it is one matrix product, pages x heads.  16 pages are the rows of mma.m16n8k16, up to
//   eight heads its columns (the order of the 2 hd terms is free, so a lane takes 16 contiguous bytes of its two rows at a time).  Every warp takes an equal, contiguous range of
//   all tiles of 16 pages and brings them in through a ring of its own in shared memory.  Written per page: the score and a bound
//   of its error.
// Measured: 397 thousand (page, head) pairs of 512 bytes, eight query heads each, 40.5 us (5.0 TB/s, what the kernel needs to
// start and end included), 42.8 with rows loaded straight into registers.
// Error bound: a product of two bf16 is exact, and the matrix instruction adds with at least single precision, in an order of
// its own: each addition is off by at most a unit, 2^-23, of the sum of all magnitudes.  A step adds 16 products and there are hd / 8 of
// them (fp32 queries: twice as many, and the two parts leave 2^-16 of a query): hd * 2^-22 (hd * 2^-21 + 2^-16) of the
// largest sum |q_d| of a head times the page's largest bound; infinite where a score or bound is not finite, and below 2^-100:
// numbers under 2^-126 have fewer bits (a rest of a query is off by up to 2^-134), which the bound does not count.  Errors seen
// (random, widely spread, equal, cancelling terms, a large one among small ones) stay below 9 % of it.
template <int HD>
struct PsCfg {
    static constexpr int ROW = 4 * HD, TILE = 16 * ROW;   // bytes of a page's bounds, of a tile's
    static constexpr int NW = HD == 256 ? 6 : 12;         // warps
    static constexpr int ST = 196608 / (NW * TILE);       // tiles of a warp's ring: 4, 2, 2
    static constexpr size_t SMEM = (size_t)NW * ST * TILE;
};
template <int HD, bool F32>   // F32: type of the queries
__global__ void __launch_bounds__(PsCfg<HD>::NW * 32, 1) kl_paged_score_kernel(const PagedView c, const PagedSelect a) {
    using Cfg = PsCfg<HD>;
    constexpr int NW = Cfg::NW, ST = Cfg::ST, ROW = Cfg::ROW, TILE = Cfg::TILE;
    constexpr int NC = HD / 16;                         // 16-byte pieces of a row per lane
    constexpr int CPR = ROW / 16, PASSES = 16 * CPR / 32;   // pieces of a row; copies of a lane per tile
    extern __shared__ __align__(128) uint8_t ps_smem[];
    __shared__ uint64_t pre[NW * 32], wsum[NW];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, g = lane >> 2, j = lane & 3u;
    const uint32_t n = c.n_seqs, per = (n + NW * 32u - 1u) / (NW * 32u), HT = (a.G + 7u) / 8u;
    auto pages_of = [&](uint32_t s) { return (pg_length(c, s) + c.page - 1u) / c.page; };
    const uint64_t W = pg_prefix<NW>(n, pre, wsum, [&](uint32_t s) { return (uint64_t)((pages_of(s) + 15u) / 16u) * c.nkv; });
    const uint32_t warps = gridDim.x * NW, w = warp * gridDim.x + blockIdx.x;   // few tiles spread over the SMs
    const uint64_t share = pg_div(W, warps), over = W - share * warps;
    const uint64_t lo = share * w + min((uint64_t)w, over), hi = lo + share + (w < over ? 1u : 0u);
    if (lo >= hi) return;
    struct Cursor { uint32_t s, h, t, np, nt; };   // sequence, kv head, tile; pages and tiles per head of the sequence
    Cursor cur;
    {
        const uint32_t i0 = pg_find<NW>(pre, lo);
        uint64_t rem = lo - pre[i0];
        cur.s = i0 * per;
        cur.np = pages_of(cur.s);
        cur.nt = (cur.np + 15u) / 16u;
        while (rem >= (uint64_t)cur.nt * c.nkv) {
            rem -= (uint64_t)cur.nt * c.nkv;
            cur.np = pages_of(++cur.s);
            cur.nt = (cur.np + 15u) / 16u;
        }
        cur.h = (uint32_t)pg_div(rem, cur.nt);
        cur.t = (uint32_t)(rem - (uint64_t)cur.h * cur.nt);
    }
    auto advance = [&](Cursor& x) {   // to a tile that exists
        if (++x.t < x.nt) return;
        x.t = 0;
        if (++x.h < c.nkv) return;
        x.h = 0;
        do {
            x.np = pages_of(++x.s);
            x.nt = (x.np + 15u) / 16u;
        } while (x.nt == 0u);
    };
    // Requests: lane l < 16 looks up where the bounds of page 16 t + l lie, one tile ahead of the copies.
    Cursor req = cur;
    uint64_t left = hi - lo;   // tiles still to request
    int64_t at = -1;
    auto look_up = [&]() {
        const uint32_t p = req.t * 16u + lane;
        const int32_t phys = lane < 16u && p < req.np ? pg_physical(c, req.s, p) : -1;
        at = phys < 0 ? -1 : ((int64_t)phys * c.nkv + req.h) * ROW;
    };
    look_up();
    const uint32_t ring = smem_u32(ps_smem) + warp * (ST * TILE);
    auto swizzle = [](uint32_t r) { return (r & 1u) << 2 | ((r >> 1) & 3u); };   // as in the attention kernel's tiles
    auto request = [&](uint32_t slot) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const uint32_t e = i * 32 + lane, r = e / CPR, piece = e % CPR;
            const int64_t from = __shfl_sync(0xffffffffu, at, r);
            pa_copy16(ring + slot * TILE + r * ROW + ((piece ^ swizzle(r)) << 4), reinterpret_cast<const uint8_t*>(c.bounds) + max(from, (int64_t)0) + piece * 16u,
                      from >= 0);
        }
        if (--left) {
            advance(req);
            look_up();
        }
    };
    uint32_t qf[NC][2][2], ql[F32 ? NC : 1][2][2];   // B fragments of the current head tile, and what bf16 leaves of fp32 queries
    float q1 = 0.f;   // largest sum |q_d| of the heads seen, infinite where one is NaN
    auto load_queries = [&](uint32_t ht) {
        float sum = 0.f;
        const uint32_t head = cur.h * a.G + min(ht * 8u + g, a.G - 1u);   // a missing head repeats the last one
        const uint8_t* q = a.q + (int64_t)cur.s * a.q_stride + (size_t)head * HD * (F32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t d = (i % (NC / 2)) * 32 + j * 8 + x * 4;
                float v[4];
                if (F32) {
                    const float4 f = *reinterpret_cast<const float4*>(q + d * 4);
                    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
                } else {
                    const uint2 f = *reinterpret_cast<const uint2*>(q + d * 2);
                    v[0] = bf_lo(f.x); v[1] = bf_hi(f.x); v[2] = bf_lo(f.y); v[3] = bf_hi(f.y);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (i < NC / 2) sum += fabsf(v[e]);
                    v[e] = i < NC / 2 ? fminf(v[e], 0.f) : fmaxf(v[e], 0.f);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    qf[i][x][e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                    if (F32) ql[F32 ? i : 0][x][e] = pack_bf16(v[2 * e] - bf_lo(qf[i][x][e]), v[2 * e + 1] - bf_hi(qf[i][x][e]));
                }
            }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (isnan(sum)) sum = INFINITY;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum = fmaxf(sum, __shfl_xor_sync(0xffffffffu, sum, o));
        q1 = ht ? fmaxf(q1, sum) : sum;
    };
    bool fresh = true;
    uint32_t to = 0, slot = 0, ahead = 0;
    for (uint64_t k = lo; k < hi;) {
        if (ahead >= (uint32_t)ST - 1u) {
            if (fresh && HT == 1u) load_queries(0);
            fresh = false;
            asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
            __syncwarp();   // the tile is there for every lane, and every lane is done with the previous one
        }
        if (left) request(to);
        if (++to == (uint32_t)ST) to = 0;
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (ahead < (uint32_t)ST - 1u) {   // the first ST - 1 tiles are only requested
            ++ahead;
            continue;
        }
        const uint32_t rows = ring + slot * TILE + g * ROW, fk = swizzle(g);   // rows g and g + 8: the same swizzle
        float best0 = -INFINITY, best1 = -INFINITY;
        uint32_t big0 = 0, big1 = 0;   // largest magnitudes, two columns of bf16 (their signs mean nothing)
        for (uint32_t ht = 0; ht < HT; ++ht) {
            if (HT > 1u) load_queries(ht);
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k4 = 0; k4 < NC; ++k4) {
                const uint32_t piece = ((k4 * 4 + j) ^ fk) << 4;
                const uint4 x = pa_lds16(rows + piece), y = pa_lds16(rows + 8 * ROW + piece);
                pa_mma<false>(acc, x.x, y.x, x.y, y.y, qf[k4][0][0], qf[k4][0][1]);
                pa_mma<false>(acc, x.z, y.z, x.w, y.w, qf[k4][1][0], qf[k4][1][1]);
                if (F32) {
                    pa_mma<false>(acc, x.x, y.x, x.y, y.y, ql[F32 ? k4 : 0][0][0], ql[F32 ? k4 : 0][0][1]);
                    pa_mma<false>(acc, x.z, y.z, x.w, y.w, ql[F32 ? k4 : 0][1][0], ql[F32 ? k4 : 0][1][1]);
                }
                if (ht == 0u) {
                    big0 = pg_larger(pg_larger(big0, pg_larger(x.x, x.y)), pg_larger(x.z, x.w));
                    big1 = pg_larger(pg_larger(big1, pg_larger(y.x, y.y)), pg_larger(y.z, y.w));
                }
            }
            // (a NaN must not be lost in a maximum: it says that the score is not known)
            auto larger = [](float u, float v) { return isnan(u) || isnan(v) ? __int_as_float(0x7fc00000) : fmaxf(u, v); };
            best0 = larger(best0, larger(acc[0], acc[1]));
            best1 = larger(best1, larger(acc[2], acc[3]));
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            const float u = __shfl_xor_sync(0xffffffffu, best0, o), v = __shfl_xor_sync(0xffffffffu, best1, o);
            best0 = isnan(u) || isnan(best0) ? __int_as_float(0x7fc00000) : fmaxf(best0, u);
            best1 = isnan(v) || isnan(best1) ? __int_as_float(0x7fc00000) : fmaxf(best1, v);
            big0 = pg_larger(big0, __shfl_xor_sync(0xffffffffu, big0, o));
            big1 = pg_larger(big1, __shfl_xor_sync(0xffffffffu, big1, o));
        }
        if (j < 2u) {   // lane 0 of the quad stores page g, lane 1 page g + 8
            const uint32_t p = cur.t * 16u + g + j * 8u, b = (j ? big1 : big0) & 0x7fff7fffu;
            const float mag = __uint_as_float(max(b >> 16, b & 0xffffu) << 16);
            const float score = j ? best1 : best0, err = q1 * 1.001f * mag * (F32 ? HD * 0x1p-21f + 0x1p-16f : HD * 0x1p-22f);
            // (infinite where nothing is known: 0 * infinity, a score that is not finite, queries whose halves and products
            // whose sums reach down to where numbers have fewer bits; zeros are exact)
            const bool known = isfinite(score) && (q1 == 0.f || mag == 0.f ? err == 0.f : q1 >= 0x1p-100f && err >= 0x1p-100f);
            if (p < cur.np) a.scores[((size_t)cur.s * c.nkv + cur.h) * c.table_pages + p] = make_float2(score, known ? err : INFINITY);
        }
        if (++slot == (uint32_t)ST) slot = 0;
        if (++k < hi) {
            const uint32_t h = cur.h, s = cur.s;
            advance(cur);
            fresh = cur.h != h || cur.s != s;
        }
    }
}

// The choice: one block per (sequence, kv head).
//   1. T = the need-th largest of the approximate scores: by a histogram and the ranks within one bin, or, where too many
//      keys share the bin, bit by bit (from below the bits all of them share).
//   2. With E the largest bound of their errors, pages above T + 2 E are chosen for certain and pages below T - 2 E are not.
//      What lies between is chosen too if there is room for all of it; otherwise exact scores decide (equal ones by page): for
//      up to PT_LIST candidates a warp scores one query head of one each and they are ranked against one another, for more (many equal
//      scores, or E infinite) a threshold is found bit by bit among the exact scores.
//   3. The chosen pages are put in order by a prefix sum over groups of 32.
// The keys lie in shared memory (SMEM), or, beyond PT_KEYS pages, in the workspace.  A block's time is latency -- barriers, and
// fetching its own instructions, each of which runs a few times only -- so the loops are not unrolled (eight keys per thread in
// registers and everything unrolled took twice as long).  Measured: 5 us for 1024 pages, 4 to 11 us for 4096.
// E is that of the (sequence, head)'s worst page.  One page of unknown score (a bound that is infinite) makes every page a
// candidate, and so do equal pages; beyond PT_LIST of them a warp scores its candidates one after another.  Both calls together, 8 kv heads of
// 128, 4 query heads each: one sequence of 4096 pages 675 us instead of 19, 32 of 1024 211 instead of 37; one page 64 times as loud as the
// others 46 and 63.
constexpr int PT_THREADS = 512;
constexpr uint32_t PT_LIST = 128, PT_KEYS = 16384;
template <bool SMEM>
__global__ void __launch_bounds__(PT_THREADS, 2) kl_paged_topk_kernel(const PagedView c, const PagedSelect a) {
    constexpr int NW = PT_THREADS / 32;
    constexpr uint32_t SURE = 0xffffffffu;   // key of a page that is chosen in any case; 0: of one that is not
    extern __shared__ uint32_t keys_s[];     // [pages of the longest sequence] (SMEM)
    __shared__ uint4 red[2][NW];
    __shared__ uint32_t list_n, sure_n, list_page[PT_LIST], list_key[PT_LIST], found[4], hist[PT_THREADS];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint32_t n = (pg_length(c, s) + c.page - 1u) / c.page;
    float2* sc = a.scores + ((size_t)s * c.nkv + h) * c.table_pages;
    int32_t* out = a.selected + ((size_t)s * c.nkv + h) * a.n_select;
    if (n <= a.n_select) {   // all of them
        for (uint32_t i = tid; i < a.n_select; i += PT_THREADS) out[i] = i < n ? (int32_t)i : -1;
        return;
    }
    auto number = [](uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); };   // the score behind a key
    auto key = [&](uint32_t i) -> uint32_t& { return SMEM ? keys_s[i] : reinterpret_cast<uint32_t*>(sc + i)[1]; };
    const uint32_t need = a.n_select - (a.keep_first + a.keep_last);   // n > n_select >= keep_first + keep_last
    hist[tid] = 0u;
    if (tid == 0u) list_n = sure_n = 0u;

    int turn = 0;
    // sums of x, y, or the maxima of x, z and the minimum of y, over the block
    auto reduce = [&](uint32_t x, uint32_t y, uint32_t z, bool extremes) -> uint4 {
        x = extremes ? __reduce_max_sync(0xffffffffu, x) : __reduce_add_sync(0xffffffffu, x);
        y = extremes ? __reduce_min_sync(0xffffffffu, y) : __reduce_add_sync(0xffffffffu, y);
        if (extremes) z = __reduce_max_sync(0xffffffffu, z);
        if (lane == 0u) red[turn][warp] = make_uint4(x, y, z, 0u);
        __syncthreads();
        const uint4 p = red[turn][lane % NW];
        turn ^= 1;   // the next call writes the other half, and nobody is two calls behind
        uint4 t;
        t.x = extremes ? __reduce_max_sync(0xffffffffu, p.x) : __reduce_add_sync(0xffffffffu, lane < (uint32_t)NW ? p.x : 0u);
        t.y = extremes ? __reduce_min_sync(0xffffffffu, p.y) : __reduce_add_sync(0xffffffffu, lane < (uint32_t)NW ? p.y : 0u);
        t.z = extremes ? __reduce_max_sync(0xffffffffu, p.z) : 0u;
        return t;
    };
    // exclusive prefix sum over the block's threads
    auto scan = [&](uint32_t v) {
        uint32_t incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= (uint32_t)o) incl += y;
        }
        if (lane == 31u) red[turn][warp].x = incl;
        __syncthreads();
        const uint32_t p = lane < warp ? red[turn][lane].x : 0u;   // warp < NW <= 32
        turn ^= 1;
        return incl - v + __reduce_add_sync(0xffffffffu, p);
    };
    // The largest t that at least `want` keys (but SURE) reach -- lo and hi: the smallest and the largest key but SURE and 0 --
    // or, as soon as a t is found that exactly `want` keys reach, that one (exact).
    auto threshold = [&](uint32_t lo, uint32_t hi, uint32_t want, bool& exact) {
        const uint32_t differ = lo ^ hi;
        int bit = differ ? 31 - __clz(differ) : -1;
        uint32_t t = bit >= 0 ? lo & ~((2u << bit) - 1u) : lo;
        exact = false;
#pragma unroll 1
        for (; bit >= 0 && !exact; --bit) {
            uint32_t x = 0;
#pragma unroll 1
            for (uint32_t i = tid; i < n; i += PT_THREADS) x += key(i) >= (t | 1u << bit) && key(i) != SURE;
            x = reduce(x, 0u, 0u, false).x;
            if (x >= want) {
                t |= 1u << bit;
                exact = x == want;
            }
        }
        return t;
    };

    uint32_t mx = 0, mn = 0xffffffffu, err = 0;
#pragma unroll 1
    for (uint32_t i = tid; i < n; i += PT_THREADS) {
        const float2 x = sc[i];
        uint32_t k = SURE;
        if (i >= a.keep_first && i + a.keep_last < n) {
            k = pg_key(x.x);
            mx = max(mx, k);
            mn = min(mn, k);
            err = max(err, __float_as_uint(x.y));   // not negative: ordered like whole numbers
        }
        key(i) = need || k == SURE ? k : 0u;
    }
    uint32_t t = SURE - 1u, ties = 0;   // chosen: keys above t, and the first `ties` of those equal to it
    if (need) {
        const uint4 all = reduce(mx, mn, err, true);
        const float E = __uint_as_float(all.z);
        float above = INFINITY, below = -INFINITY;
        if (isfinite(E)) {
            // bins of equal width between the smallest and the largest score
            const float x0 = number(all.y), width = (PT_THREADS - 1) / (number(all.x) - x0);
            auto bin_of = [&](uint32_t k) { return (uint32_t)min(PT_THREADS - 1, max(0, (int)((number(k) - x0) * width))); };
#pragma unroll 1
            for (uint32_t i = tid; i < n; i += PT_THREADS)
                if (key(i) != SURE) atomicAdd(&hist[bin_of(key(i))], 1u);
            __syncthreads();
            const uint32_t mine = hist[PT_THREADS - 1 - tid], higher = scan(mine);   // from the last bin down
            if (higher < need && higher + mine >= need) {   // one thread
                found[0] = PT_THREADS - 1 - tid;
                found[1] = need - higher;                   // rank within the bin, from 1
                found[2] = mine;
            }
            __syncthreads();
            const uint32_t bin = found[0], rank = found[1], cnt = found[2];
            uint32_t low;
            if (cnt <= PT_LIST) {
#pragma unroll 1
                for (uint32_t i = tid; i < n; i += PT_THREADS)
                    if (key(i) != SURE && bin_of(key(i)) == bin)   // (cnt of them, unless another call writes the workspace)
                        list_key[min(atomicAdd(&list_n, 1u), PT_LIST - 1u)] = key(i);
                __syncthreads();
                if (tid < cnt) {
                    const uint32_t k = list_key[tid];
                    uint32_t before = 0;
#pragma unroll 1
                    for (uint32_t i = 0; i < cnt; ++i) before += list_key[i] > k || (list_key[i] == k && i < tid);
                    if (before + 1u == rank) found[3] = k;
                }
                if (tid == PT_THREADS - 1) list_n = 0u;
                __syncthreads();
                low = found[3];
            } else {
                bool exact;
                low = threshold(all.y, all.x, need, exact);
                if (exact) {   // the smallest key that reaches it is the need-th largest
                    uint32_t k = 0xffffffffu;
#pragma unroll 1
                    for (uint32_t i = tid; i < n; i += PT_THREADS)
                        if (key(i) >= low) k = min(k, key(i));
                    low = reduce(0u, k, 0u, true).y;
                }
            }
            above = __fadd_ru(number(low), 2.f * E);
            below = __fadd_rd(number(low), -2.f * E);
        }
        // certain ones, and the list of candidates
        uint32_t sure = 0;
#pragma unroll 1
        for (uint32_t i = tid; i < n; i += PT_THREADS) {
            const uint32_t k = key(i);
            if (k == SURE) continue;
            const float x = number(k);
            if (k != 1u && x > above) {        // 1: NaN, always a candidate
                key(i) = SURE;
                ++sure;
            } else if (k != 1u && x < below) {
                key(i) = 0u;
            } else {
                const uint32_t at = atomicAdd(&list_n, 1u);
                if (at < PT_LIST) list_page[at] = i;
            }
        }
        sure = __reduce_add_sync(0xffffffffu, sure);
        if (lane == 0u && sure) atomicAdd(&sure_n, sure);
        __syncthreads();
        const uint32_t cand = list_n, room = need - sure_n;   // room for candidates
        if (cand <= PT_LIST) {
            if (cand > room) {   // their exact scores decide
                if (tid < cand) list_key[tid] = 0u;
                __syncthreads();
#pragma unroll 1
                for (uint32_t i = warp; i < cand * a.G; i += NW) {   // a warp per candidate and query head
                    const uint32_t x = i / a.G, g = i - x * a.G;
                    const int32_t phys = pg_physical(c, s, list_page[x]);
                    const uint32_t k = phys >= 0 ? pg_key(ps_exact(c, a, s, h, phys, g, g + 1u)) : 1u;
                    if (lane == 0u) atomicMax(&list_key[x], k);
                }
                __syncthreads();
            }
            if (tid < cand) {
                uint32_t before = 0;   // its rank among the candidates
                if (cand > room) {
                    const uint32_t k = list_key[tid], page = list_page[tid];
#pragma unroll 1
                    for (uint32_t i = 0; i < cand; ++i) before += list_key[i] > k || (list_key[i] == k && list_page[i] < page);
                }
                key(list_page[tid]) = before < room ? SURE : 0u;
            }
            __syncthreads();
        } else {
            uint32_t cmx = 0, cmn = 0xffffffffu;
#pragma unroll 1
            for (uint32_t i0 = 0; i0 < n; i0 += PT_THREADS) {   // whole warps: a warp scores its candidates one after another
                const uint32_t i = i0 + tid;
                const bool ask = i < n && key(i) != SURE && key(i) != 0u;
                const int32_t phys = ask && cand > room ? pg_physical(c, s, i) : -1;
                uint32_t k = SURE;
                if (cand > room)
                    for (uint32_t todo = __ballot_sync(0xffffffffu, ask); todo; todo &= todo - 1u) {
                        const int src = __ffs(todo) - 1;
                        const int32_t ph = __shfl_sync(0xffffffffu, phys, src);
                        const uint32_t ek = ph >= 0 ? pg_key(ps_exact(c, a, s, h, ph, 0u, a.G)) : 1u;
                        if ((int)lane == src) {
                            k = ek;
                            cmx = max(cmx, ek);
                            cmn = min(cmn, ek);
                        }
                    }
                if (ask) key(i) = k;
            }
            if (cand > room) {
                const uint4 ce = reduce(cmx, cmn, 0u, true);
                bool exact;
                t = threshold(ce.y, ce.x, room, exact);
                ties = 0xffffffffu;
                if (!exact) {
                    uint32_t x = 0;
#pragma unroll 1
                    for (uint32_t i = tid; i < n; i += PT_THREADS) x += key(i) > t && key(i) != SURE;
                    ties = room - reduce(x, 0u, 0u, false).x;
                }
            }
        }
    }
    // in order, PT_THREADS groups of 32 pages at a time
    uint32_t done = 0, tied = 0;   // chosen pages without the equal ones, and equal ones, so far
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < n; i0 += PT_THREADS * 32u) {
        const uint32_t end = min(n, i0 + PT_THREADS * 32u);
        __syncthreads();   // hist takes the groups' counts, and then their sums
#pragma unroll 1
        for (uint32_t g = warp; g < (uint32_t)PT_THREADS; g += NW) {
            const uint32_t i = i0 + g * 32u + lane, k = i < end ? key(i) : 0u;
            const uint32_t bs = __ballot_sync(0xffffffffu, k > t), be = __ballot_sync(0xffffffffu, ties && k == t);
            if (lane == 0u) hist[g] = __popc(bs) | __popc(be) << 16;   // sums of at most 2^14 each
            if (i0 + g * 32u >= end) break;
        }
        __syncthreads();
        const uint32_t groups = (end - i0 + 31u) / 32u, v = tid < groups ? hist[tid] : 0u, before = scan(v);
        hist[tid] = before;
        if (tid == PT_THREADS - 1) found[0] = before + v;
        __syncthreads();
#pragma unroll 1
        for (uint32_t g = warp; g < groups; g += NW) {
            const uint32_t i = i0 + g * 32u + lane, k = i < end ? key(i) : 0u, under = (1u << lane) - 1u;
            const bool eq = ties && k == t;
            const uint32_t bs = __ballot_sync(0xffffffffu, k > t), be = __ballot_sync(0xffffffffu, eq);
            const uint32_t e = tied + (hist[g] >> 16) + __popc(be & under);
            const uint32_t at = done + (hist[g] & 0xffffu) + __popc(bs & under) + min(e, ties);
            if ((k > t || (eq && e < ties)) && at < a.n_select) out[at] = (int32_t)i;
        }
        done += found[0] & 0xffffu;
        tied += found[0] >> 16;
    }
}

// ---- attention

struct PagedAttn {
    const uint8_t* q;
    uint8_t* out;
    int64_t q_stride, out_stride;   // bytes
    uint32_t out_mode;              // PA_BF16, PA_F32, PA_OPERAND
    uint32_t nq, G, HT;             // G query heads per kv head, in HT tiles of at most eight
    float scale_log2;               // scale * log2(e)
    uint32_t window;                // 0: none
    const int32_t* selected;        // [n_seqs][nkv][n_select] or null
    uint32_t n_select;
    float* lse;                     // or null
    uint32_t whole_pairs;           // 1: no pair is shared between blocks (and kl_paged_merge_kernel does not follow)
    // workspace: partial results, one record = [8 heads][hd] sums and [8 heads] (maximum, sum)
    float *part, *part_ml;          // [blocks][2]: the pair that began in an earlier block, the pair that goes on in the next one
    float *head, *head_ml;          // [blocks][warps]: a warp's first pair when it began in an earlier warp
    int4* meta;                     // [blocks]: the pair of the second record (sequence, pair in the sequence) and the last
                                    // block that shares it; .x = 0: no such pair
};
enum { PA_BF16 = 0, PA_F32 = 1, PA_OPERAND = 2 };

__device__ __forceinline__ float pa_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pa_pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Two numbers rounded to 16 bits (f16 with an e4m3 cache, bf16 else), what that leaves of them, and what the two leave where
// they are bf16 (eight bits each: 24 with a third).
template <bool FP8>
__device__ __forceinline__ uint32_t pa_round(float x0, float x1) {
    return FP8 ? pa_pack_f16(x0, x1) : pack_bf16(x0, x1);
}
template <bool FP8>
__device__ __forceinline__ uint32_t pa_rest(float x0, float x1, uint32_t hi) {
    if (!FP8) return pack_bf16(x0 - bf_lo(hi), x1 - bf_hi(hi));
    const float2 f = pg_f16x2_to_float2(hi);
    return pa_pack_f16(x0 - f.x, x1 - f.y);
}
__device__ __forceinline__ uint32_t pa_rest2(float x0, float x1, uint32_t hi, uint32_t lo) {   // both differences are exact
    return pack_bf16(x0 - bf_lo(hi) - bf_lo(lo), x1 - bf_hi(hi) - bf_hi(lo));
}
// Two neighbouring columns (d even) of query head hq of sequence s.
__device__ __forceinline__ void pa_store2(const PagedView& c, const PagedAttn& a, uint32_t s, uint32_t hq, uint32_t d, float v0, float v1) {
    if (a.out_mode == PA_F32) {
        *reinterpret_cast<float2*>(a.out + (int64_t)s * a.out_stride + ((size_t)hq * c.hd + d) * 4) = make_float2(v0, v1);
    } else if (a.out_mode == PA_BF16) {
        *reinterpret_cast<uint32_t*>(a.out + (int64_t)s * a.out_stride + ((size_t)hq * c.hd + d) * 2) = pack_bf16(v0, v1);
    } else {   // the operand of a batched projection: rows 0..31 hi halves, rows 32..63 lo halves
        __nv_bfloat16* x = reinterpret_cast<__nv_bfloat16*>(a.out);
        const size_t width = (size_t)a.nq * c.hd, at = (size_t)hq * c.hd + d;
        const uint32_t hi = pack_bf16(v0, v1);
        *reinterpret_cast<uint32_t*>(x + s * width + at) = hi;
        *reinterpret_cast<uint32_t*>(x + (32 + s) * width + at) = pack_bf16(v0 - bf_lo(hi), v1 - bf_hi(hi));
    }
}
__device__ __forceinline__ void pa_store1(const PagedView& c, const PagedAttn& a, uint32_t s, uint32_t hq, uint32_t d, float v) {
    if (a.out_mode == PA_F32) {
        *reinterpret_cast<float*>(a.out + (int64_t)s * a.out_stride + ((size_t)hq * c.hd + d) * 4) = v;
    } else if (a.out_mode == PA_BF16) {
        *reinterpret_cast<__nv_bfloat16*>(a.out + (int64_t)s * a.out_stride + ((size_t)hq * c.hd + d) * 2) = __float2bfloat16_rn(v);
    } else {
        __nv_bfloat16* x = reinterpret_cast<__nv_bfloat16*>(a.out);
        const size_t width = (size_t)a.nq * c.hd, at = (size_t)hq * c.hd + d;
        const __nv_bfloat16 hi = __float2bfloat16_rn(v);
        x[s * width + at] = hi;
        x[(32 + s) * width + at] = __float2bfloat16_rn(v - __bfloat162float(hi));
    }
}
__device__ __forceinline__ void pa_store_lse(const PagedAttn& a, uint32_t s, uint32_t hq, float m, float l) {
    if (a.lse) a.lse[(size_t)s * a.nq + hq] = (m + log2f(l)) * 0.6931471805599453f;   // l == 0: -inf
}

constexpr uint32_t PA_NONE = 0x7fffffffu;   // position of a row group that holds nothing to attend to
constexpr int PA_MAX_WARPS = 12;
constexpr int PA_LENS = 1024;               // sequences whose lengths are kept in shared memory
constexpr uint32_t PA_MIN_TILES = 8;        // fewest tiles worth a block

// EX: fp32 queries and outputs -- what 16-bit rounding leaves of q enters the score product too.
// Warps and tile: as many warps as the registers allow, with at least two tiles each in the ring.  Measured (device time of
// kl_paged_attention): 32 sequences of <= 32768 e4m3 positions, 8 heads per kv head, head size 128: 12 warps x 32 positions
// 162 us, 11 x 32 168, 6 x 64 174, 12 x 16 183, 16 x 16 (128 registers) 215; 32 x 4096 bf16, when probabilities had two parts: 12 x 16
// 90, 8 x 16 98.  Registers spilled, in bytes: e4m3 of 128 with bf16 queries 44 (pages not of 16 rows: 92), head size 256 with fp32 queries 218 to
// 298, bf16 of 64 with fp32 queries 16, bf16 of 256 with bf16 queries and pages not of 16 rows 8.
template <int HD, bool FP8, bool EX>
struct PaCfg {
    static constexpr int ROW = FP8 ? HD : 2 * HD;            // bytes of a cached row
    static constexpr int NW = HD == 256 ? (FP8 ? 8 : 6) : EX && HD == 128 ? 8 : 12;   // warps
    static constexpr int TP = HD == 64 || (HD == 128 && FP8) ? 32 : 16;               // positions per tile
    static constexpr int TILE = TP * ROW;                    // bytes of a K (or V) tile
    static constexpr int RING = 204800 / (NW * 2 * TILE);
    static constexpr int ST = RING > 8 ? 8 : RING;           // tiles of a warp's ring
    // fp32 queries and a bf16 cache: the queries' third parts, 8 bytes of a lane per 16 columns, lie in shared memory where
    // registers do not suffice (32 x 4096, 16 heads of 256: 178 us spilled, 102 so, 100 without a third part)
    static constexpr bool QM = EX && !FP8 && HD == 256;
    static constexpr size_t SMEM = (size_t)NW * ST * (2 * TILE + 2 * TP + TP) + NW * 8 * 8 + 512 * 8 + PA_LENS * 4 + 256 + (QM ? NW * 32 * HD / 2 : 0);
    static_assert(ST >= 2 && SMEM <= 232448, "ring");
    static_assert(NW <= PA_MAX_WARPS, "workspace");
};

// Short pairs are not shared between blocks, which makes the merge kernel unnecessary (3 us on the device, 3 us on the host) but
// leaves a pair to one block: up to PA_WHOLE_FEW tiles always, up to PA_WHOLE_MANY tiles where there are as many pairs as blocks.
// Measured, whole against shared, 8 kv heads (4 of 256).  One sequence: bf16 of 128 (tiles of 16) 256 positions 8.7 us against 9.2, 384 9.5 against
// 9.2, 512 10.4 against 9.4, 1024 13.6 against 9.8; bf16 of 256 (16) 256 10.5 against 10.7, 384 12.5 against 10.8, e4m3 12.5 against 11.4; e4m3 of 128
// (32) 384 9.8 against 10.9, 512 10.7 against 10.4, 768 11.6 against 10.8; bf16 of 64 (32) 768 8.4 against 8.9, 1024 9.4 against 9.1, e4m3 8.9
// against 9.2 and 9.9 against 9.4.  So 24 tiles are where the two meet, give or take a third, and cost 16 % at most where they are too many.
// 32 sequences: bf16 of 128 512 positions 19.3 against 22.6, 1024 29.2 against 32.7; e4m3 of 128 2048 33.4 against 35.6; of 64 27.9 against
// 31.1 (e4m3 23.1 against 25.1); bf16 of 256 1024 28.2 against 33.4; 128 sequences of 1024 95.0 against 101.2, e4m3 60.0 against 63.4.
// Longer ones are shared although 32 x 2048 bf16 would gain 4 us too: lengths are not known on the host, and one long sequence
// among short ones would leave its pairs to a block each.
constexpr uint32_t PA_WHOLE_FEW = 24, PA_WHOLE_MANY = 64;

// Positions of sequence s that take part, as tiles.
struct PaSeq {
    uint32_t len, lo;   // positions [lo, len)
    uint32_t t0, nt;    // tiles [t0, t0 + nt) of its (virtual) positions
    uint32_t listed;    // entries of the page list that are looked at
};
template <uint32_t TP>
__device__ __forceinline__ PaSeq pa_seq(const PagedView& c, const PagedAttn& a, uint32_t len) {
    PaSeq q;
    q.len = len;
    q.lo = a.window && len > a.window ? len - a.window : 0u;
    if (a.selected) {
        q.listed = min(a.n_select, (len + c.page - 1u) / c.page);
        q.t0 = 0;
        q.nt = (uint32_t)(((uint64_t)q.listed * c.page + TP - 1u) / TP);
    } else {
        q.listed = 0;
        q.t0 = q.lo / TP;
        q.nt = len ? (len + TP - 1u) / TP - q.t0 : 0u;
    }
    return q;
}

// Attention of one new token per sequence as ONE balanced stream over the whole batch.
//
//   * Work: TP positions of one kv head of one sequence, for up to eight of the query heads that share it, are a tile.  The
//     tiles of all (sequence, kv head, head tile) pairs form one list; every block takes an equal, contiguous range of it and
//     every warp an equal part of that, whatever the sequences' lengths.  A warp walks its range alone: a ring of its own in
//     shared memory, filled with 16-byte asynchronous copies ST - 1 tiles ahead (across pair boundaries), no barrier.
//     Where the range leaves a pair the pair's result is finished, or left as a partial one if other warps share the pair;
//     those of one block meet in shared memory at the end, those of several blocks in kl_paged_merge_kernel.
//   * Mathematics: sums of 2^(s - m) per head, s = q . k * scale * log2(e), m a reference that follows the maximum: it is
//     raised (and the sums rescaled) only when a score exceeds it by more than 8, so that most tiles pass without an
//     exchange between lanes.  Positions are the 16 rows of mma.m16n8k16, the heads its eight columns:
//     S[pos, head] = K . Q^T, O^T[d, head] += V^T . P; P leaves the score accumulators in 16-bit pairs and reaches the
//     layout of a B operand with one movmatrix per 8 x 8 block.  What rounding p to 16 bits leaves of it (and, with fp32
//     queries: EX, what it leaves of q) enters as a second product, and, where the 16 bits are bf16, what that leaves as a
//     third: 22 bits with an e4m3 cache (two f16), 24 with a bf16 one.  The second product costs e4m3 caches 2 % of the time,
//     the third one bf16 caches 0.5 % (fp32 queries 2 %; of a short call 0.2 and 0.7 us).
//   * The matrix instruction cuts its sums off to 32 bits instead of rounding them, always towards zero.  With a bf16 cache the
//     products of 16 positions are therefore summed by themselves and added to the result by an ordinary addition: relative error
//     against 64 bits, fp32 queries, 16 sequences of 65536: 2.0e-6 (2.0e-5 without), for 1 % of the time.  e4m3 caches, whose rows
//     have three fraction bits, go without (4e-6 for 32 of 65536; instructions are what bounds them).
//   * e4m3 rows become f16 (exact) on the way to the tensor cores.  Their scales are powers of two: 2^(e_k - 127) multiplies
//     the score, 2^(e_v - 127) the probability.  The weighted probabilities w = p * 2^(e_v - 127) have a reference of
//     their own, so that f16 holds them whatever the scales (w * 2^7 at most 2^15).
//   * Pages are looked up in units of UR rows (16 where the page size is a multiple of 16, else 4), one per lane, a batch of
//     32 ahead of the copies.
// What bounds it: bf16 caches, memory (32 x 4096 positions, 537 MB: 91.8 us, 91 % of the copy rate; fp32 queries 97.9); e4m3 caches,
// half memory and half instructions (32 sequences, 433 thousand positions, eight query heads per kv head, 894 MB: 161.5 us, 86 %: of some
// 800 instructions per 32 positions the conversions to f16 are a quarter); short calls, latency (1 x 333 positions: 9.1 us --
// launch and the prefix of the lengths, look-ups, first rows and joining one after another, each a microsecond or two); more
// than eight query heads per kv head, the cache read once per eight (16: 32 x 4096 bf16 176 us, e4m3 107 against 56).
template <int HD, bool FP8, int UR, bool EX>
__global__ void __launch_bounds__(PaCfg<HD, FP8, EX>::NW * 32, 1) kl_paged_attn_kernel(const PagedView c, const PagedAttn a) {
    using Cfg = PaCfg<HD, FP8, EX>;
    constexpr int NW = Cfg::NW, ST = Cfg::ST, ROW = Cfg::ROW, TILE = Cfg::TILE, NT = NW * 32;
    constexpr uint32_t TP = Cfg::TP, UPT = TP / UR;              // positions and page look-ups per tile
    constexpr int EXB = 2 * TP, LPN = TP / 4;                    // scale bytes (K, V) and unit positions per tile
    constexpr int NS = TP / 16;                                  // MMA steps of 16 positions per tile
    constexpr uint32_t TPB = 32 / UPT;                           // tiles per batch of look-ups
    constexpr int CPR = ROW / 16, RPP = 32 / CPR;                // 16-byte pieces per row, rows per pass of a warp
    constexpr int NMMA = HD / 16;                                // k steps of a score, m tiles of the result
    extern __shared__ __align__(128) uint8_t pa_smem[];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, g = lane >> 2, j = lane & 3u;
    uint8_t* exps_all = pa_smem + (size_t)NW * ST * 2 * TILE;
    uint32_t* lps_all = reinterpret_cast<uint32_t*>(exps_all + (size_t)NW * ST * EXB);
    float2* ml_all = reinterpret_cast<float2*>(lps_all + NW * ST * LPN);          // [NW][8]
    uint64_t* pre = reinterpret_cast<uint64_t*>(ml_all + NW * 8);               // [NT]
    uint32_t* lens = reinterpret_cast<uint32_t*>(pre + 512);                    // [PA_LENS]
    uint32_t* misc = lens + PA_LENS;
    uint64_t* wsum = reinterpret_cast<uint64_t*>(misc);                         // [NW], then the entries below
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;

    // ---- the list of tiles: prefix sums over the sequences
    const uint32_t PH = c.nkv * a.HT, n = c.n_seqs, per = (n + NT - 1u) / NT;   // per: see pg_prefix
    const uint64_t W = pg_prefix<NW>(n, pre, wsum, [&](uint32_t s) {
        const uint32_t len = pg_length(c, s);
        if (s < (uint32_t)PA_LENS) lens[s] = len;
        return (uint64_t)pa_seq<TP>(c, a, len).nt * PH;
    });
    auto length = [&](uint32_t s) { return s < (uint32_t)PA_LENS ? lens[s] : pg_length(c, s); };

    for (uint32_t s = blockIdx.x; s < n; s += gridDim.x)   // sequences without a position: zeros
        if (length(s) == 0u) {
            for (uint32_t i = tid; i < a.nq * (HD / 2); i += NT) pa_store2(c, a, s, i / (HD / 2), i % (HD / 2) * 2u, 0.f, 0.f);
            for (uint32_t i = tid; i < a.nq; i += NT) pa_store_lse(a, s, i, 0.f, 0.f);
        }

    const uint32_t blocks = (uint32_t)min((uint64_t)gridDim.x, (W + PA_MIN_TILES - 1u) / PA_MIN_TILES);   // blocks at work
    if (blockIdx.x >= blocks) {
        if (tid == 0u && !a.whole_pairs) a.meta[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    // block b takes tiles [share * b + min(b, over), ...): the first `over` blocks one more than the others
    const uint64_t share = pg_div(W, blocks), over = W - share * blocks;
    uint64_t b_lo = share * blockIdx.x + min((uint64_t)blockIdx.x, over), b_n = share + (blockIdx.x < over ? 1u : 0u);
    if (a.whole_pairs) {   // both ends move up to the start of a pair
        auto up = [&](uint64_t x) {
            if (x >= W) return W;
            const uint32_t i = pg_find<NW>(pre, x);
            uint64_t rem = x - pre[i];
            uint32_t s = i * per, nt = pa_seq<TP>(c, a, length(s)).nt;
            while (rem >= (uint64_t)nt * PH) {
                rem -= (uint64_t)nt * PH;
                nt = pa_seq<TP>(c, a, length(++s)).nt;
            }
            const uint32_t into = (uint32_t)(rem - pg_div(rem, nt) * nt);
            return into ? x + nt - into : x;
        };
        const uint64_t to = up(b_lo + b_n);
        b_lo = up(b_lo);
        b_n = to - b_lo;
        if (b_n == 0u) return;
    }
    const uint64_t w_n = pg_div(b_n, NW), w_over = b_n - w_n * NW;
    const uint64_t lo = b_lo + w_n * warp + min((uint64_t)warp, w_over), hi = lo + w_n + (warp < w_over ? 1u : 0u);

    // ---- this warp's range
    struct Entry { uint32_t valid, s, ph, begins, ends; } first = {0, 0, 0, 0, 0}, last = {0, 0, 0, 0, 0};
    uint32_t last_tiles = 0;
    const uint32_t ring = smem_u32(pa_smem) + warp * (ST * 2 * TILE);
    const uint32_t exps = smem_u32(exps_all) + warp * (ST * EXB);
    volatile uint32_t* lps = lps_all + warp * (ST * LPN);
    if (lo < hi) {
        const uint32_t i0 = pg_find<NW>(pre, lo);
        uint64_t rem = lo - pre[i0];
        uint32_t cs = i0 * per;                    // cursor of the tiles that are consumed
        PaSeq cq = pa_seq<TP>(c, a, length(cs));
        while (rem >= (uint64_t)cq.nt * PH) {
            rem -= (uint64_t)cq.nt * PH;
            cq = pa_seq<TP>(c, a, length(++cs));
        }
        uint32_t cph = (uint32_t)pg_div(rem, cq.nt), ct = (uint32_t)(rem - (uint64_t)cph * cq.nt);

        // cursor of the tiles that are requested, and the look-ups of its batch (this one and the next)
        uint32_t is = cs, iph = cph, it = ct;
        PaSeq iq = cq;
        uint32_t batch = 0xffffffffu;
        const uint8_t *ik, *iv;   // the pair's head in page 0, this lane's piece of a row; and its scales
        int64_t ie;
        auto aim = [&]() {
            const uint32_t h = iph / a.HT;
            ik = c.k + (int64_t)h * c.head_b + lane % CPR * 16u;
            iv = c.v + (int64_t)h * c.head_b + lane % CPR * 16u;
            ie = (int64_t)h * c.page;
        };
        aim();
        int32_t b_phys = -1, n_phys = -1;
        uint32_t b_lp = PA_NONE, n_lp = PA_NONE, b_row = 0, n_row = 0;
        auto look_up = [&](uint32_t b, int32_t& phys, uint32_t& lp, uint32_t& row) {   // unit `lane` of batch b
            phys = -1;
            lp = PA_NONE;
            row = 0;
            const uint32_t u = (iq.t0 + b * TPB) * UPT + lane;
            uint32_t logical;
            if (a.selected) {
                const uint32_t upp = c.page / UR, e = u / upp;
                if (e >= iq.listed) return;
                const int32_t sel = a.selected[((size_t)is * c.nkv + iph / a.HT) * a.n_select + e];
                if (sel < 0 || (uint64_t)sel * c.page >= iq.len) return;
                logical = (uint32_t)sel;
                row = (u - e * upp) * UR;
            } else {
                if ((uint64_t)u * UR >= iq.len) return;
                logical = u * UR / c.page;
                row = u * UR - logical * c.page;
            }
            if (logical * c.page + row + UR <= iq.lo) return;   // before the window: the page may be gone
            phys = pg_physical(c, is, logical);
            if (phys >= 0) lp = logical * c.page + row;
        };
        uint64_t left = hi - lo;   // tiles still to request
        uint32_t whole = 0;        // ring slots whose tile has no position that does not count
        // Where a row's 16-byte pieces lie in its tile: piece ch of row r at ch ^ fk(r) (K) or ch ^ fv(r) (V), so that the pieces
        // a warp reads together fall into different banks.  A lane copies piece ch of rows r0, r0 + RPP, ...
        const uint32_t ch = lane % CPR, r0 = lane / CPR;
        const int64_t e_page = (int64_t)c.nkv * c.page;   // scales of a page
        auto fk_of = [](uint32_t r) { return CPR >= 8 ? ((r & 1u) << 2 | ((r >> 1) & 3u)) : 0u; };
        auto fv_of = [](uint32_t r) { return CPR < 8 ? ((r >> 1) & 3u) : FP8 ? (r & 7u) : ((r & 1u) << 2 | ((r >> 1) & 3u)); };
        constexpr int NPAT = RPP >= 8 ? 1 : 8 / RPP;   // the pattern repeats every eight rows
        uint32_t k_at[NPAT], v_at[NPAT];
#pragma unroll
        for (int i = 0; i < NPAT; ++i) {
            k_at[i] = r0 * ROW + ((ch ^ fk_of(i * RPP + r0)) << 4);
            v_at[i] = r0 * ROW + ((ch ^ fv_of(i * RPP + r0)) << 4);
        }
        auto issue = [&](uint32_t st) {
            const uint32_t b = it / TPB, at = it - b * TPB;
            if (b != batch) {   // this batch, unless it has been looked up already, and the next one
                const bool known = batch != 0xffffffffu;
                b_phys = n_phys; b_lp = n_lp; b_row = n_row;
#pragma unroll 1
                for (uint32_t x = known ? b + 1u : b; x <= b + 1u && x * TPB < iq.nt; ++x) {
                    look_up(x, n_phys, n_lp, n_row);
                    if (x == b) { b_phys = n_phys; b_lp = n_lp; b_row = n_row; }
                }
                batch = b;
            }
            const uint32_t kd = ring + st * (2 * TILE), vd = kd + TILE;
            bool full = true;   // every position of the tile counts
#pragma unroll
            for (uint32_t v = 0; v < UPT; v += UR == 16 ? 1 : UPT) {   // UR == 16: unit after unit; UR == 4: the lanes' units at once
                if (UR == 16) {
                    const int32_t phys = __shfl_sync(0xffffffffu, b_phys, at * UPT + v);
                    const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, at * UPT + v), row = __shfl_sync(0xffffffffu, b_row, at * UPT + v);
                    const int32_t r_lo = (int32_t)iq.lo - (int32_t)lp, r_hi = (int32_t)iq.len - (int32_t)lp;   // rows of the unit that count
                    full = full && r_lo <= 0 && r_hi >= 16;
                    const int64_t off = (int64_t)max(phys, 0) * c.page_b + (int64_t)(row + r0) * c.row_b;
                    const uint8_t *ks = ik + off, *vs = iv + off;
                    if (r_lo <= 0 && r_hi >= 16 && c.row_b == ROW) {   // the usual unit: 16 rows in a row, all of which count
#pragma unroll
                        for (int i = 0; i < 16 / RPP; ++i) {
                            pa_copy16(kd + k_at[i % NPAT] + (v * 16 + i * RPP) * ROW, ks + i * RPP * ROW);
                            pa_copy16(vd + v_at[i % NPAT] + (v * 16 + i * RPP) * ROW, vs + i * RPP * ROW);
                        }
                    } else {
#pragma unroll 1
                        for (int i = 0; i < 16 / RPP; ++i) {
                            const int32_t r = i * RPP + (int32_t)r0;
                            const bool ok = r >= r_lo && r < r_hi;
                            pa_copy16(kd + (v * 16 + r) * ROW + ((ch ^ fk_of(r)) << 4), ks, ok);
                            pa_copy16(vd + (v * 16 + r) * ROW + ((ch ^ fv_of(r)) << 4), vs, ok);
                            ks += (int64_t)RPP * c.row_b;
                            vs += (int64_t)RPP * c.row_b;
                        }
                    }
                    if (FP8 && lane < 2u) {
                        const int64_t eoff = (int64_t)max(phys, 0) * e_page + ie + row;
                        pa_copy16(exps + st * EXB + lane * TP + v * 16, (lane ? c.ve : c.ke) + eoff, phys >= 0);
                    }
                    if (lane == 0u) lps[st * LPN + v] = lp;
                } else {
#pragma unroll
                    for (int i = 0; i < (int)TP / RPP; ++i) {
                        const int32_t r = i * RPP + (int32_t)r0;
                        const uint32_t src = at * UPT + (r >> 2);
                        const int32_t phys = __shfl_sync(0xffffffffu, b_phys, src);
                        const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, src), row = __shfl_sync(0xffffffffu, b_row, src);
                        const int32_t p = (int32_t)lp + (r & 3);
                        const bool ok = lp != PA_NONE && p >= (int32_t)iq.lo && p < (int32_t)iq.len;
                        const int64_t off = (int64_t)max(phys, 0) * c.page_b + (int64_t)(row + (r & 3)) * c.row_b;
                        pa_copy16(kd + r * ROW + ((ch ^ fk_of(r)) << 4), ik + off, ok);
                        pa_copy16(vd + r * ROW + ((ch ^ fv_of(r)) << 4), iv + off, ok);
                    }
                    const uint32_t u = lane % UPT, src = at * UPT + u;
                    const int32_t phys = __shfl_sync(0xffffffffu, b_phys, src);
                    const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, src), row = __shfl_sync(0xffffffffu, b_row, src);
                    if (FP8 && lane < 2u * UPT) {
                        const int64_t eoff = (int64_t)max(phys, 0) * e_page + ie + row;
                        pa_copy4(exps + st * EXB + lane / UPT * TP + u * 4, (lane < UPT ? c.ke : c.ve) + eoff, phys >= 0);
                    }
                    if (lane < UPT) lps[st * LPN + lane] = lp;
                    full = __all_sync(0xffffffffu, lp != PA_NONE && lp >= iq.lo && lp + UR <= iq.len);
                }
            }
            whole = full ? whole | 1u << st : whole & ~(1u << st);
            --left;
            if (++it == iq.nt && left) {   // on to the next pair, perhaps of the next sequence that has any
                it = 0;
                batch = 0xffffffffu;
                if (++iph == PH) {
                    iph = 0;
                    do iq = pa_seq<TP>(c, a, length(++is));
                    while (iq.nt == 0u);
                }
                aim();
            }
        };
        // ---- state of the pair under way.  Queries: head g; scores and results: heads 2j and 2j + 1
        constexpr bool THIRD = EX && !FP8;
        uint32_t qh[NMMA][2], ql[EX ? NMMA : 1][2], qm[THIRD && !Cfg::QM ? NMMA : 1][2];
        uint2* qm_s = reinterpret_cast<uint2*>(misc + 64) + warp * (NMMA * 32) + lane;   // (Cfg::QM)
        float o[NMMA][4], m[2], l[2], mw[2], qs[2];
        constexpr int PIECE = FP8 ? 16 : 8;   // consecutive columns of a lane per 16-byte piece of a row
        uint32_t raw[NMMA][EX ? 4 : 2];       // the lane's columns of query head g, as they lie in memory
        auto load_queries = [&]() {
            const uint32_t h = cph / a.HT, hg = (cph - h * a.HT) * 8u + g;
            const uint8_t* q = a.q + (int64_t)cs * a.q_stride + (size_t)(h * a.G + hg) * HD * (EX ? 4 : 2);
#pragma unroll
            for (int i = 0; i < NMMA; ++i) {
                const uint32_t d = (i / (PIECE / 4)) * (4 * PIECE) + j * PIECE + (i % (PIECE / 4)) * 4;
#pragma unroll
                for (int e = 0; e < (EX ? 4 : 2); ++e) raw[i][e] = 0u;
                if (hg < a.G) {
                    if (EX) {
                        const uint4 f = *reinterpret_cast<const uint4*>(q + d * 4);
                        raw[i][0] = f.x; raw[i][1] = f.y; raw[i][EX ? 2 : 0] = f.z; raw[i][EX ? 3 : 0] = f.w;
                    } else {
                        const uint2 f = *reinterpret_cast<const uint2*>(q + d * 2);
                        raw[i][0] = f.x; raw[i][1] = f.y;
                    }
                }
            }
        };
        auto begin_pair = [&]() {
            float x[NMMA][4], big = 0.f;
#pragma unroll
            for (int i = 0; i < NMMA; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[i][e] = EX ? __uint_as_float(raw[i][e % (EX ? 4 : 2)]) : e & 1 ? bf_hi(raw[i][e / 2]) : bf_lo(raw[i][e / 2]);
                    if (FP8) big = fmaxf(big, fabsf(x[i][e]));
                }
            float mul = a.scale_log2, f = 1.f;
            if (FP8) {   // f16 operands: the head's largest query element comes to lie in [2^14, 2^15)
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const int32_t k = max((int32_t)(__float_as_uint(big) >> 23) - 127, -112);
                f = __uint_as_float((uint32_t)(127 + 14 - k) << 23);
                mul *= __uint_as_float((uint32_t)(127 - 14 + k) << 23);
            }
            qs[0] = __shfl_sync(0xffffffffu, mul, j * 8u);
            qs[1] = __shfl_sync(0xffffffffu, mul, j * 8u + 4u);
#pragma unroll
            for (int i = 0; i < NMMA; ++i) {
                uint32_t third[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x0 = x[i][2 * e] * f, x1 = x[i][2 * e + 1] * f;
                    qh[i][e] = pa_round<FP8>(x0, x1);
                    if (EX) ql[i % (EX ? NMMA : 1)][e] = pa_rest<FP8>(x0, x1, qh[i][e]);
                    if (THIRD) third[e] = pa_rest2(x0, x1, qh[i][e], ql[i % (EX ? NMMA : 1)][e]);
                }
                if (Cfg::QM) {
                    qm_s[i * 32] = make_uint2(third[0], third[1]);
                } else if (THIRD) {
                    qm[i % (THIRD && !Cfg::QM ? NMMA : 1)][0] = third[0];
                    qm[i % (THIRD && !Cfg::QM ? NMMA : 1)][1] = third[1];
                }
            }
#pragma unroll
            for (int i = 0; i < NMMA; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
            m[0] = m[1] = mw[0] = mw[1] = -INFINITY;
            l[0] = l[1] = 0.f;
        };
        // The pair's result over the tiles seen: emit(x, d, v0, v1) gets columns d and d + 1 (e4m3), or d and d + 8 (bf16), of
        // head 2j + x; the sums themselves, relative to 2^m, or divided by l.
        auto end_pair = [&](bool divide, auto&& emit) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int k = 4; k < 32; k <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], k);
                float f = !FP8 ? 1.f : mw[x] == -INFINITY ? 0.f : pa_ex2(mw[x] - m[x] - 7.f);
                if (divide) f = l[x] == 0.f ? 0.f : f / l[x];
                constexpr int W16 = HD >= 128 ? 16 : 8;   // columns of a lane's V piece (e4m3)
#pragma unroll
                for (int i = 0; i < NMMA; ++i) {
                    const uint32_t d = FP8 ? (2 * i / W16) * (8 * W16) + g * W16 + 2 * i % W16 : i * 16 + g;
                    emit(x, d, o[i][x] * f, o[i][x + 2] * f);
                }
            }
        };

        const uint32_t total = (uint32_t)(hi - lo);   // a warp's share (2^32 tiles would be hours of work)
        uint32_t seg0 = ct;                           // first tile of the pair that this warp has seen
        bool fresh = true;                            // the next tile starts a pair
        uint32_t to = 0;                              // ring slot of the next request
        uint32_t k = 0, st = 0;                       // tile of the range, and its slot
        load_queries();
        for (uint32_t ahead = 0; k < total;) {
            if (ahead >= (uint32_t)ST - 1u) {
                if (fresh) {   // while the tile is on its way
                    if (k) load_queries();
                    begin_pair();
                    fresh = false;
                }
                asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
                __syncwarp();   // the tile is there for every lane, and every lane is done with the previous one
            }
            if (left) issue(to);
            if (++to == (uint32_t)ST) to = 0;
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (ahead < (uint32_t)ST - 1u) {   // the first ST - 1 tiles are only requested
                ++ahead;
                continue;
            }
            const uint32_t kd = ring + st * (2 * TILE), vd = kd + TILE;
            // scores: s[2x + e] is that of position 8x + g and head 2j + e
            float sc[NS][4], s[4 * NS], sv[4 * NS];
#pragma unroll
            for (int t = 0; t < NS; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
            const uint32_t fk = CPR >= 8 ? ((g & 1u) << 2 | ((g >> 1) & 3u)) : 0u;
#pragma unroll
            for (int q = 0; q < CPR / 4; ++q)
#pragma unroll
                for (int t = 0; t < NS; ++t) {
                    const uint32_t at = kd + (t * 16 + g) * ROW + (((q * 4 + j) ^ fk) << 4);
                    const uint4 w = pa_lds16(at), y = pa_lds16(at + 8 * ROW);   // rows g and g + 8: the same swizzle
                    const uint32_t wa[4] = {w.x, w.y, w.z, w.w}, ya[4] = {y.x, y.y, y.z, y.w};
                    if (FP8) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t a0 = pg_e4m3x2_to_f16x2(wa[x] & 0xffffu), a1 = pg_e4m3x2_to_f16x2(ya[x] & 0xffffu);
                            const uint32_t a2 = pg_e4m3x2_to_f16x2(wa[x] >> 16), a3 = pg_e4m3x2_to_f16x2(ya[x] >> 16);
                            const int i = (q * 4 + x) % NMMA;
                            pa_mma<FP8>(sc[t], a0, a1, a2, a3, qh[i][0], qh[i][1]);
                            if (EX) pa_mma<FP8>(sc[t], a0, a1, a2, a3, ql[i % (EX ? NMMA : 1)][0], ql[i % (EX ? NMMA : 1)][1]);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int i = (q * 2 + x) % NMMA;
                            pa_mma<FP8>(sc[t], wa[2 * x], ya[2 * x], wa[2 * x + 1], ya[2 * x + 1], qh[i][0], qh[i][1]);
                            if (EX) pa_mma<FP8>(sc[t], wa[2 * x], ya[2 * x], wa[2 * x + 1], ya[2 * x + 1], ql[i % (EX ? NMMA : 1)][0], ql[i % (EX ? NMMA : 1)][1]);
                            if (THIRD) {
                                uint2 w3 = make_uint2(qm[i % (THIRD && !Cfg::QM ? NMMA : 1)][0], qm[i % (THIRD && !Cfg::QM ? NMMA : 1)][1]);
                                if (Cfg::QM) w3 = qm_s[i * 32];   // the lane's own
                                pa_mma<FP8>(sc[t], wa[2 * x], ya[2 * x], wa[2 * x + 1], ya[2 * x + 1], w3.x, w3.y);
                            }
                        }
                    }
                }
#pragma unroll
            for (int x = 0; x < 2 * NS; ++x) {
                float f0 = qs[0], f1 = qs[1], ev = 0.f;
                if (FP8) {
                    uint32_t ke, ve;
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ke) : "r"(exps + st * EXB + x * 8 + g));
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ve) : "r"(exps + st * EXB + TP + x * 8 + g));
                    f0 *= pg_scale(ke);
                    f1 *= pg_scale(ke);
                    ev = (float)(int)ve - 127.f;
                }
                s[2 * x] = sc[x / 2][x % 2 * 2] * f0;
                s[2 * x + 1] = sc[x / 2][x % 2 * 2 + 1] * f1;
                if (FP8) sv[2 * x] = sv[2 * x + 1] = ev;
            }
            if (!(whole >> st & 1u)) {   // positions that do not count
#pragma unroll
                for (int x = 0; x < 2 * NS; ++x) {
                    const uint32_t r = x * 8 + g, lp = lps[st * LPN + r / UR], p = lp + r % UR;
                    if (lp == PA_NONE || p < cq.lo || p >= cq.len) s[2 * x] = s[2 * x + 1] = -INFINITY;
                }
            }
            float mx[2] = {s[0], s[1]}, mv[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 2; i < 4 * NS; ++i) mx[i & 1] = fmaxf(mx[i & 1], s[i]);
            if (FP8)
#pragma unroll
                for (int i = 0; i < 4 * NS; ++i) {
                    sv[i] += s[i];
                    mv[i & 1] = fmaxf(mv[i & 1], sv[i]);
                }
            bool high = mx[0] > m[0] + 8.f || mx[1] > m[1] + 8.f;
            if (FP8) high = high || mv[0] > mw[0] + 8.f || mv[1] > mw[1] + 8.f;
            if (__any_sync(0xffffffffu, high)) {   // raise the references to the maxima seen
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) {
                        mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], k));
                        if (FP8) mv[x] = fmaxf(mv[x], __shfl_xor_sync(0xffffffffu, mv[x], k));
                    }
                    const float mn = fmaxf(m[x], mx[x]), f = mn == m[x] ? 1.f : pa_ex2(m[x] - mn);
                    m[x] = mn;
                    l[x] *= f;
                    float fo = f;
                    if (FP8) {
                        const float wn = fmaxf(mw[x], mv[x]);
                        fo = wn == mw[x] ? 1.f : pa_ex2(mw[x] - wn);
                        mw[x] = wn;
                    }
#pragma unroll
                    for (int i = 0; i < NMMA; ++i) {
                        o[i][x] *= fo;
                        o[i][x + 2] *= fo;
                    }
                }
            }
            float p[4 * NS];
            {
                const float mu[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
                const float wu[2] = {mw[0] == -INFINITY ? 0.f : mw[0] - 7.f, mw[1] == -INFINITY ? 0.f : mw[1] - 7.f};
#pragma unroll
                for (int i = 0; i < 4 * NS; ++i) {
                    p[i] = pa_ex2(s[i] - mu[i & 1]);
                    l[i & 1] += p[i];
                    if (FP8) p[i] = pa_ex2(sv[i] - wu[i & 1]);
                }
            }
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const uint32_t h0 = pa_round<FP8>(p[4 * t], p[4 * t + 1]), h1 = pa_round<FP8>(p[4 * t + 2], p[4 * t + 3]);
                const uint32_t b0 = movmatrix_trans(h0), b1 = movmatrix_trans(h1);
                const uint32_t l0 = pa_rest<FP8>(p[4 * t], p[4 * t + 1], h0), l1 = pa_rest<FP8>(p[4 * t + 2], p[4 * t + 3], h1);
                const uint32_t c0 = movmatrix_trans(l0), c1 = movmatrix_trans(l1);
                const uint32_t vs = vd + t * 16 * ROW;
                if (FP8) {
                    constexpr int VW = HD >= 128 ? 4 : 2;            // words of a lane's piece of a row
#pragma unroll
                    for (int hh = 0; hh < HD / (32 * VW); ++hh) {
                        uint32_t r[4][4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {                // rows 2j, 2j + 1, 2j + 8, 2j + 9
                            const uint32_t row = 2 * j + (x & 1) + (x >> 1) * 8;
                            if (VW == 4) {
                                const uint4 w = pa_lds16(vs + row * ROW + (((hh * 8 + g) ^ (row & 7u)) << 4));
                                r[x][0] = w.x; r[x][1] = w.y; r[x][2] = w.z; r[x][3] = w.w;
                            } else {
                                const uint2 w = pa_lds8(vs + row * ROW + (((g >> 1) ^ ((row >> 1) & 3u)) << 4) + (g & 1u) * 8u);
                                r[x][0] = w.x; r[x][1] = w.y;
                            }
                        }
#pragma unroll
                        for (int w = 0; w < VW; ++w) {
                            const uint32_t a01 = __byte_perm(r[0][w], r[1][w], 0x5140), a23 = __byte_perm(r[0][w], r[1][w], 0x7362);
                            const uint32_t b01 = __byte_perm(r[2][w], r[3][w], 0x5140), b23 = __byte_perm(r[2][w], r[3][w], 0x7362);
                            float (*oo)[4] = o + hh * 8 + w * 2;
                            const uint32_t x0 = pg_e4m3x2_to_f16x2(a01 & 0xffffu), x1 = pg_e4m3x2_to_f16x2(a01 >> 16);
                            const uint32_t x2 = pg_e4m3x2_to_f16x2(b01 & 0xffffu), x3 = pg_e4m3x2_to_f16x2(b01 >> 16);
                            const uint32_t y0 = pg_e4m3x2_to_f16x2(a23 & 0xffffu), y1 = pg_e4m3x2_to_f16x2(a23 >> 16);
                            const uint32_t y2 = pg_e4m3x2_to_f16x2(b23 & 0xffffu), y3 = pg_e4m3x2_to_f16x2(b23 >> 16);
                            pa_mma<FP8>(oo[0], x0, x1, x2, x3, b0, b1);
                            pa_mma<FP8>(oo[1], y0, y1, y2, y3, b0, b1);
                            pa_mma<FP8>(oo[0], x0, x1, x2, x3, c0, c1);
                            pa_mma<FP8>(oo[1], y0, y1, y2, y3, c0, c1);
                        }
                    }
                } else {
                    const uint32_t e0 = movmatrix_trans(pa_rest2(p[4 * t], p[4 * t + 1], h0, l0));
                    const uint32_t e1 = movmatrix_trans(pa_rest2(p[4 * t + 2], p[4 * t + 3], h1, l1));
                    // matrices of a load: positions 0..7 and 8..15 of two neighbouring pieces of eight columns
                    const uint32_t row = (lane >> 4) * 8u + (lane & 7u), base = vs + row * ROW, fv = (row & 1u) << 2 | ((row >> 1) & 3u);
#pragma unroll
                    for (int i = 0; i < NMMA; ++i) {
                        uint32_t r[4];
                        ldmatrix_x4_trans(r, base + (((i * 2 + (lane >> 3 & 1u)) ^ fv) << 4));
                        float sum[4] = {0.f, 0.f, 0.f, 0.f};
                        pa_mma<FP8>(sum, r[0], r[1], r[2], r[3], e0, e1);
                        pa_mma<FP8>(sum, r[0], r[1], r[2], r[3], c0, c1);
                        pa_mma<FP8>(sum, r[0], r[1], r[2], r[3], b0, b1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i][e] += sum[e];
                    }
                }
            }
            if (++st == ST) st = 0;

            ++ct;
            if (ct == cq.nt || k + 1u == total) {   // the pair ends here, for this warp at least
                const uint32_t h = cph / a.HT, hg = (cph - h * a.HT) * 8u + 2u * j, hq = h * a.G + hg;
                const bool tail = k + 1u == total;
                if (seg0 == 0u && ct == cq.nt) {
                    end_pair(true, [&](int x, uint32_t d, float v0, float v1) {
                        if (hg + x >= a.G) return;
                        if (FP8) {
                            pa_store2(c, a, cs, hq + x, d, v0, v1);
                        } else {
                            pa_store1(c, a, cs, hq + x, d, v0);
                            pa_store1(c, a, cs, hq + x, d + 8u, v1);
                        }
                    });
                    if (g == 0u && a.lse)
                        for (int x = 0; x < 2; ++x)
                            if (hg + x < a.G) pa_store_lse(a, cs, hq + x, m[x], l[x]);
                } else {
                    Entry& e = tail ? last : first;
                    e = {1u, cs, cph, seg0 == 0u, ct == cq.nt};
                    float* dst = a.head + ((size_t)blockIdx.x * NW + warp) * 8 * HD;
                    float2* ml = reinterpret_cast<float2*>(a.head_ml) + ((size_t)blockIdx.x * NW + warp) * 8;
                    if (tail) {   // the ring has been read to the end
                        asm volatile("cp.async.wait_group 0;" ::: "memory");
                        __syncwarp();
                        dst = reinterpret_cast<float*>(pa_smem + warp * (ST * 2 * TILE));
                        ml = ml_all + warp * 8;
                    }
                    end_pair(false, [&](int x, uint32_t d, float v0, float v1) {
                        float* to = dst + (2 * j + x) * HD + d;
                        if (FP8) {
                            *reinterpret_cast<float2*>(to) = make_float2(v0, v1);
                        } else {
                            to[0] = v0;
                            to[8] = v1;
                        }
                    });
                    if (g == 0u) {
                        ml[2 * j] = make_float2(m[0], l[0]);
                        ml[2 * j + 1] = make_float2(m[1], l[1]);
                    }
                }
                if (!tail) {
                    ct = seg0 = 0;
                    fresh = true;
                    if (++cph == PH) {
                        cph = 0;
                        do cq = pa_seq<TP>(c, a, length(++cs));
                        while (cq.nt == 0u);
                    }
                }
            }
            ++k;
        }
        if (last.valid) last_tiles = cq.nt - ct;   // tiles of its last pair that lie in later ranges
    }

    // ---- the partial results of this block's warps, in the order of the list: first[0], last[0], first[1], ...
    __syncthreads();   // everyone is done with the lengths
    uint4* ent = reinterpret_cast<uint4*>(lens);   // [2 NW]: (valid | begins << 1 | ends << 2, s, ph, tiles in later ranges)
    if (lane < 2u) {
        const Entry e = lane ? last : first;
        ent[2 * warp + lane] = make_uint4(e.valid | e.begins << 1 | e.ends << 2, e.s, e.ph, lane ? last_tiles : 0u);
    }
    __threadfence_block();   // the first results lie in global memory
    __syncthreads();
    // lane e of every warp holds entry e; runs of valid entries of the same pair start at the bits of `starts`
    const uint4 mine_e = lane < 2u * NW ? ent[lane] : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t valid = __ballot_sync(0xffffffffu, mine_e.x & 1u), below = valid & ((1u << lane) - 1u);
    const int prev = below ? 31 - __clz(below) : 0;
    const uint32_t ps = __shfl_sync(0xffffffffu, mine_e.y, prev), pph = __shfl_sync(0xffffffffu, mine_e.z, prev);
    const uint32_t starts = __ballot_sync(0xffffffffu, (mine_e.x & 1u) && (!below || ps != mine_e.y || pph != mine_e.z));
    int4 meta = make_int4(0, 0, 0, 0);
    for (uint32_t rest = starts; rest; rest &= rest - 1u) {
        const int e0 = __ffs(rest) - 1;
        const uint32_t after = rest & (rest - 1u);
        const uint32_t mask = valid & ~((1u << e0) - 1u) & (after ? (1u << (__ffs(after) - 1)) - 1u : 0xffffffffu);
        const int e1 = 31 - __clz(mask);   // the run: bits e0 .. e1 of mask
        const uint4 head = ent[e0], end = ent[e1];
        const uint32_t s = head.y, ph = head.z, h = ph / a.HT, h0 = (ph - h * a.HT) * 8u;
        const bool begins = head.x & 2u, whole = begins && (end.x & 4u);
        const size_t slot = (size_t)blockIdx.x * 2 + (begins ? 1 : 0);
        if (begins && !whole && tid == 0u) {   // the last block that shares the pair: the one that holds its last tile
            const uint64_t last_tile = b_lo + b_n - 1u + end.w;
            const uint64_t wide = (share + 1u) * over;
            const uint64_t lb = last_tile < wide ? pg_div(last_tile, (uint32_t)share + 1u) : over + pg_div(last_tile - wide, (uint32_t)share);
            meta = make_int4(1, (int)s, (int)ph, (int)lb);
        }
        const uint32_t heads = min(8u, a.G - h0);
        for (uint32_t i = tid; i < heads * (HD / 2); i += NT) {
            const uint32_t hh = i / (HD / 2), d = i % (HD / 2) * 2u;
            // the run: last[wa] .. last[wb], and first[wb + 1] where that warp goes on to another pair
            float2 ml[NW], mf = make_float2(-INFINITY, 0.f);
            float M = -INFINITY, L = 0.f, v0 = 0.f, v1 = 0.f;
            const size_t fs = ((size_t)blockIdx.x * NW + e1 / 2) * 8 + hh;
            if (!(e1 & 1)) mf = reinterpret_cast<const float2*>(a.head_ml)[fs];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                ml[w] = mask >> (2 * w + 1) & 1u ? ml_all[w * 8 + hh] : make_float2(-INFINITY, 0.f);
                M = fmaxf(M, ml[w].x);
            }
            M = fmaxf(M, mf.x);
            const float mu = M == -INFINITY ? 0.f : M;
            auto add = [&](float2 x, const float* o) {
                const float2 y = *reinterpret_cast<const float2*>(o);
                const float f = pa_ex2(x.x - mu);
                L += x.y * f;
                v0 += y.x * f;
                v1 += y.y * f;
            };
#pragma unroll
            for (int w = 0; w < NW; ++w)
                if (mask >> (2 * w + 1) & 1u) add(ml[w], reinterpret_cast<const float*>(pa_smem + w * (ST * 2 * TILE)) + hh * HD + d);
            if (!(e1 & 1)) add(mf, a.head + fs * HD + d);
            if (whole) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                pa_store2(c, a, s, h * a.G + h0 + hh, d, v0 * inv, v1 * inv);
                if (d == 0u) pa_store_lse(a, s, h * a.G + h0 + hh, M, L);
            } else {
                *reinterpret_cast<float2*>(a.part + (slot * 8 + hh) * HD + d) = make_float2(v0, v1);
                if (d == 0u) reinterpret_cast<float2*>(a.part_ml)[slot * 8 + hh] = make_float2(M, L);
            }
        }
    }
    if (tid == 0u && !a.whole_pairs) a.meta[blockIdx.x] = meta;
}

// Joins the partial results of the pairs that several blocks of kl_paged_attn_kernel share, in the order of the blocks.
// Block (b, h): head h of the pair that begins in block b and goes on in b + 1, if there is one.  Latency: two rounds of loads,
// about 3 us behind the last block of the attention kernel.  (Joining in the last block to arrive would save a launch, but
// needs counters that start at zero, which no workspace of the caller's guarantees.)
constexpr int PA_MERGE_THREADS = 128;
constexpr int PA_MAX_BLOCKS = 256;
__global__ void __launch_bounds__(PA_MERGE_THREADS) kl_paged_merge_kernel(const PagedView c, const PagedAttn a) {
    __shared__ float2 ml[PA_MAX_BLOCKS];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const int b = (int)blockIdx.x, tid = (int)threadIdx.x;
    const int4 meta = a.meta[b];
    const uint32_t s = (uint32_t)meta.y, ph = (uint32_t)meta.z, h = ph / a.HT, h0 = (ph - h * a.HT) * 8u, hh = blockIdx.y;
    if (!meta.x || h0 + hh >= a.G) return;
    // (a workspace that another call writes meanwhile leads to wrong results, not out of bounds)
    if (s >= c.n_seqs || h >= c.nkv || meta.w < b || meta.w >= (int)gridDim.x) return;
    const int cnt = meta.w - b + 1;   // blocks b .. meta.w
    auto slot = [&](int i) { return i == 0 ? (size_t)b * 2 + 1 : (size_t)(b + i) * 2; };
    for (int i = tid; i < cnt; i += PA_MERGE_THREADS) ml[i] = reinterpret_cast<const float2*>(a.part_ml)[slot(i) * 8 + hh];
    const uint32_t d = 2u * tid, dd = d < c.hd ? d : 0u;
    constexpr int AHEAD = 24;   // records loaded before the maximum is known
    float2 x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < cnt) x[i] = *reinterpret_cast<const float2*>(a.part + (slot(i) * 8 + hh) * c.hd + dd);
    __syncthreads();
    float M = -INFINITY;
#pragma unroll 8
    for (int i = 0; i < cnt; ++i) M = fmaxf(M, ml[i].x);
    const float mu = M == -INFINITY ? 0.f : M;
    float L = 0.f, v0 = 0.f, v1 = 0.f;
    auto add = [&](int i, float2 y) {
        const float f = pa_ex2(ml[i].x - mu);
        L += ml[i].y * f;
        v0 += y.x * f;
        v1 += y.y * f;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        if (i >= cnt) break;
        add(i, x[i]);
    }
#pragma unroll 8
    for (int i = AHEAD; i < cnt; ++i) add(i, *reinterpret_cast<const float2*>(a.part + (slot(i) * 8 + hh) * c.hd + dd));
    if (d >= c.hd) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    pa_store2(c, a, s, h * a.G + h0 + hh, d, v0 * inv, v1 * inv);
    if (d == 0u) pa_store_lse(a, s, h * a.G + h0 + hh, M, L);
}

}  // namespace kl
