// Kernels of the paged key-value cache (contracts in include/kl.h): append with quantisation and page bounds, read back,
// page selection by bounds, attention of one new token over pages.
#pragma once

#include "kl_device.cuh"

#include <cuda_fp16.h>

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

// 2^(e - 127) of a scale byte, and its inverse for the exponents a row can have (e - 127 in [-127, 120]).
__device__ __forceinline__ float pg_scale(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x00400000u); }
__device__ __forceinline__ float pg_inv_scale(int32_t e) { return __uint_as_float((uint32_t)(127 - e) << 23); }

// Scale exponent of a row whose largest finite magnitude is `big`: the smallest e >= -127 with big <= 448 * 2^e.
// big = m * 2^k with m in [1, 2): 448 = 1.75 * 2^8, so e = k - 8, or k - 7 where m > 1.75 (the 23 fraction bits of 1.75
// are 0x600000).  Numbers below 2^-119 all get -127.
__device__ __forceinline__ int32_t pg_exponent(float big) {
    const uint32_t u = __float_as_uint(big);
    const int32_t e = (int32_t)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -127 ? -127 : e;
}

// Two floats to two e4m3 codes (lo in the low byte), nearest even, saturating.
__device__ __forceinline__ uint32_t pg_to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
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

// Eight consecutive elements at src (16-byte aligned) as floats.
template <class T>
__device__ __forceinline__ void pg_load8(const T* src, float (&x)[8]);
template <>
__device__ __forceinline__ void pg_load8<float>(const float* src, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(src)[0], b = reinterpret_cast<const float4*>(src)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <>
__device__ __forceinline__ void pg_load8<__nv_bfloat16>(const __nv_bfloat16* src, float (&x)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(src);
    x[0] = bf_lo(u.x); x[1] = bf_hi(u.x); x[2] = bf_lo(u.y); x[3] = bf_hi(u.y);
    x[4] = bf_lo(u.z); x[5] = bf_hi(u.z); x[6] = bf_lo(u.w); x[7] = bf_hi(u.w);
}
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
// Eight consecutive cached elements of a row (columns col .. col + 7) as floats.
__device__ __forceinline__ void pg_load_cached8(const uint8_t* row, uint32_t col, bool fp8, float scale, float (&x)[8]) {
    if (fp8) {
        const uint2 u = *reinterpret_cast<const uint2*>(row + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(((i < 2 ? u.x : u.y) >> (16 * (i & 1))) & 0xffffu));
            x[2 * i] = f.x * scale;
            x[2 * i + 1] = f.y * scale;
        }
    } else {
        pg_load8<__nv_bfloat16>(reinterpret_cast<const __nv_bfloat16*>(row) + col, x);
    }
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

// Append.  One block = the rows of one call that fall into one page, for one kv head, so that the page's bounds have one
// writer and its rows are quantised where they pass by.  Sequence s touches at most rows / page + 2 pages, so block u of
// the grid belongs to the sequence s with base(s) <= u < base(s + 1), base(s) = row_starts[s] / page + 2 s, and is its
// page number u - base(s) (blocks without a page leave).  hd / 8 lanes share a row, eight columns each; half of the
// lane groups take keys, the other half values.
template <class T>
__global__ void __launch_bounds__(PG_THREADS) kl_paged_append_kernel(const PagedView c, const PagedRows rows) {
    extern __shared__ float pg_red[];   // [groups of K rows][2][hd] when the cache has bounds
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t u = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    uint32_t s, j;
    if (!rows.row_starts) {
        s = u;
        j = 0;
    } else {
        uint32_t lo = 0, hi = c.n_seqs;   // base(lo) <= u < base(hi)
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) / 2u;
            if (pg_row_start(c, rows, mid) / c.page + 2u * mid <= u) lo = mid;
            else hi = mid;
        }
        s = lo;
        j = u - (pg_row_start(c, rows, s) / c.page + 2u * s);
    }
    const uint32_t r0 = pg_row_start(c, rows, s), r1 = pg_row_start(c, rows, s + 1u);
    if (rows.row_starts && j == 0u && tid == 0u) {   // an array that descends or leaves [0, n_rows]
        const int32_t a = rows.row_starts[s], b = rows.row_starts[s + 1u];
        if (a < 0 || b < a || (uint32_t)b > rows.n_rows) pg_error(c);
    }
    const int32_t pos = c.positions[s];
    if (pos < 0 || r1 <= r0) return;
    const uint64_t n = r1 - r0, p0 = (uint64_t)pos, p1 = p0 + n;            // positions [p0, p1)
    const uint64_t lp = p0 / c.page + j, a0 = max(p0, lp * c.page), a1 = min(p1, (lp + 1u) * c.page);
    if (a0 >= a1) return;
    if (lp >= c.table_pages) {
        if (tid == 0u) pg_error(c);
        return;
    }
    const int32_t phys = pg_physical(c, s, (uint32_t)lp);
    if (phys < 0) return;

    const uint32_t hd = c.hd, lanes = hd / 8u, groups = PG_THREADS / lanes / 2u;   // lane groups per side (K, V)
    const uint32_t grp = tid / lanes, lane = tid % lanes, col = lane * 8u;
    const bool is_v = grp >= groups;
    const uint32_t g = is_v ? grp - groups : grp;
    const uint32_t off0 = (uint32_t)(a0 - lp * c.page), cnt = (uint32_t)(a1 - a0), row0 = r0 + (uint32_t)(a0 - p0);
    const uint8_t* src = is_v ? rows.v : rows.k;
    const int64_t src_stride = is_v ? rows.v_stride : rows.k_stride;
    uint8_t* dst = (is_v ? c.v : c.k) + (int64_t)phys * c.page_b + (int64_t)h * c.head_b;
    uint8_t* exps = c.fp8 ? (is_v ? c.ve : c.ke) + ((int64_t)phys * c.nkv + h) * c.page : nullptr;
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = INFINITY;
        hi[i] = -INFINITY;
    }
    for (uint32_t i0 = 0; i0 < cnt; i0 += groups) {   // every lane of a warp takes part in the shuffles
        const uint32_t i = i0 + g;
        const bool live = i < cnt;
        float x[8] = {};
        if (live) pg_load8<T>(reinterpret_cast<const T*>(src + (int64_t)(row0 + i) * src_stride) + (size_t)h * hd + col, x);
        uint8_t* out = dst + (int64_t)(off0 + (live ? i : 0u)) * c.row_b;
        if (c.fp8) {
            float big = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float a = fabsf(x[q]);
                if (a < INFINITY) big = fmaxf(big, a);
            }
            for (uint32_t o = lanes / 2u; o > 0u; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            const int32_t e = pg_exponent(big);
            const float inv = pg_inv_scale(e), scale = pg_scale((uint32_t)(e + 127));
            uint32_t code[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                code[q] = pg_to_e4m3x2(x[2 * q] * inv, x[2 * q + 1] * inv);
                const float2 f = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(code[q]));
                x[2 * q] = f.x * scale;
                x[2 * q + 1] = f.y * scale;
            }
            if (live) {
                *reinterpret_cast<uint2*>(out + col) = make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
                if (lane == 0u) exps[off0 + i] = (uint8_t)(e + 127);
            }
        } else if (live) {
            const uint4 w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
            *reinterpret_cast<uint4*>(out + col * 2u) = w;
            x[0] = bf_lo(w.x); x[1] = bf_hi(w.x); x[2] = bf_lo(w.y); x[3] = bf_hi(w.y);
            x[4] = bf_lo(w.z); x[5] = bf_hi(w.z); x[6] = bf_lo(w.w); x[7] = bf_hi(w.w);
        }
        if (live) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {   // fminf and fmaxf leave NaN out
                lo[q] = fminf(lo[q], x[q]);
                hi[q] = fmaxf(hi[q], x[q]);
            }
        }
    }
    if (!c.bounds) return;
    if (!is_v) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            pg_red[(g * 2u) * hd + col + q] = lo[q];
            pg_red[(g * 2u + 1u) * hd + col + q] = hi[q];
        }
    }
    __syncthreads();
    for (uint32_t t = tid; t < 2u * hd; t += PG_THREADS) {
        const bool up = t >= hd;
        __nv_bfloat16* b = c.bounds + (((int64_t)phys * c.nkv + h) * 2) * hd + t;
        float x = off0 == 0u ? (up ? -INFINITY : INFINITY) : __bfloat162float(*b);
        for (uint32_t k = 0; k < groups; ++k) {
            const float y = pg_red[k * 2u * hd + t];
            x = up ? fmaxf(x, y) : fminf(x, y);
        }
        *b = __float2bfloat16_rn(x);
    }
}

// Sequence a row belongs to: the largest s with row_starts[s] <= row (the last of several that start there).
__device__ __forceinline__ uint32_t pg_seq_of_row(const PagedView& c, const PagedRows& r, uint32_t row) {
    if (!r.row_starts) return row;
    uint32_t lo = 0, hi = c.n_seqs;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) / 2u;
        if (pg_row_start(c, r, mid) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Read back: hd / 8 lanes per (row, head, K or V).
template <class T>
__global__ void __launch_bounds__(PG_THREADS) kl_paged_read_kernel(const PagedView c, const PagedRows rows) {
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t lanes = c.hd / 8u, groups = PG_THREADS / lanes, grp = threadIdx.x / lanes, col = threadIdx.x % lanes * 8u;
    const uint32_t row = blockIdx.x;
    if (rows.row_starts && row == 0u)
        for (uint32_t s = threadIdx.x; s < c.n_seqs; s += PG_THREADS) {
            const int32_t a = rows.row_starts[s], b = rows.row_starts[s + 1u];
            if (a < 0 || b < a || (uint32_t)b > rows.n_rows) pg_error(c);
        }
    const uint32_t s = pg_seq_of_row(c, rows, row);
    if (s >= c.n_seqs) return;
    const uint32_t r0 = pg_row_start(c, rows, s), r1 = pg_row_start(c, rows, s + 1u);
    const int32_t pos = c.positions[s];
    if (pos < 0 || row < r0 || row >= r1) return;
    const uint64_t at = (uint64_t)pos + (row - r0), lp = at / c.page;
    if (lp >= c.table_pages) {
        if (threadIdx.x == 0u) pg_error(c);
        return;
    }
    const int32_t phys = pg_physical(c, s, (uint32_t)lp);
    if (phys < 0) return;
    const uint32_t off = (uint32_t)(at - lp * c.page);
    for (uint32_t i = grp; i < 2u * c.nkv; i += groups) {
        const bool is_v = i >= c.nkv;
        const uint32_t h = is_v ? i - c.nkv : i;
        const uint8_t* src = (is_v ? c.v : c.k) + (int64_t)phys * c.page_b + (int64_t)h * c.head_b + (int64_t)off * c.row_b;
        const float scale = c.fp8 ? pg_scale((is_v ? c.ve : c.ke)[((int64_t)phys * c.nkv + h) * c.page + off]) : 1.f;
        float x[8];
        pg_load_cached8(src, col, c.fp8, scale, x);
        uint8_t* out = is_v ? rows.v + (int64_t)row * rows.v_stride : rows.k + (int64_t)row * rows.k_stride;
        pg_store8<T>(reinterpret_cast<T*>(out) + (size_t)h * c.hd + col, x);
    }
}

// ---- page selection

struct PagedSelect {
    const uint8_t* q;
    int64_t q_stride;      // bytes
    uint32_t q_f32, nq, G;
    uint32_t keep_first, keep_last, n_select;
    int32_t* selected;
    float* scores;         // [n_seqs][nkv][table_pages]
};
__device__ __forceinline__ float pg_q(const uint8_t* row, uint32_t f32, uint32_t i) {
    return f32 ? reinterpret_cast<const float*>(row)[i] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[i]);
}

// A score as a whole number of the same order: NaN below everything.
__device__ __forceinline__ uint32_t pg_key(float x) {
    if (isnan(x)) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);   // -0 becomes +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One warp per page: scores in 64 bits (the products of a bf16 bound and a query are exact there), rounded once.
__global__ void __launch_bounds__(PG_THREADS) kl_paged_score_kernel(const PagedView c, const PagedSelect a) {
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t s = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31u;
    const uint32_t lp = blockIdx.x * (PG_THREADS / 32u) + (threadIdx.x >> 5);
    const uint32_t n = (pg_length(c, s) + c.page - 1u) / c.page;
    if (lp >= n) return;
    const int32_t phys = pg_physical(c, s, lp);
    float best = -INFINITY;
    if (phys >= 0) {
        const __nv_bfloat16* b = c.bounds + ((int64_t)phys * c.nkv + h) * 2 * c.hd;
        bool first = true;
        for (uint32_t g = 0; g < a.G; ++g) {
            const uint8_t* q = a.q + (int64_t)s * a.q_stride;
            double sum = 0.0;
            for (uint32_t d = lane; d < c.hd; d += 32u) {
                const float x = pg_q(q, a.q_f32, (h * a.G + g) * c.hd + d);
                sum += (double)x * (double)__bfloat162float(x >= 0.f ? b[c.hd + d] : b[d]);
            }
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float sc = (float)sum;
            best = first ? sc : (isnan(sc) || isnan(best) ? (isnan(best) ? sc : best) : fmaxf(best, sc));
            first = false;
        }
    }
    if (lane == 0u) a.scores[((size_t)s * c.nkv + h) * c.table_pages + lp] = best;
}

// One block per (sequence, kv head): the n_select-th largest key by bisection over its bits, then the pages above it and
// the first ones equal to it, in order.
__global__ void __launch_bounds__(PG_THREADS) kl_paged_topk_kernel(const PagedView c, const PagedSelect a) {
    __shared__ uint32_t red[PG_THREADS / 32 * 2 + 4];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint32_t n = (pg_length(c, s) + c.page - 1u) / c.page;
    const float* sc = a.scores + ((size_t)s * c.nkv + h) * c.table_pages;
    int32_t* out = a.selected + ((size_t)s * c.nkv + h) * a.n_select;
    auto key = [&](uint32_t i) { return i < a.keep_first || i + a.keep_last >= n ? 0xffffffffu : pg_key(sc[i]); };
    auto count = [&](uint32_t t) {   // pages with key >= t
        uint32_t x = 0;
        for (uint32_t i = tid; i < n; i += PG_THREADS) x += key(i) >= t;
        x = __reduce_add_sync(0xffffffffu, x);
        __syncthreads();
        if (lane == 0u) red[warp] = x;
        __syncthreads();
        uint32_t y = 0;
        for (int w = 0; w < PG_THREADS / 32; ++w) y += red[w];
        return y;
    };
    uint32_t t = 0, above = 0;
    if (n > a.n_select) {
        for (int b = 31; b >= 0; --b)   // the largest t with at least n_select keys >= t
            if (count(t | 1u << b) >= a.n_select) t |= 1u << b;
        above = t == 0xffffffffu ? 0u : count(t + 1u);
    }
    const uint32_t ties = n > a.n_select ? a.n_select - above : 0u;   // pages equal to t that still fit
    uint32_t done = 0, tied = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += PG_THREADS) {
        const uint32_t i = i0 + tid, k = i < n ? key(i) : 0u;
        const bool eq = i < n && n > a.n_select && k == t, gt = i < n && (n <= a.n_select || k > t);
        const uint32_t be = __ballot_sync(0xffffffffu, eq), bg = __ballot_sync(0xffffffffu, gt);
        __syncthreads();
        if (lane == 0u) {
            red[2 * warp] = __popc(be);
            red[2 * warp + 1] = __popc(bg);
        }
        __syncthreads();
        uint32_t e = tied + __popc(be & ((1u << lane) - 1u)), ge = __popc(bg & ((1u << lane) - 1u)), et = 0, gt_ = 0;
        for (uint32_t w = 0; w < PG_THREADS / 32; ++w) {
            if (w < warp) {
                e += red[2 * w];
                ge += red[2 * w + 1];
            }
            et += red[2 * w];
            gt_ += red[2 * w + 1];
        }
        // chosen before this page: the larger ones and as many equal ones as fit
        const uint32_t at = done + ge + min(e, ties) - min(tied, ties);
        if ((gt || (eq && e < ties)) && at < a.n_select) out[at] = (int32_t)i;
        done += gt_ + min(tied + et, ties) - min(tied, ties);
        tied += et;
    }
    for (uint32_t i = done + tid; i < a.n_select; i += PG_THREADS) out[i] = -1;
}

// ---- attention

struct PagedAttn {
    const uint8_t* q;
    uint8_t* out;
    int64_t q_stride, out_stride;   // bytes
    uint32_t f32;                   // element type of q and out
    uint32_t nq, G;
    float scale_log2;               // scale * log2(e)
    uint32_t window;                // 0: none
    const int32_t* selected;        // [n_seqs][nkv][n_select] or null
    uint32_t n_select;
    float* lse;                     // or null
};

// One block per (query head, sequence), one position per warp at a time, softmax with a running maximum.
__global__ void __launch_bounds__(PG_THREADS) kl_paged_attn_kernel(const PagedView c, const PagedAttn a) {
    constexpr int NW = PG_THREADS / 32;
    __shared__ float sm_m[NW], sm_l[NW], sm_o[NW][256];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t s = blockIdx.y, hq = blockIdx.x, h = hq / a.G, tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint32_t len = pg_length(c, s), lo = a.window && len > a.window ? len - a.window : 0u;
    const uint32_t lanes = c.hd / 8u;   // lanes that hold columns (eight each)
    const bool live = lane < lanes;
    float q[8] = {}, o[8] = {}, m = -INFINITY, l = 0.f;
    if (live)
        for (int i = 0; i < 8; ++i) q[i] = pg_q(a.q + (int64_t)s * a.q_stride, a.f32, hq * c.hd + lane * 8u + i);
    const uint32_t pages = (len + c.page - 1u) / c.page;
    const int32_t* sel = a.selected ? a.selected + ((size_t)s * c.nkv + h) * a.n_select : nullptr;
    const uint32_t total = sel ? min(a.n_select, pages) : pages;
    for (uint32_t i = 0; i < total; ++i) {
        const int32_t lpi = sel ? sel[i] : (int32_t)i;
        if (lpi < 0 || (uint32_t)lpi >= pages) continue;
        const uint32_t lp = (uint32_t)lpi, p0 = lp * c.page;
        if (p0 + c.page <= lo) continue;
        const int32_t phys = pg_physical(c, s, lp);
        if (phys < 0) continue;
        for (uint32_t r = warp; r < c.page; r += NW) {
            const uint32_t p = p0 + r;
            if (p < lo || p >= len) continue;
            const int64_t off = (int64_t)phys * c.page_b + (int64_t)h * c.head_b + (int64_t)r * c.row_b;
            const int64_t eoff = ((int64_t)phys * c.nkv + h) * c.page + r;
            float x[8] = {}, dot = 0.f;
            if (live) pg_load_cached8(c.k + off, lane * 8u, c.fp8, c.fp8 ? pg_scale(c.ke[eoff]) : 1.f, x);
            for (int j = 0; j < 8; ++j) dot += q[j] * x[j];
            for (int k = 16; k > 0; k >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, k);
            const float sc = dot * a.scale_log2, mn = fmaxf(m, sc), mu = mn == -INFINITY ? 0.f : mn;
            const float f = exp2f(m - mu), w = exp2f(sc - mu);
            m = mn;
            l = l * f + w;
            if (live) pg_load_cached8(c.v + off, lane * 8u, c.fp8, c.fp8 ? pg_scale(c.ve[eoff]) : 1.f, x);
            for (int j = 0; j < 8; ++j) o[j] = o[j] * f + w * x[j];
        }
    }
    if (lane == 0u) {
        sm_m[warp] = m;
        sm_l[warp] = l;
    }
    if (live)
        for (int i = 0; i < 8; ++i) sm_o[warp][lane * 8u + i] = o[i];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w]);
    const float mu = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < NW; ++w) L += sm_l[w] * exp2f(sm_m[w] - mu);
    for (uint32_t d = tid; d < c.hd; d += PG_THREADS) {
        float v = 0.f;
        for (int w = 0; w < NW; ++w) v += sm_o[w][d] * exp2f(sm_m[w] - mu);
        v = L == 0.f ? 0.f : v / L;
        uint8_t* out = a.out + (int64_t)s * a.out_stride;
        if (a.f32) reinterpret_cast<float*>(out)[hq * c.hd + d] = v;
        else reinterpret_cast<__nv_bfloat16*>(out)[hq * c.hd + d] = __float2bfloat16_rn(v);
    }
    if (a.lse && tid == 0u) a.lse[(size_t)s * a.nq + hq] = (M + log2f(L)) * 0.6931471805599453f;
}

}  // namespace kl
