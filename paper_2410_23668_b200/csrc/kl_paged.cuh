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
    uint32_t q_f32;                 // element type of q
    uint32_t out_mode;              // PA_BF16, PA_F32, PA_OPERAND
    uint32_t nq, G, HT;             // G query heads per kv head, in HT tiles of at most eight
    float scale_log2;               // scale * log2(e)
    uint32_t window;                // 0: none
    const int32_t* selected;        // [n_seqs][nkv][n_select] or null
    uint32_t n_select;
    float* lse;                     // or null
    // workspace: partial results, one record = [8 heads][hd] sums and [8 heads] (maximum, sum)
    float *part, *part_ml;          // [blocks][2]: the pair that began in an earlier block, the pair that goes on in the next one
    float *head, *head_ml;          // [blocks][warps]: a warp's first pair when it began in an earlier warp
    int4* meta;                     // [blocks]: (PA_* flags, sequence and pair-in-sequence of the second record)
};
enum { PA_BF16 = 0, PA_F32 = 1, PA_OPERAND = 2 };
enum { PA_FIRST = 1, PA_FIRST_GOES_ON = 2, PA_SECOND = 4 };

__device__ __forceinline__ float pa_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pa_pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void pa_mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool FP8>
__device__ __forceinline__ void pa_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (FP8) pa_mma_f16(d, a, b0, b1);
    else mma_16816(d, a, b0, b1);
}
// Two numbers as their halves: hi rounded to 16 bits, lo what is left (an f16 pair with an e4m3 cache, a bf16 pair else).
template <bool FP8>
__device__ __forceinline__ void pa_split(float x0, float x1, uint32_t& hi, uint32_t& lo) {
    if (FP8) {
        hi = pa_pack_f16(x0, x1);
        const float2 f = pg_f16x2_to_float2(hi);
        lo = pa_pack_f16(x0 - f.x, x1 - f.y);
    } else {
        hi = pack_bf16(x0, x1);
        lo = pack_bf16(x0 - bf_lo(hi), x1 - bf_hi(hi));
    }
}
// 16 (or 4) bytes to shared memory, asynchronously; nothing is read and zeros are written when `ok` is false.
__device__ __forceinline__ void pa_copy16(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
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
__device__ __forceinline__ void pa_store_lse(const PagedAttn& a, uint32_t s, uint32_t hq, float m, float l) {
    if (a.lse) a.lse[(size_t)s * a.nq + hq] = (m + log2f(l)) * 0.6931471805599453f;   // l == 0: -inf
}

constexpr uint32_t PA_NONE = 0x7fffffffu;   // position of a row group that holds nothing to attend to
constexpr int PA_TILE = 16;                 // positions per tile
constexpr int PA_LENS = 1024;               // sequences whose lengths are kept in shared memory
constexpr uint32_t PA_MIN_TILES = 8;        // fewest tiles worth a block

template <int HD, bool FP8>
struct PaCfg {
    static constexpr int ROW = FP8 ? HD : 2 * HD;            // bytes of a cached row
    static constexpr int TILE = PA_TILE * ROW;               // bytes of a K (or V) tile
    static constexpr int NW = HD == 256 && !FP8 ? 6 : 8;     // warps
    static constexpr int RING = 196608 / (NW * 2 * TILE);
    static constexpr int ST = RING > 8 ? 8 : RING;           // tiles of a warp's ring
    static constexpr size_t SMEM = (size_t)NW * ST * (2 * TILE + 32 + 16) + NW * 8 * 8 + 256 * 8 + PA_LENS * 4 + 256;
};

// Positions of sequence s that take part, as tiles.
struct PaSeq {
    uint32_t len, lo;   // positions [lo, len)
    uint32_t t0, nt;    // tiles [t0, t0 + nt) of its (virtual) positions
    uint32_t listed;    // entries of the page list that are looked at
};
__device__ __forceinline__ PaSeq pa_seq(const PagedView& c, const PagedAttn& a, uint32_t len) {
    PaSeq q;
    q.len = len;
    q.lo = a.window && len > a.window ? len - a.window : 0u;
    if (a.selected) {
        q.listed = min(a.n_select, (len + c.page - 1u) / c.page);
        q.t0 = 0;
        q.nt = (uint32_t)(((uint64_t)q.listed * c.page + PA_TILE - 1u) / PA_TILE);
    } else {
        q.listed = 0;
        q.t0 = q.lo / PA_TILE;
        q.nt = len ? (len + PA_TILE - 1u) / PA_TILE - q.t0 : 0u;
    }
    return q;
}

// Attention of one new token per sequence as ONE balanced stream over the whole batch.
//
//   * Work: 16 positions of one kv head of one sequence, for up to eight of the query heads that share it, are a tile.  The
//     tiles of all (sequence, kv head, head tile) pairs form one list; every block takes an equal, contiguous range of it and
//     every warp an equal part of that, whatever the sequences' lengths.  A warp walks its range alone: a ring of its own in
//     shared memory, filled with 16-byte asynchronous copies ST - 1 tiles ahead (across pair boundaries), no barrier.
//     Where the range leaves a pair the pair's result is finished, or left as a partial one if other warps share the pair;
//     those of one block meet in shared memory at the end, those of several blocks in kl_paged_merge_kernel.
//   * Mathematics: running maximum m and sum l of 2^(s - m) per head, s = q . k * scale * log2(e).  Both products run on
//     mma.m16n8k16 with the eight heads as rows 0..7 of the A operand and what 16-bit rounding leaves of them as rows
//     8..15: q = hi + lo and p = hi + lo cost no extra instruction, the sums of the two halves are added in 32 bits.
//     A score fragment holds head lane / 4 in every register, so p goes straight into the A operand of the value product.
//   * e4m3 rows become f16 (exact) on the way to the tensor cores.  Their scales are powers of two: 2^(e_k - 127) multiplies
//     the score, 2^(e_v - 127) the probability.  The weighted probabilities w = p * 2^(e_v - 127) have a running maximum
//     of their own, so that f16 holds them whatever the scales (w * 2^14 at most 2^14).
//   * UPT = page_size % 16 == 0 ? 1 : 4 page look-ups per tile (a lane looks up one, 32 / UPT tiles in a go).
template <int HD, bool FP8, int UPT>
__global__ void __launch_bounds__(PaCfg<HD, FP8>::NW * 32, 1) kl_paged_attn_kernel(const PagedView c, const PagedAttn a) {
    using Cfg = PaCfg<HD, FP8>;
    constexpr int NW = Cfg::NW, ST = Cfg::ST, ROW = Cfg::ROW, TILE = Cfg::TILE, NT = NW * 32;
    constexpr uint32_t UR = PA_TILE / UPT;                       // rows per page look-up
    constexpr uint32_t TPB = 32 / UPT;                           // tiles per batch of look-ups
    constexpr int CPR = ROW / 16, RPP = 32 / CPR;                // 16-byte pieces per row, rows per pass of a warp
    constexpr int NMMA = HD / 16, NOUT = HD / 8;
    extern __shared__ __align__(128) uint8_t pa_smem[];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, g = lane >> 2, j = lane & 3u;
    uint8_t* exps_all = pa_smem + (size_t)NW * ST * 2 * TILE;
    uint32_t* lps_all = reinterpret_cast<uint32_t*>(exps_all + (size_t)NW * ST * 32);
    float2* ml_all = reinterpret_cast<float2*>(lps_all + NW * ST * 4);          // [NW][8]
    uint64_t* pre = reinterpret_cast<uint64_t*>(ml_all + NW * 8);               // [NT]
    uint32_t* lens = reinterpret_cast<uint32_t*>(pre + 256);                    // [PA_LENS]
    uint32_t* misc = lens + PA_LENS;
    uint64_t* wsum = reinterpret_cast<uint64_t*>(misc);                         // [NW], then the entries below
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;

    // ---- the list of tiles: prefix sums over the sequences
    const uint32_t PH = c.nkv * a.HT, n = c.n_seqs, per = (n + NT - 1u) / NT;
    uint64_t mine = 0;
    for (uint32_t s = tid * per; s < min(n, (tid + 1u) * per); ++s) {
        const uint32_t len = pg_length(c, s);
        if (s < (uint32_t)PA_LENS) lens[s] = len;
        mine += (uint64_t)pa_seq(c, a, len).nt * PH;
    }
    uint64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31u) wsum[warp] = incl;
    __syncthreads();
    uint64_t W = 0, before = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < (int)warp) before += wsum[w];
        W += wsum[w];
    }
    pre[tid] = before + incl - mine;
    __syncthreads();
    auto length = [&](uint32_t s) { return s < (uint32_t)PA_LENS ? lens[s] : pg_length(c, s); };

    for (uint32_t s = blockIdx.x; s < n; s += gridDim.x)   // sequences without a position: zeros
        if (length(s) == 0u) {
            for (uint32_t i = tid; i < a.nq * (HD / 2); i += NT) pa_store2(c, a, s, i / (HD / 2), i % (HD / 2) * 2u, 0.f, 0.f);
            for (uint32_t i = tid; i < a.nq; i += NT) pa_store_lse(a, s, i, 0.f, 0.f);
        }

    const uint64_t blocks = min((uint64_t)gridDim.x, (W + PA_MIN_TILES - 1u) / PA_MIN_TILES);   // blocks at work
    if (blockIdx.x >= blocks) {
        if (tid == 0u) a.meta[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    const uint64_t b_lo = W * blockIdx.x / blocks, b_hi = W * (blockIdx.x + 1u) / blocks;
    const uint64_t lo = b_lo + (b_hi - b_lo) * warp / NW, hi = b_lo + (b_hi - b_lo) * (warp + 1u) / NW;

    // ---- this warp's range
    struct Entry { uint32_t valid, s, ph, begins, ends; } first = {0, 0, 0, 0, 0}, last = {0, 0, 0, 0, 0};
    const uint32_t ring = smem_u32(pa_smem) + warp * (ST * 2 * TILE);
    const uint32_t exps = smem_u32(exps_all) + warp * (ST * 32);
    volatile uint32_t* lps = lps_all + warp * (ST * 4);
    if (lo < hi) {
        uint32_t i0 = 0, i1 = NT;
        while (i1 - i0 > 1u) {
            const uint32_t mid = (i0 + i1) / 2u;
            if (pre[mid] <= lo) i0 = mid;
            else i1 = mid;
        }
        uint64_t rem = lo - pre[i0];
        uint32_t cs = i0 * per;                    // cursor of the tiles that are consumed
        PaSeq cq = pa_seq(c, a, length(cs));
        while (rem >= (uint64_t)cq.nt * PH) {
            rem -= (uint64_t)cq.nt * PH;
            cq = pa_seq(c, a, length(++cs));
        }
        uint32_t cph = (uint32_t)(rem / cq.nt), ct = (uint32_t)(rem % cq.nt);

        // cursor of the tiles that are requested, and the look-ups of its batch (this one and the next)
        uint32_t is = cs, iph = cph, it = ct;
        PaSeq iq = cq;
        uint32_t batch = 0xffffffffu;
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
            phys = pg_physical(c, is, logical);
            if (phys >= 0) lp = logical * c.page + row;
        };
        uint64_t left = hi - lo;   // tiles still to request
        auto issue = [&](uint32_t st) {
            const uint32_t b = it / TPB, at = it - b * TPB;
            if (b != batch) {
                if (batch != 0xffffffffu && b == batch + 1u) {
                    b_phys = n_phys; b_lp = n_lp; b_row = n_row;
                } else {
                    look_up(b, b_phys, b_lp, b_row);
                }
                batch = b;
                if ((b + 1u) * TPB < iq.nt) look_up(b + 1u, n_phys, n_lp, n_row);
            }
            const uint32_t h = iph / a.HT;
            const uint32_t kd = ring + st * (2 * TILE), vd = kd + TILE;
            const int64_t hoff = (int64_t)h * c.head_b;
            const uint32_t ch = lane % CPR, r0 = lane / CPR;
            if (UPT == 1) {
                const int32_t phys = __shfl_sync(0xffffffffu, b_phys, at);
                const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, at), row = __shfl_sync(0xffffffffu, b_row, at);
                const int32_t r_lo = (int32_t)iq.lo - (int32_t)lp, r_hi = (int32_t)iq.len - (int32_t)lp;   // rows of the tile that count
                int64_t off = (int64_t)max(phys, 0) * c.page_b + hoff + (int64_t)(row + r0) * c.row_b + ch * 16u;
                const int64_t step = (int64_t)RPP * c.row_b;
#pragma unroll
                for (int i = 0; i < PA_TILE / RPP; ++i) {
                    const int32_t r = i * RPP + (int32_t)r0;
                    const bool ok = r >= r_lo && r < r_hi;
                    const uint32_t fk = CPR >= 8 ? ((r & 1) << 2 | ((r >> 1) & 3)) : 0u;
                    const uint32_t fv = CPR >= 8 ? (FP8 ? (r & 7) : fk) : ((r >> 1) & 3);
                    pa_copy16(kd + r * ROW + ((ch ^ fk) << 4), c.k + off, ok);
                    pa_copy16(vd + r * ROW + ((ch ^ fv) << 4), c.v + off, ok);
                    off += step;
                }
                if (FP8 && lane < 2u) {
                    const int64_t eoff = ((int64_t)max(phys, 0) * c.nkv + h) * c.page + row;
                    pa_copy16(exps + st * 32 + lane * 16, (lane ? c.ve : c.ke) + eoff, phys >= 0);
                }
                if (lane == 0u) lps[st * 4] = lp;
            } else {
#pragma unroll
                for (int i = 0; i < PA_TILE / RPP; ++i) {
                    const int32_t r = i * RPP + (int32_t)r0;
                    const uint32_t src = at * UPT + (r >> 2);
                    const int32_t phys = __shfl_sync(0xffffffffu, b_phys, src);
                    const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, src), row = __shfl_sync(0xffffffffu, b_row, src);
                    const int32_t p = (int32_t)lp + (r & 3);
                    const bool ok = lp != PA_NONE && p >= (int32_t)iq.lo && p < (int32_t)iq.len;
                    const int64_t off = (int64_t)max(phys, 0) * c.page_b + hoff + (int64_t)(row + (r & 3)) * c.row_b + ch * 16u;
                    const uint32_t fk = CPR >= 8 ? ((r & 1) << 2 | ((r >> 1) & 3)) : 0u;
                    const uint32_t fv = CPR >= 8 ? (FP8 ? (r & 7) : fk) : ((r >> 1) & 3);
                    pa_copy16(kd + r * ROW + ((ch ^ fk) << 4), c.k + off, ok);
                    pa_copy16(vd + r * ROW + ((ch ^ fv) << 4), c.v + off, ok);
                }
                {
                    const uint32_t src = at * UPT + (lane & 3u);
                    const int32_t phys = __shfl_sync(0xffffffffu, b_phys, src);
                    const uint32_t lp = __shfl_sync(0xffffffffu, b_lp, src), row = __shfl_sync(0xffffffffu, b_row, src);
                    if (FP8 && lane < 8u) {
                        const int64_t eoff = ((int64_t)max(phys, 0) * c.nkv + h) * c.page + row;
                        pa_copy4(exps + st * 32 + lane * 4, (lane < 4u ? c.ke : c.ve) + eoff, phys >= 0);
                    }
                    if (lane < 4u) lps[st * 4 + lane] = lp;
                }
            }
            --left;
            if (++it == iq.nt && left) {   // on to the next pair, perhaps of the next sequence that has any
                it = 0;
                batch = 0xffffffffu;
                if (++iph == PH) {
                    iph = 0;
                    do iq = pa_seq(c, a, length(++is));
                    while (iq.nt == 0u);
                }
            }
        };
#pragma unroll
        for (int st = 0; st < ST - 1; ++st) {
            if (left) issue(st);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }

        // ---- state of the pair under way: head g of the tile in every lane of its quad
        uint32_t qa[NMMA][4];
        float o[NOUT][4], m = -INFINITY, l = 0.f, mw = -INFINITY, qs = 0.f;
        auto begin_pair = [&]() {
            const uint32_t h = cph / a.HT, hg = (cph - h * a.HT) * 8u + g;
            const bool live = hg < a.G;
            const uint8_t* q = a.q + (int64_t)cs * a.q_stride;
            const uint32_t base = (h * a.G + hg) * HD;
            float x[NMMA][4];
            constexpr int PIECE = FP8 ? 16 : 8;   // consecutive columns of a lane per 16-byte piece of a row
            float big = 0.f;
#pragma unroll
            for (int i = 0; i < NMMA; ++i) {
                const uint32_t d = (i / (PIECE / 4)) * (4 * PIECE) + j * PIECE + (i % (PIECE / 4)) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = 0.f;
                if (live) {
                    if (a.q_f32) {
                        const float4 f = *reinterpret_cast<const float4*>(q + (size_t)(base + d) * 4);
                        x[i][0] = f.x; x[i][1] = f.y; x[i][2] = f.z; x[i][3] = f.w;
                    } else {
                        const uint2 f = *reinterpret_cast<const uint2*>(q + (size_t)(base + d) * 2);
                        x[i][0] = bf_lo(f.x); x[i][1] = bf_hi(f.x); x[i][2] = bf_lo(f.y); x[i][3] = bf_hi(f.y);
                    }
                }
                if (FP8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) big = fmaxf(big, fabsf(x[i][e]));
            }
            qs = a.scale_log2;
            float f = 1.f;
            if (FP8) {   // f16 operands: the head's largest query element comes to lie in [2^14, 2^15)
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const int32_t k = max((int32_t)(__float_as_uint(big) >> 23) - 127, -112);
                f = __uint_as_float((uint32_t)(127 + 14 - k) << 23);
                qs *= __uint_as_float((uint32_t)(127 - 14 + k) << 23);
            }
#pragma unroll
            for (int i = 0; i < NMMA; ++i) {
                pa_split<FP8>(x[i][0] * f, x[i][1] * f, qa[i][0], qa[i][1]);
                pa_split<FP8>(x[i][2] * f, x[i][3] * f, qa[i][2], qa[i][3]);
            }
#pragma unroll
            for (int i = 0; i < NOUT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
            m = mw = -INFINITY;
            l = 0.f;
        };
        // The pair's result over the tiles seen: sums relative to 2^m, columns as emit(head, d, v0, v1) gets them.
        auto end_pair = [&](auto&& emit) {
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            const float f = !FP8 ? 1.f : mw == -INFINITY ? 0.f : pa_ex2(mw - m - 14.f);
            if (FP8) {
                constexpr int W16 = HD >= 128 ? 16 : 8;   // columns of a lane's V piece
#pragma unroll
                for (int i = 0; i < NOUT; i += 2) {
                    const uint32_t d = (i / W16) * (8 * W16) + i % W16;
                    emit(d + 2u * j * W16, (o[i][0] + o[i][2]) * f, (o[i + 1][0] + o[i + 1][2]) * f);
                    emit(d + (2u * j + 1u) * W16, (o[i][1] + o[i][3]) * f, (o[i + 1][1] + o[i + 1][3]) * f);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NOUT; ++i) emit(i * 8u + 2u * j, o[i][0] + o[i][2], o[i][1] + o[i][3]);
            }
        };

        const uint32_t total = (uint32_t)(hi - lo);   // a warp's share (2^32 tiles would be hours of work)
        uint32_t seg0 = ct;                           // first tile of the pair that this warp has seen
        begin_pair();
        for (uint32_t k = 0, st = 0; k < total; ++k) {
            asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
            __syncwarp();
            if (left) issue(st == 0 ? ST - 1 : st - 1);
            asm volatile("cp.async.commit_group;" ::: "memory");

            const uint32_t kd = ring + st * (2 * TILE), vd = kd + TILE;
            // scores of positions 2j, 2j + 1 (s[0], s[1]) and 2j + 8, 2j + 9 (s[2], s[3]) of the tile for head g
            float sc[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
                const uint32_t r = t * 8 + g, row = kd + r * ROW;
                const uint32_t fk = CPR >= 8 ? ((r & 1u) << 2 | ((r >> 1) & 3u)) : 0u;
#pragma unroll
                for (int q = 0; q < CPR / 4; ++q) {
                    const uint4 w = pa_lds16(row + (((q * 4 + j) ^ fk) << 4));
                    if (FP8) {
                        pa_mma<true>(sc[t], qa[q * 4 % NMMA], pg_e4m3x2_to_f16x2(w.x & 0xffffu), pg_e4m3x2_to_f16x2(w.x >> 16));
                        pa_mma<true>(sc[t], qa[(q * 4 + 1) % NMMA], pg_e4m3x2_to_f16x2(w.y & 0xffffu), pg_e4m3x2_to_f16x2(w.y >> 16));
                        pa_mma<true>(sc[t], qa[(q * 4 + 2) % NMMA], pg_e4m3x2_to_f16x2(w.z & 0xffffu), pg_e4m3x2_to_f16x2(w.z >> 16));
                        pa_mma<true>(sc[t], qa[(q * 4 + 3) % NMMA], pg_e4m3x2_to_f16x2(w.w & 0xffffu), pg_e4m3x2_to_f16x2(w.w >> 16));
                    } else {
                        pa_mma<false>(sc[t], qa[q * 2 % NMMA], w.x, w.y);
                        pa_mma<false>(sc[t], qa[(q * 2 + 1) % NMMA], w.z, w.w);
                    }
                }
            }
            float s[4] = {(sc[0][0] + sc[0][2]) * qs, (sc[0][1] + sc[0][3]) * qs, (sc[1][0] + sc[1][2]) * qs, (sc[1][1] + sc[1][3]) * qs};
            float sv[4];
            if (FP8) {
                const uint32_t e = exps + st * 32 + 2 * j;
                uint16_t k0, k1, v0, v1;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(k0) : "r"(e));
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(k1) : "r"(e + 8));
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v0) : "r"(e + 16));
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v1) : "r"(e + 24));
                s[0] *= pg_scale(k0 & 0xffu);
                s[1] *= pg_scale(k0 >> 8);
                s[2] *= pg_scale(k1 & 0xffu);
                s[3] *= pg_scale(k1 >> 8);
                sv[0] = (float)(int)(v0 & 0xffu) - 127.f;
                sv[1] = (float)(int)(v0 >> 8) - 127.f;
                sv[2] = (float)(int)(v1 & 0xffu) - 127.f;
                sv[3] = (float)(int)(v1 >> 8) - 127.f;
            }
            // positions that do not count
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t r = t * 8 + 2 * j;
                const uint32_t lp = UPT == 1 ? lps[st * 4] : lps[st * 4 + (r >> 2)];
                const uint32_t p = lp + (UPT == 1 ? r : (r & 3u));
                const bool none = lp == PA_NONE;
                if (none || p < cq.lo || p >= cq.len) s[2 * t] = -INFINITY;
                if (none || p + 1u < cq.lo || p + 1u >= cq.len) s[2 * t + 1] = -INFINITY;
            }
            float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn;
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pa_ex2(s[i] - mu);
            l = l * pa_ex2(m - mu) + ((p[0] + p[1]) + (p[2] + p[3]));
            float old = m, ref = mn;
            if (FP8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sv[i] += s[i];
                mx = fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3]));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                old = mw;
                ref = mw = fmaxf(mw, mx);
                const float wu = ref == -INFINITY ? 0.f : ref - 14.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = pa_ex2(sv[i] - wu);
            }
            m = mn;
            if (__any_sync(0xffffffffu, ref > old)) {
                const float f = ref == -INFINITY ? 1.f : pa_ex2(old - ref);
#pragma unroll
                for (int i = 0; i < NOUT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] *= f;
            }
            uint32_t pa[4];
            pa_split<FP8>(p[0], p[1], pa[0], pa[1]);
            pa_split<FP8>(p[2], p[3], pa[2], pa[3]);
            if (FP8) {
                constexpr int VW = HD >= 128 ? 4 : 2;            // words of a lane's piece of a row
#pragma unroll
                for (int hh = 0; hh < HD / (32 * VW); ++hh) {
                    uint32_t r[4][4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {                // rows 2j, 2j + 1, 2j + 8, 2j + 9
                        const uint32_t row = 2 * j + (x & 1) + (x >> 1) * 8;
                        if (VW == 4) {
                            const uint4 w = pa_lds16(vd + row * ROW + (((hh * 8 + g) ^ (row & 7u)) << 4));
                            r[x][0] = w.x; r[x][1] = w.y; r[x][2] = w.z; r[x][3] = w.w;
                        } else {
                            const uint2 w = pa_lds8(vd + row * ROW + (((g >> 1) ^ ((row >> 1) & 3u)) << 4) + (g & 1u) * 8u);
                            r[x][0] = w.x; r[x][1] = w.y;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        const uint32_t a01 = __byte_perm(r[0][w], r[1][w], 0x5140), a23 = __byte_perm(r[0][w], r[1][w], 0x7362);
                        const uint32_t b01 = __byte_perm(r[2][w], r[3][w], 0x5140), b23 = __byte_perm(r[2][w], r[3][w], 0x7362);
                        float (*oo)[4] = o + hh * 16 + w * 4;
                        pa_mma<true>(oo[0], pa, pg_e4m3x2_to_f16x2(a01 & 0xffffu), pg_e4m3x2_to_f16x2(b01 & 0xffffu));
                        pa_mma<true>(oo[1], pa, pg_e4m3x2_to_f16x2(a01 >> 16), pg_e4m3x2_to_f16x2(b01 >> 16));
                        pa_mma<true>(oo[2], pa, pg_e4m3x2_to_f16x2(a23 & 0xffffu), pg_e4m3x2_to_f16x2(b23 & 0xffffu));
                        pa_mma<true>(oo[3], pa, pg_e4m3x2_to_f16x2(a23 >> 16), pg_e4m3x2_to_f16x2(b23 >> 16));
                    }
                }
            } else {
                const uint32_t row = (lane >> 3 & 1u) * 8u + (lane & 7u), base = vd + row * ROW, fv = (row & 1u) << 2 | ((row >> 1) & 3u);
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    uint32_t r[4];
                    ldmatrix_x4_trans(r, base + (((i * 2 + (lane >> 4)) ^ fv) << 4));
                    pa_mma<false>(o[2 * i], pa, r[0], r[1]);
                    pa_mma<false>(o[2 * i + 1], pa, r[2], r[3]);
                }
            }
            if (++st == ST) st = 0;

            ++ct;
            if (ct == cq.nt || k + 1u == total) {   // the pair ends here, for this warp at least
                const uint32_t h = cph / a.HT, hg = (cph - h * a.HT) * 8u + g, hq = h * a.G + hg;
                const bool live = hg < a.G, whole = seg0 == 0u && ct == cq.nt;
                if (whole) {
                    float inv = 0.f;
                    end_pair([&](uint32_t d, float v0, float v1) {
                        inv = l == 0.f ? 0.f : 1.f / l;
                        if (live) pa_store2(c, a, cs, hq, d, v0 * inv, v1 * inv);
                    });
                    if (live && j == 0u) pa_store_lse(a, cs, hq, m, l);
                } else {
                    const bool tail = k + 1u == total;
                    Entry& e = tail ? last : first;
                    e = {1u, cs, cph, seg0 == 0u, ct == cq.nt};
                    float* dst;
                    float2* ml;
                    if (tail) {   // the ring has been read to the end
                        asm volatile("cp.async.wait_group 0;" ::: "memory");
                        __syncwarp();
                        dst = reinterpret_cast<float*>(pa_smem + warp * (ST * 2 * TILE));
                        ml = ml_all + warp * 8;
                    } else {
                        const size_t slot = (size_t)blockIdx.x * NW + warp;
                        dst = a.head + slot * 8 * HD;
                        ml = reinterpret_cast<float2*>(a.head_ml) + slot * 8;
                    }
                    end_pair([&](uint32_t d, float v0, float v1) { *reinterpret_cast<float2*>(dst + g * HD + d) = make_float2(v0, v1); });
                    if (j == 0u) ml[g] = make_float2(m, l);
                }
                if (k + 1u < total) {
                    ct = seg0 = 0;
                    if (++cph == PH) {
                        cph = 0;
                        do cq = pa_seq(c, a, length(++cs));
                        while (cq.nt == 0u);
                    }
                    begin_pair();
                }
            }
        }
    }

    // ---- the partial results of this block's warps, in the order of the list: first[0], last[0], first[1], ...
    __syncthreads();   // everyone is done with `wsum`, and with the lengths
    uint32_t* ent = lens;   // [2 NW][4]: valid | begins << 1 | ends << 2, s, ph
    if (lane == 0u) {
        for (int x = 0; x < 2; ++x) {
            const Entry& e = x ? last : first;
            uint32_t* t = ent + (2 * warp + x) * 4;
            t[0] = e.valid | e.begins << 1 | e.ends << 2;
            t[1] = e.s;
            t[2] = e.ph;
        }
    }
    __threadfence_block();
    __syncthreads();
    int4 meta = make_int4(0, 0, 0, 0);
    for (uint32_t e0 = 0; e0 < 2u * NW;) {
        if (!(ent[e0 * 4] & 1u)) {
            ++e0;
            continue;
        }
        uint32_t e1 = e0 + 1u, end = e0;   // entries [e0, e1) of one pair, `end` the last of them
        while (e1 < 2u * NW && (!(ent[e1 * 4] & 1u) || (ent[e1 * 4 + 1] == ent[e0 * 4 + 1] && ent[e1 * 4 + 2] == ent[e0 * 4 + 2]))) {
            if (ent[e1 * 4] & 1u) end = e1;
            ++e1;
        }
        const uint32_t s = ent[e0 * 4 + 1], ph = ent[e0 * 4 + 2], h = ph / a.HT, h0 = (ph - h * a.HT) * 8u;
        const bool begins = ent[e0 * 4] & 2u, ends = ent[end * 4] & 4u, whole = begins && ends;
        const size_t slot = (size_t)blockIdx.x * 2 + (begins ? 1 : 0);
        if (!whole) {
            if (begins) {
                meta.x |= PA_SECOND;
                meta.y = (int)s;
                meta.z = (int)ph;
            } else {
                meta.x |= PA_FIRST | (ends ? 0 : PA_FIRST_GOES_ON);
            }
        }
        const uint32_t heads = min(8u, a.G - h0);
        for (uint32_t i = tid; i < heads * (HD / 2); i += NT) {
            const uint32_t hh = i / (HD / 2), d = i % (HD / 2) * 2u;
            auto rec = [&](uint32_t e, const float*& o, float2& ml) {
                const size_t gs = (size_t)blockIdx.x * NW + e / 2u;
                if (e & 1u) {
                    o = reinterpret_cast<const float*>(pa_smem + (e / 2u) * (ST * 2 * TILE));
                    ml = ml_all[(e / 2u) * 8 + hh];
                } else {
                    o = a.head + gs * 8 * HD;
                    ml = reinterpret_cast<const float2*>(a.head_ml)[gs * 8 + hh];
                }
                o += hh * HD + d;
            };
            float M = -INFINITY, L = 0.f, v0 = 0.f, v1 = 0.f;
            for (uint32_t e = e0; e < e1; ++e)
                if (ent[e * 4] & 1u) {
                    const float* o;
                    float2 ml;
                    rec(e, o, ml);
                    M = fmaxf(M, ml.x);
                }
            const float mu = M == -INFINITY ? 0.f : M;
            for (uint32_t e = e0; e < e1; ++e)
                if (ent[e * 4] & 1u) {
                    const float* o;
                    float2 ml;
                    rec(e, o, ml);
                    const float f = pa_ex2(ml.x - mu);
                    const float2 x = *reinterpret_cast<const float2*>(o);
                    L += ml.y * f;
                    v0 += x.x * f;
                    v1 += x.y * f;
                }
            if (whole) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                pa_store2(c, a, s, h * a.G + h0 + hh, d, v0 * inv, v1 * inv);
                if (d == 0u) pa_store_lse(a, s, h * a.G + h0 + hh, M, L);
            } else {
                *reinterpret_cast<float2*>(a.part + (slot * 8 + hh) * HD + d) = make_float2(v0, v1);
                if (d == 0u) reinterpret_cast<float2*>(a.part_ml)[slot * 8 + hh] = make_float2(M, L);
            }
        }
        e0 = e1;
    }
    if (tid == 0u) a.meta[blockIdx.x] = meta;
}

// Joins the partial results of the pairs that several blocks of kl_paged_attn_kernel share, in the order of the blocks.
// Block (b, h): head h of the pair that begins in block b and goes on in b + 1, if there is one.
constexpr int PA_MERGE_THREADS = 128;
constexpr int PA_MAX_BLOCKS = 256;
__global__ void __launch_bounds__(PA_MERGE_THREADS) kl_paged_merge_kernel(const PagedView c, const PagedAttn a) {
    __shared__ float2 ml[PA_MAX_BLOCKS];
    __shared__ int end_s;
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const int b = (int)blockIdx.x, nb = (int)gridDim.x, tid = (int)threadIdx.x;
    const int4 meta = a.meta[b];
    const uint32_t s = (uint32_t)meta.y, ph = (uint32_t)meta.z, h = ph / a.HT, h0 = (ph - h * a.HT) * 8u, hh = blockIdx.y;
    if (!(meta.x & PA_SECOND) || h0 + hh >= a.G) return;
    if (tid == 0) end_s = nb - 1;
    __syncthreads();
    for (int i = b + 1 + tid; i < nb; i += PA_MERGE_THREADS)   // the last block that shares the pair
        if (!(a.meta[i].x & PA_FIRST_GOES_ON)) atomicMin(&end_s, i);
    __syncthreads();
    const int cnt = end_s - b + 1;
    auto slot = [&](int i) { return i == 0 ? (size_t)b * 2 + 1 : (size_t)(b + i) * 2; };
    for (int i = tid; i < cnt; i += PA_MERGE_THREADS) ml[i] = reinterpret_cast<const float2*>(a.part_ml)[slot(i) * 8 + hh];
    __syncthreads();
    float M = -INFINITY;
    for (int i = 0; i < cnt; ++i) M = fmaxf(M, ml[i].x);
    const float mu = M == -INFINITY ? 0.f : M;
    const uint32_t d = 2u * tid;
    if (d >= c.hd) return;
    float L = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll 8
    for (int i = 0; i < cnt; ++i) {
        const float f = pa_ex2(ml[i].x - mu);
        const float2 x = *reinterpret_cast<const float2*>(a.part + (slot(i) * 8 + hh) * c.hd + d);
        L += ml[i].y * f;
        v0 += x.x * f;
        v1 += x.y * f;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    pa_store2(c, a, s, h * a.G + h0 + hh, d, v0 * inv, v1 * inv);
    if (d == 0u) pa_store_lse(a, s, h * a.G + h0 + hh, M, L);
}

}  // namespace kl
