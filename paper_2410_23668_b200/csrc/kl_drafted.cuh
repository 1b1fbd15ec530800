// Kernels for drafted tokens on a paged cache (contracts in include/kl.h): append with the position rotation on the way, attention
// of a tree of new tokens.
#pragma once

#include "kl_paged_common.cuh"

namespace kl {

// ---- append with rotation

struct RotateArgs {
    const double* freqs;            // [hd / 2] radians per position
    const int32_t* row_positions;   // [n_rows] positions the angles go by, or null: where the rows lie
    const uint8_t* q;               // [n_rows][nq][hd], or null
    uint8_t* q_out;
    int64_t q_stride, q_out_stride; // bytes
    uint32_t nq;
    uint32_t kv_blocks;             // blocks of keys and values: units x head groups; the rest turn queries
    uint32_t heads, head_groups;    // kv heads of a block, blocks of a unit
    uint32_t q_heads, q_groups;     // query heads of a block, blocks of a run of rows
};

constexpr int RT_THREADS = 256;
constexpr int RT_ROWS = 16;   // rows whose angles a block holds at a time

// Rounded to 32 bits towards zero, the last bit set where something was cut off: a number that rounds to any type of fewer bits
// (22 at most) as the 64-bit one does.
__device__ __forceinline__ float rt_sticky(double x) {
    const float f = __double2float_rz(x);
    return __uint_as_float(__float_as_uint(f) | ((__double2loint(x) & 0x1fffffff) != 0 ? 1u : 0u));
}

// Eight consecutive elements as floats.
template <class T>
struct RtPiece {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const uint8_t* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t a[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = bf_lo(a[i]);
                x[2 * i + 1] = bf_hi(a[i]);
            }
        } else {
            const uint4 v = w[sizeof(T) / 2 - 1];
            const uint32_t b[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __uint_as_float(a[i]);
                x[4 + i] = __uint_as_float(b[i]);
            }
        }
    }
};

// One block = the rows of a call that fall into one page (as in kl_paged_append: block u of the units belongs to the sequence s with
// base(s) <= u, base(s) = row_starts[s] / page + 2 s), for `heads` kv heads, so that a page's bounds have one writer; or RT_ROWS
// rows' queries for `q_heads` query heads.  hd / 16 lanes share a row of a head, eight columns of either half each: a pair
// (i, i + hd / 2) that turns together is in one lane's hands.  Cosines and sines of RT_ROWS rows are computed once for all heads.
// Angles, cosines, sines and the two products of a key are held in 64 bits and the key is rounded once: a scale byte is a whole
// number, and whether a key passes a border between two scales or codes is a comparison that 32 bits get wrong now and then.
template <class T, int HD, bool FP8>
__global__ void __launch_bounds__(RT_THREADS) kl_paged_append_rotated_kernel(const PagedView c, const PagedRows rows, const RotateArgs a) {
    constexpr uint32_t LANES = HD / 16, GROUPS = RT_THREADS / LANES, HALF = HD / 2;
    extern __shared__ __align__(16) uint8_t rt_smem[];   // cosines and sines; at the end the groups' bounds
    __shared__ uint32_t found[4];
    __shared__ int32_t turn_s[RT_ROWS], live_s[RT_ROWS];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint32_t tid = threadIdx.x, grp = tid / LANES, lane = tid % LANES, col = lane * 8u;

    if (blockIdx.x >= a.kv_blocks) {   // queries
        const uint32_t b = blockIdx.x - a.kv_blocks, row0 = b / a.q_groups * RT_ROWS, h0 = b % a.q_groups * a.q_heads;
        const uint32_t n = min((uint32_t)RT_ROWS, rows.n_rows - row0), nh = min(a.q_heads, a.nq - h0);
        if (tid < RT_ROWS) live_s[tid] = 0;
        __syncthreads();
        if (!rows.row_starts) {
            if (tid < n) {
                const int32_t p = c.positions[row0 + tid];
                live_s[tid] = p >= 0;
                turn_s[tid] = a.row_positions ? a.row_positions[row0 + tid] : p;
            }
        } else {
            for (uint32_t s = tid; s < c.n_seqs; s += RT_THREADS) {
                const uint32_t x = pg_row_start(c, rows, s), y = pg_row_start(c, rows, s + 1u);
                if (x >= row0 + n || y <= row0) continue;
                const int32_t p = c.positions[s];
                if (p < 0) continue;
                for (uint32_t r = max(x, row0); r < min(y, row0 + n); ++r) {
                    live_s[r - row0] = 1;
                    turn_s[r - row0] = a.row_positions ? a.row_positions[r] : (int32_t)((uint32_t)p + (r - x));
                }
            }
        }
        __syncthreads();
        float2* cs = reinterpret_cast<float2*>(rt_smem);   // [row][hd / 2]
        for (uint32_t i = tid; i < n * HALF; i += RT_THREADS) {
            const uint32_t r = i / HALF;
            if (live_s[r]) {
                double sn, cn;
                sincos((double)turn_s[r] * a.freqs[i % HALF], &sn, &cn);
                cs[i] = make_float2((float)cn, (float)sn);
            }
        }
        __syncthreads();
        const uint32_t items = n * nh;
        for (uint32_t it = grp; it < items; it += GROUPS) {
            const uint32_t r = it / nh, h = h0 + it % nh;
            if (!live_s[r]) continue;
            const uint8_t* src = a.q + (int64_t)(row0 + r) * a.q_stride + ((size_t)h * HD + col) * sizeof(T);
            T* dst = reinterpret_cast<T*>(a.q_out + (int64_t)(row0 + r) * a.q_out_stride) + (size_t)h * HD + col;
            RtPiece<T> lo, hi;
            lo.load(src);
            hi.load(src + HALF * sizeof(T));
            float x[8], y[8], u[8], v[8];
            lo.get(x);
            hi.get(y);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float2 t = cs[r * HALF + col + q];
                u[q] = x[q] * t.x - y[q] * t.y;
                v[q] = y[q] * t.x + x[q] * t.y;
            }
            pg_store8<T>(dst, u);
            pg_store8<T>(dst + HALF, v);
        }
        return;
    }

    const uint32_t u = blockIdx.x / a.head_groups, h0 = blockIdx.x % a.head_groups * a.heads;
    uint32_t s = u, j = 0, r0 = u, r1 = u + 1u;
    int32_t pos;
    if (rows.row_starts) {
        if (blockIdx.x == 0u) pg_check_starts(c, rows);
        if (tid == 0u) found[0] = 0u;
        __syncthreads();
        uint32_t best = 0, b0 = 0, b1 = 0;
        int32_t bp = 0;
        for (uint32_t t = tid; t < c.n_seqs; t += RT_THREADS) {
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
        if (found[0] == 0u) return;
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
    const uint64_t p0 = (uint64_t)pos, p1 = p0 + (r1 - r0);
    const uint64_t lp = (uint64_t)((uint32_t)pos / c.page) + j, a0 = max(p0, lp * c.page), a1 = min(p1, (lp + 1u) * c.page);
    if (a0 >= a1) return;
    if (lp >= c.table_pages) {
        if (tid == 0u) pg_error(c);
        return;
    }
    const int32_t phys = pg_physical(c, s, (uint32_t)lp);
    if (phys < 0) return;

    const uint32_t off0 = (uint32_t)(a0 - lp * c.page), cnt = (uint32_t)(a1 - a0), row0 = r0 + (uint32_t)(a0 - p0);
    const uint32_t slots = GROUPS / a.heads, hs = grp % a.heads, rs = grp / a.heads, h = h0 + hs;   // `heads` is a power of two
    const bool mine = h < c.nkv;
    const int64_t head_at = (int64_t)phys * c.page_b + (int64_t)h * c.head_b + (int64_t)off0 * c.row_b + col * (FP8 ? 1 : 2);
    uint8_t* const kd = c.k + head_at;
    uint8_t* const vd = c.v + head_at;
    const int64_t exp_at = ((int64_t)phys * c.nkv + h) * c.page + off0;
    const size_t row_at = ((size_t)h * HD + col) * sizeof(T);
    __nv_bfloat16* const bounds = c.bounds ? c.bounds + ((int64_t)phys * c.nkv + h0) * 2 * HD : nullptr;
    float lo[16], hi[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        lo[i] = INFINITY;
        hi[i] = -INFINITY;
    }
    // sixteen columns of a row into the cache; `held` becomes what the cache stands for
    auto put = [&](float (&x)[16], uint8_t* dst, uint8_t* exps, uint32_t i, bool keep) {
        dst += (int64_t)i * c.row_b;
        if constexpr (FP8) {
            uint32_t big = 0u;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const uint32_t b = __float_as_uint(x[q]) & 0x7fffffffu;
                if (b < 0x7f800000u) big = max(big, b);   // infinities and NaN do not count
            }
#pragma unroll
            for (uint32_t o = LANES / 2u; o > 0u; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
            const uint32_t e = pg_exponent(big);
            const float inv = pg_inv_scale(e), scale = pg_scale(e);
            uint32_t code[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) code[q] = pg_to_e4m3x4(x[4 * q] * inv, x[4 * q + 1] * inv, x[4 * q + 2] * inv, x[4 * q + 3] * inv);
            if (keep) {
                *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[1]);
                *reinterpret_cast<uint2*>(dst + HALF) = make_uint2(code[2], code[3]);
                if (lane == 0u) exps[i] = (uint8_t)e;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float2 f = pg_f16x2_to_float2(pg_e4m3x2_to_f16x2(code[q / 2] >> 16 * (q & 1) & 0xffffu));
                x[2 * q] = f.x * scale;
                x[2 * q + 1] = f.y * scale;
            }
        } else {
            uint32_t v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = pack_bf16(x[2 * q], x[2 * q + 1]);
            if (keep) {
                *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint4*>(dst + HALF * 2) = make_uint4(v[4], v[5], v[6], v[7]);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                x[2 * q] = bf_lo(v[q]);
                x[2 * q + 1] = bf_hi(v[q]);
            }
        }
    };
    double2* cs = reinterpret_cast<double2*>(rt_smem);   // [row][hd / 2]
    for (uint32_t c0 = 0; c0 < cnt; c0 += RT_ROWS) {
        const uint32_t n = min((uint32_t)RT_ROWS, cnt - c0);
        __syncthreads();
        for (uint32_t i = tid; i < n * HALF; i += RT_THREADS) {
            const uint32_t r = i / HALF;
            const int32_t at = a.row_positions ? a.row_positions[row0 + c0 + r] : (int32_t)(a0 + c0 + r);
            double sn, cn;
            sincos((double)at * a.freqs[i % HALF], &sn, &cn);
            cs[i] = make_double2(cn, sn);
        }
        __syncthreads();
        for (uint32_t i0 = 0; i0 < n; i0 += slots) {   // every lane of a warp takes part in the shuffles
            const uint32_t r = min(i0 + rs, n - 1u), i = c0 + r;
            const bool keep = mine && i0 + rs < n;
            const size_t hat = mine ? row_at : 0;
            RtPiece<T> k0, k1, v0, v1;
            const uint8_t* ks = rows.k + (int64_t)(row0 + i) * rows.k_stride + hat;
            const uint8_t* vs = rows.v + (int64_t)(row0 + i) * rows.v_stride + hat;
            k0.load(ks);
            k1.load(ks + HALF * sizeof(T));
            v0.load(vs);
            v1.load(vs + HALF * sizeof(T));
            float x[8], y[8], w[16];
            k0.get(x);
            k1.get(y);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const double2 t = cs[r * HALF + col + q];
                const double dx = (double)x[q], dy = (double)y[q];
                w[q] = rt_sticky(fma(dx, t.x, -(dy * t.y)));
                w[8 + q] = rt_sticky(fma(dy, t.x, dx * t.y));
            }
            put(w, kd, FP8 ? c.ke + exp_at : nullptr, i, keep);
            if (bounds && keep)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    lo[q] = fminf(lo[q], w[q]);
                    hi[q] = fmaxf(hi[q], w[q]);
                }
            v0.get(x);
            v1.get(y);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                w[q] = x[q];
                w[8 + q] = y[q];
            }
            put(w, vd, FP8 ? c.ve + exp_at : nullptr, i, keep);
        }
    }
    if (!bounds) return;
    float* red = reinterpret_cast<float*>(rt_smem);   // [row slot][head][2][hd]
    __syncthreads();
    float* to = red + ((size_t)rs * a.heads + hs) * 2 * HD;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        to[col + q] = lo[q];
        to[HALF + col + q] = lo[8 + q];
        to[HD + col + q] = hi[q];
        to[HD + HALF + col + q] = hi[8 + q];
    }
    __syncthreads();
    const uint32_t heads = min(a.heads, c.nkv - h0);
    for (uint32_t t = tid; t < heads * 2 * HD; t += RT_THREADS) {
        const bool up = t % (2 * HD) >= (uint32_t)HD;
        float x = off0 == 0u ? (up ? -INFINITY : INFINITY) : __bfloat162float(bounds[t]);
        for (uint32_t k = 0; k < slots; ++k) {
            const float y = red[(size_t)k * a.heads * 2 * HD + t];
            x = up ? fmaxf(x, y) : fminf(x, y);
        }
        bounds[t] = up ? __float2bfloat16_ru(x) : __float2bfloat16_rd(x);   // exact but for e4m3 rows of scale bytes 0 .. 2
    }
}
template <int HD>
constexpr size_t rt_smem_bytes() {
    return (size_t)RT_ROWS * (HD / 2) * 16 > (size_t)RT_THREADS / (HD / 16) * 2 * HD * 4 ? (size_t)RT_ROWS * (HD / 2) * 16
                                                                                        : (size_t)RT_THREADS / (HD / 16) * 2 * HD * 4;
}

}  // namespace kl
