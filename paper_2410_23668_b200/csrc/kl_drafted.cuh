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

constexpr int RT_MANY = 512, RT_FEW = 256;   // threads of a block: several rows of a sequence, one row of each
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
//
// What bounds it: for few rows the chain of look-ups (position, page, rows) and the 64-bit sines, about 2 us of them (one row of eight
// kv and 32 query heads 4.4 us; 32 sequences of eight rows 7.8); for many the instructions of turning, scaling and packing with one block
// on an SM (8191 rows to e4m3 with 32 query heads 60 us, 173 MB in all and hence 26 at the copy rate).  All heads of a page in one block
// compute the angles once instead of per head; a row's loads are requested while the one before is worked on (66 us without).
template <class T, int HD, bool FP8, int RT_THREADS>
__global__ void __launch_bounds__(RT_THREADS, 1) kl_paged_append_rotated_kernel(const PagedView c, const PagedRows rows, const RotateArgs a) {
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
        for (uint32_t it0 = grp; it0 < items; it0 += 2u * GROUPS) {   // two rows' loads under way
            RtPiece<T> lo[2], hi[2];
            uint32_t r[2];
            T* dst[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const uint32_t it = it0 + z * GROUPS, h = h0 + it % nh;
                r[z] = it / nh;
                dst[z] = nullptr;
                if (it >= items || !live_s[r[z]]) continue;
                const uint8_t* src = a.q + (int64_t)(row0 + r[z]) * a.q_stride + ((size_t)h * HD + col) * sizeof(T);
                dst[z] = reinterpret_cast<T*>(a.q_out + (int64_t)(row0 + r[z]) * a.q_out_stride) + (size_t)h * HD + col;
                lo[z].load(src);
                hi[z].load(src + HALF * sizeof(T));
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                if (!dst[z]) continue;
                float x[8], y[8], u[8], v[8];
                lo[z].get(x);
                hi[z].get(y);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float2 t = cs[r[z] * HALF + col + q];
                    u[q] = x[q] * t.x - y[q] * t.y;
                    v[q] = y[q] * t.x + x[q] * t.y;
                }
                pg_store8<T>(dst[z], u);
                pg_store8<T>(dst[z] + HALF, v);
            }
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
    // a row of keys and of values, requested while the angles (or the row before) are worked on
    RtPiece<T> k0, k1, v0, v1;
    const size_t hat = mine ? row_at : 0;
    auto request = [&](uint32_t i) {
        const uint8_t* ks = rows.k + (int64_t)(row0 + i) * rows.k_stride + hat;
        const uint8_t* vs = rows.v + (int64_t)(row0 + i) * rows.v_stride + hat;
        k0.load(ks);
        k1.load(ks + HALF * sizeof(T));
        v0.load(vs);
        v1.load(vs + HALF * sizeof(T));
    };
    request(min(rs, cnt - 1u));
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
            float vx[8], vy[8];
            v0.get(vx);
            v1.get(vy);
            request(min(i0 + slots < n ? c0 + min(i0 + slots + rs, n - 1u) : c0 + RT_ROWS + rs, cnt - 1u));   // the next one
            put(w, kd, FP8 ? c.ke + exp_at : nullptr, i, keep);
            if (bounds && keep)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    lo[q] = fminf(lo[q], w[q]);
                    hi[q] = fmaxf(hi[q], w[q]);
                }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                w[q] = vx[q];
                w[8 + q] = vy[q];
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
template <int HD, int RT_THREADS>
constexpr size_t rt_smem_bytes() {
    return (size_t)RT_ROWS * (HD / 2) * 16 > (size_t)RT_THREADS / (HD / 16) * 2 * HD * 4 ? (size_t)RT_ROWS * (HD / 2) * 16
                                                                                        : (size_t)RT_THREADS / (HD / 16) * 2 * HD * 4;
}


// ---- attention of new tokens, a tree or a chain of them, over a paged cache
//
// For a (sequence, kv head) the queries of all new tokens and all G query heads of the group are rows of one matrix product with
// the cached keys, 128 at a time: S = Q K^T on the tensor cores (accumulators in TMEM), the softmax on S by the threads that own the
// rows, O += P V on the tensor cores again, with P read from TMEM.  A cached row thus leaves memory once for 128 (token, head) pairs, or 256.
//
// One pass over the keys with a running reference m of the exponent and the running sum l: p = 2^(s - m), l += p, O += p v; m is
// raised, and l and O scaled, only when a score exceeds it by TaCfg::RAISE binades -- until then p is larger than one, which 32-bit sums and
// the 16-bit types of P bear.
//
// The work of a call is one list of key tiles: sequences, kv heads, runs of up to 256 rows, tiles; every block of the grid (one per SM) takes
// an equal share of it.  A unit (sequence, head, run of rows) cut by the border between two blocks leaves its parts (O, m, l) in the
// workspace, and kl_paged_tree_merge_kernel joins them in order.
//
// Types.  bf16 caches: Q, K, V as they are, P as two bf16 parts (15 bits of it), both multiplied with V: one part alone would cost
// results 8 bits of every probability.  e4m3 caches: Q as f16, a row divided by a power of two (exact but for elements below 2^-28 of its
// largest), K's codes as f16 (exact), its scales applied to the scores in 32 bits; V's codes as f16 (exact), its scales applied to P, which
// enters as one f16 (11 bits) scaled by a power of two common to all columns so far (the largest value scale seen).
//
// Two streams.  There are two score buffers and two groups of four softmax warps, each with a reference, a sum and an O of its own.  Where a
// unit has at most 128 rows, the groups take its tiles in turn and are joined at its end; where it has up to 256, each group
// takes 128 rows of every tile.  Either way the tensor cores work for one group while the other has its softmax, no two groups have
// to agree on anything, and a tile's keys and values serve up to 256 rows.  With at most 64 (32) rows each row lies in TMEM's lanes
// twice (four times), and a copy takes one half (quarter) of the tile's keys -- P is zero elsewhere -- so that all warps share a
// single row's exponentials.  (Head size 256: O fills half of TMEM, one group of warps takes the buffers in turn, 128 rows.)
//
// Roles: 4 or 8 softmax warps (a thread owns a row), a warp that issues Q K^T, one that issues P V (a lone warp needs some five cycles per
// instruction and one matrix instruction 64: one warp for both fell behind), 4 (bf16: asynchronous copies) or 8 (e4m3: widened in
// registers) producers.
//
// What bounds it (head size 128, 8 kv heads).  Few rows over a bf16 cache: memory (32 x 8 tokens, four heads to a kv head, over 4096
// positions 123 us for 542 MB, 4.4 TB/s).  Many rows: the softmax -- with both groups at work 128 columns of a warp take some 4100 cycles
// beside the 3100 that a tile's matrix instructions take (24 trees of up to 32 tokens, eight heads, 308 us; the tensor cores 48 % busy;
// score buffers of 64 keys, two to a group, so that Q K^T runs ahead of the softmax: 348 where this form took 350, and slower elsewhere).
// Few rows over an e4m3 cache: the latency of a tile's way through all roles with two tiles under way (32 single tokens, window 2044: 84 us for
// 121 MB).  Small calls: the chain of look-ups, one tile and the join (five tokens over 700 positions 20.7 us).

struct TreeArgs {
    const int32_t* row_starts;      // [n_seqs + 1] or null: one row per sequence
    uint32_t n_rows;
    const uint8_t* q;               // bf16 [n_rows][nq][hd], strides in bytes
    uint8_t* out;
    int64_t q_stride, out_stride;
    uint32_t nq, G;
    float scale_log2;
    uint32_t window, sinks;
    const int32_t* row_positions;   // or null
    const uint32_t* mask;           // [n_rows][mask_words] or null
    uint32_t mask_words;
    float* lse;                     // [n_rows][nq] or null
    float* part;                    // [2 blocks][TA_RECORD][hd]
    float2* part_ml;                // [2 blocks][TA_RECORD]
};

constexpr int TA_MAX_BLOCKS = 160;
constexpr uint64_t TA_WAIT_NS = 2000000000ull;
constexpr int TA_RING = 8;          // tiles whose scale bytes (e4m3) are kept; also pieces whose ends are told apart

template <int HD, bool FP8>
struct TaCfg {
    static constexpr int NG = HD == 256 ? 1 : 2;              // groups of softmax warps
    static constexpr int NK = HD == 256 ? 64 : 128;           // keys of a tile
    static constexpr int PW = FP8 ? 8 : 4;                    // producer warps
    static constexpr int NW = 4 * NG + 2 + PW;                // softmax, two that issue matrix instructions, producers
    static constexpr int QK_WARP = 4 * NG, PV_WARP = 4 * NG + 1;
    static constexpr int SLOT = NK * HD * 2;
    static constexpr int NS = HD == 64 ? 8 : 4;
    static constexpr int QBYTES = 128 * HD * 2;               // of 128 rows
    static constexpr uint32_t O_COL = 2 * NK;                 // TMEM columns: two score buffers (P on them), an O for every group
    static constexpr int RAISE = FP8 ? 4 : 8;
};
constexpr float TA_HEAD = 10.f;     // e4m3: binades between P's largest (2^RAISE) and the largest f16 that stay free
constexpr int TA_RECORD = 256;      // rows of a part in the workspace

struct TaShared {
    alignas(16) float x[256 * 16];           // exchange between the parts of a row; before the first piece: prefix sums over the sequences
    alignas(16) float factor[8][2][128];     // per softmax warp: key scales (with the score scale), value scales
    float qscale[4][2][128];                 // e4m3: what a row's queries were divided by; pieces in turn (scores run up to two short pieces ahead)
    uint8_t exps[TA_RING][2][128];
    uint64_t wsum[18];
    float ml[3][256];                        // reference, sum and unit of the values of every softmax thread
    uint64_t kv_full[8], kv_empty[8], exp_full[TA_RING], piece_end[TA_RING];
    uint64_t q_full, q_empty, qs_full[4], o_empty, end;
    uint64_t scores[2], probs[2], done[2];   // per stream: Q K^T has landed, P is written, P V has landed
    uint32_t bad[TA_RING];                   // pieces whose partly visible tiles hold values that are no numbers
    uint32_t tmem;
    int abort;
};
template <int HD, bool FP8>
constexpr size_t ta_smem() {
    return 1024 + (size_t)TaCfg<HD, FP8>::NG * TaCfg<HD, FP8>::QBYTES + (size_t)TaCfg<HD, FP8>::NS * TaCfg<HD, FP8>::SLOT + sizeof(TaShared);
}

// A bounded wait of a whole warp; every lane gets the same answer.
__device__ __noinline__ bool ta_wait_on(uint32_t bar, uint32_t parity, int* abort, int32_t* status) {
    const uint64_t t0 = globaltimer_ns();
    bool done = false;
    for (uint32_t it = 1; !done; ++it) {
        done = mbar_try_wait(bar, parity);
        if (!done && (it & 63u) == 0u) {
            if (*(volatile int*)abort) break;
            if (globaltimer_ns() - t0 > TA_WAIT_NS) {
                if (status) atomicCAS(status, 0, ERR_SYNC_TIMEOUT);
                *(volatile int*)abort = 1;
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, done);
}
__device__ __forceinline__ bool ta_wait(uint64_t* bar, uint32_t parity, TaShared& s, int32_t* status) {
    const uint32_t b = smem_u32(bar);
    if (__all_sync(0xffffffffu, mbar_try_wait(b, parity))) return true;
    return ta_wait_on(b, parity, &s.abort, status);
}
__device__ __forceinline__ void tm_commit_to(uint64_t* bar) { tm_commit(smem_u32(bar)); }
// A barrier of the softmax warps, by its number.
__device__ __forceinline__ void ta_named_sync(uint32_t id, uint32_t threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ bool ta_named_all(uint32_t id, uint32_t threads, bool x) {   // ... and whether x holds for all of them
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbar.red.and.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(id), "r"(threads), "r"(x ? 1u : 0u) : "memory");
    return r != 0u;
}
__device__ __forceinline__ void ta_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ta_cp16(uint32_t dst, const void* src, uint32_t bytes) {   // bytes: 16, or 0 for zeros
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ta_st16(uint32_t dst, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void ta_tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void ta_tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void ta_tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void ta_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A B with both operands in shared memory, and with A in TMEM (lane = row, one column = two values of K).
__device__ __forceinline__ void ta_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
        "r"(acc)
        : "memory");
}
__device__ __forceinline__ void ta_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
        "r"(acc)
        : "memory");
}
// Descriptors of tiles stored as runs of 64 columns: [row][128 bytes], 16-byte pieces exchanged by the 128-byte swizzle, eight rows =
// 1024 bytes.  K-major (Q, K: the contraction runs along the 128 bytes): stride between groups of eight rows 1024.  MN-major (V: the
// contraction runs along the rows): `lead` bytes between runs of 64 columns, 1024 between groups of eight rows.
__device__ __forceinline__ uint64_t ta_desc(uint32_t smem_addr, uint32_t lead) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3ffffu) >> 4);
    d |= (uint64_t)(lead >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// kind::f16, fp32 accumulators, M = 128; type 1: bf16, 0: f16; B MN-major for V.
__device__ __forceinline__ constexpr uint32_t ta_idesc(uint32_t type, uint32_t N, bool b_mn) {
    return (1u << 4) | (type << 7) | (type << 10) | (b_mn ? 1u << 16 : 0u) | ((N >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ float ta_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two floats as f16 (x0 in the low half), nearest, saturating.
__device__ __forceinline__ uint32_t ta_pack_f16(float x0, float x1) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(x0), "f"(x1));
    return r;
}
// Two floats in one register pair.
__device__ __forceinline__ uint64_t ta_pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void ta_unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t ta_fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t ta_mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t ta_add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Sixteen bytes, or zeros (no branch around the load).
__device__ __forceinline__ uint4 ta_load_if(bool yes, const void* p) {
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((uint32_t)yes));
    return v;
}

// A sequence of the call.
struct TaSeq {
    uint32_t T, r0, base, len, lo;   // new tokens, their first row, cached positions, positions in all, first position of the window
    uint32_t tiles, head_tiles, first_tile, halves; // key tiles: head_tiles from position 0 on (sinks), the others from first_tile on; runs of 128 rows
};
template <int NK, int UR>
__device__ __forceinline__ TaSeq ta_seq(const PagedView& c, const TreeArgs& a, uint32_t s) {
    TaSeq q;
    q.T = 1u;
    q.r0 = s;
    if (a.row_starts) {
        const int32_t x = a.row_starts[s], y = a.row_starts[s + 1u];
        q.r0 = x < 0 ? 0u : min((uint32_t)x, a.n_rows);
        const uint32_t r1 = y < 0 ? 0u : min((uint32_t)y, a.n_rows);
        q.T = r1 > q.r0 ? r1 - q.r0 : 0u;
    }
    const int32_t pos = c.positions[s];
    q.base = pos < 0 ? 0u : (uint32_t)pos;
    if (pos < 0) q.T = 0u;
    const uint32_t most = c.table_pages * c.page;
    if (q.T > 0u && ((uint64_t)q.base + q.T > most)) {
        pg_error(c);
        q.base = min(q.base, most);
        q.T = min(q.T, most - q.base);
    }
    q.len = q.base + q.T;
    q.lo = a.window && q.base + 1u > a.window ? q.base + 1u - a.window : 0u;
    q.first_tile = q.lo / NK;
    q.head_tiles = q.lo ? min((min(a.sinks, q.base) + NK - 1u) / NK, q.first_tile) : 0u;
    q.tiles = q.T ? q.head_tiles + (q.len + NK - 1u) / NK - q.first_tile : 0u;
    q.halves = (uint32_t)(((uint64_t)q.T * a.G + 127u) / 128u);
    return q;
}
// What the shares are counted in: a tile of a unit of up to 128 rows is one, of more than 128 two -- it takes twice the matrix
// instructions and exponentials (24 trees of 1 .. 32 tokens, eight query heads to a kv head, 308 us; every tile one: 350).
__device__ __forceinline__ uint64_t ta_work(const PagedView& c, const TaSeq& q) { return (uint64_t)q.tiles * c.nkv * q.halves; }
// The unit that `off` lies in, counted from the sequence's first.
struct TaUnit {
    uint32_t h, row0, rows, twice;   // kv head, first row, rows, whether a tile counts two
    uint64_t begin;                  // in the same count as `off`
    __device__ __forceinline__ uint32_t tile_at(uint64_t at) const { return (uint32_t)(at - begin + twice >> twice); }   // first tile that begins at `at` or behind it
};
template <int UR>
__device__ __forceinline__ TaUnit ta_unit(const TreeArgs& a, const TaSeq& q, uint64_t off) {
    TaUnit u;
    const uint64_t k = pg_div(off, q.tiles);
    u.h = (uint32_t)pg_div(k, q.halves);
    uint32_t half = (uint32_t)(k - (uint64_t)u.h * q.halves);
    if (UR == 256) half &= ~1u;
    u.row0 = half * 128u;
    u.rows = (uint32_t)min((uint64_t)UR, (uint64_t)q.T * a.G - u.row0);
    u.twice = u.rows > 128u ? 1u : 0u;
    u.begin = ((uint64_t)u.h * q.halves + half) * q.tiles;
    return u;
}

// Equal shares of the list; block b's begins at border(b), with the first tile that begins there or behind it.
struct TaShares {
    uint64_t per;
    uint32_t rest, blocks;
    __device__ __forceinline__ TaShares(uint64_t work, uint32_t n) : per(pg_div(work, n)), blocks(n) { rest = (uint32_t)(work - per * n); }
    __device__ __forceinline__ uint64_t border(uint32_t b) const { return per * b + rest * b / blocks; }   // (rest and b below TA_MAX_BLOCKS + 1)
};

// One block's share of the list, piece by piece.
struct TaPiece {
    TaSeq q;
    uint32_t h, row0, t0, t1;   // kv head, first row of the unit among the (token, head) pairs, tiles
    uint32_t rows, slot;        // rows of the unit, part in the workspace (~0: the whole unit is here)
    bool two;                   // two runs of rows
    uint32_t split, R;          // copies of a row in TMEM's lanes, rows between them
};
template <int NK, int NW, int UR>
struct TaIter {
    uint32_t s;
    uint64_t off, left;
    bool begun;
    TaSeq q;
    // `g`: first tile of the share; all lanes of a warp
    __device__ __forceinline__ TaIter(const PagedView& c, const TreeArgs& a, const uint64_t* pre, uint64_t g, uint64_t count) : left(count), begun(false) {
        s = 0;
        off = 0;
        if (!count) return;
        const uint32_t share = pg_find<NW>(pre, g), per = (c.n_seqs + NW * 32u - 1u) / (NW * 32u);
        s = share * per;
        off = g - pre[share];
        q = ta_seq<NK, UR>(c, a, s);
    }
    __device__ __forceinline__ bool next(const PagedView& c, const TreeArgs& a, TaPiece& p) {
        for (;;) {   // (the last half of a tile that counts two is nobody's)
            if (!left) return false;
            while (off >= ta_work(c, q)) {
                off -= ta_work(c, q);
                if (++s >= c.n_seqs) return false;
                q = ta_seq<NK, UR>(c, a, s);
            }
            const TaUnit u = ta_unit<UR>(a, q, off);
            const uint64_t end = min(off + left, u.begin + ((uint64_t)q.tiles << u.twice));
            p.q = q;
            p.t0 = u.tile_at(off);
            p.t1 = u.tile_at(end);
            p.h = u.h;
            p.row0 = u.row0;
            p.rows = u.rows;
            p.two = p.rows > 128u;
            p.split = p.rows <= 32u && NK == 128 ? 4u : p.rows <= 64u ? 2u : 1u;   // a copy takes 32 keys or more
            p.R = 128u / p.split;
            p.slot = p.t0 == 0u && p.t1 == q.tiles ? ~0u : 2u * blockIdx.x + (begun ? 1u : 0u);
            begun = true;
            left -= end - off;
            off = end;
            if (p.t0 < p.t1) return true;
        }
    }
};
__device__ __forceinline__ uint32_t ta_tile_pos(const TaSeq& q, uint32_t t, uint32_t nk) {   // first position of tile t
    return (t < q.head_tiles ? t : q.first_tile + t - q.head_tiles) * nk;
}
// Whether the tokens of a sequence may see different parts of the tile at `pos`; far: largest position in the text minus the window.
__device__ __forceinline__ bool ta_mixed(const TreeArgs& a, const TaSeq& q, uint32_t pos, uint32_t nk, int64_t far) {
    return q.T > 1u && (pos + nk > q.base || (a.window && (int64_t)pos <= far));
}
// Largest position in the text of a sequence's tokens, minus the window (whole warps).
__device__ __forceinline__ int64_t ta_far(const TreeArgs& a, const TaSeq& q) {
    if (!a.window) return 0;
    int32_t m = (int32_t)(q.base + q.T - 1u);
    if (a.row_positions) {
        m = 0;
        for (uint32_t i = threadIdx.x & 31u; i < q.T; i += 32u) m = max(m, a.row_positions[q.r0 + i]);
        m = __reduce_max_sync(0xffffffffu, m);
    }
    return (int64_t)m - (int64_t)a.window;
}

// What a row sees.
struct TaRow {
    uint32_t base, T, i;            // cached positions, new tokens, the row's own number (T == 0: not a row)
    int32_t after;                  // cached positions up to this one are behind the window (-1: none)
    const uint32_t* mask;
};
// What a row sees of positions p .. p + 31, as bits.
__device__ __noinline__ uint32_t ta_sees(uint32_t p, uint32_t base, uint32_t T, uint32_t i, int32_t after, uint32_t sinks, uint32_t window, const uint32_t* mask,
                                         uint32_t mask_words) {
    if (!T) return 0u;
    uint32_t bits = 0xffffffffu;
    if (p + 32u > base) bits = p >= base ? 0u : 0xffffffffu >> (p + 32u - base);
    if ((int32_t)p <= after) {
        uint32_t old = (int32_t)p + 31 <= after ? 0u : 0xffffffffu << (uint32_t)(after + 1 - (int32_t)p);
        if (p < sinks) old |= p + 32u <= sinks ? 0xffffffffu : 0xffffffffu >> (p + 32u - sinks);
        bits &= old;
    }
    if (p + 32u > base && p < base + T) {   // new tokens j = j0 .. j0 + 31
        const int64_t j0 = (int64_t)p - base;
        uint32_t b;
        if (mask) {
            const int64_t w = j0 >> 5;      // floor
            const uint32_t lo = w >= 0 && w < mask_words ? mask[w] : 0u, hi = w + 1 >= 0 && w + 1 < mask_words ? mask[w + 1] : 0u;
            b = __funnelshift_r(lo, hi, (uint32_t)j0 & 31u);
        } else {
            const int64_t d = (int64_t)i - j0;   // j <= i
            b = d < 0 ? 0u : d >= 31 ? 0xffffffffu : 0xffffffffu >> (31u - (uint32_t)d);
            const int64_t e = d - (int64_t)window;   // j > i - window
            if (window && e >= 0) b &= e >= 31 ? 0u : 0xffffffffu << (uint32_t)(e + 1);
        }
        const int64_t end = (int64_t)T - j0;   // j < T
        if (end < 32) b &= 0xffffffffu >> (uint32_t)(32 - end);
        bits |= b & (j0 >= 0 ? 0xffffffffu : 0xffffffffu << (uint32_t)(-j0));
    }
    return bits;
}
__device__ __forceinline__ uint32_t ta_sees(const TreeArgs& a, const TaRow& w, uint32_t p) {
    return ta_sees(p, w.base, w.T, w.i, w.after, a.sinks, a.window, w.mask, a.mask_words);
}
__device__ __forceinline__ TaRow ta_row(const TreeArgs& a, const TaPiece& p, uint32_t r) {
    TaRow w = {};
    w.base = p.q.base;
    w.after = -1;
    if (r < p.rows) {
        w.T = p.q.T;
        w.i = (p.row0 + r) / a.G;
        if (a.mask) w.mask = a.mask + (size_t)(p.q.r0 + w.i) * a.mask_words;
        if (a.window) {
            const int64_t at = a.row_positions ? max((int64_t)a.row_positions[p.q.r0 + w.i], (int64_t)w.base) : (int64_t)w.base + w.i;
            w.after = (int32_t)max(at - (int64_t)a.window, (int64_t)-1);
        }
    }
    return w;
}

// e4m3 codes, sixteen at a time, as f16 (exact); `tidy`: codes that are no numbers become zero and are told of.
__device__ __forceinline__ bool ta_widen(const uint4& raw, uint4 (&to)[2], bool tidy) {
    uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w}, r[8];
    bool bad = false;
    if (tidy) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t nan = ((w[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // 0x7f alone carries into the sign
            if (nan) {
                bad = true;
                w[i] &= ~((nan >> 7) * 0xffu);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = pg_e4m3x2_to_f16x2(w[i / 2] >> 16 * (i & 1) & 0xffffu);
    to[0] = make_uint4(r[0], r[1], r[2], r[3]);
    to[1] = make_uint4(r[4], r[5], r[6], r[7]);
    return bad;
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(TaCfg<HD, FP8>::NW * 32, 1) kl_paged_tree_kernel(const PagedView c, const TreeArgs a) {
    using Cfg = TaCfg<HD, FP8>;
    constexpr int NG = Cfg::NG, NK = Cfg::NK, PW = Cfg::PW, NW = Cfg::NW, NS = Cfg::NS, UR = NG * 128;
    extern __shared__ uint8_t ta_raw[];
    const uint32_t raw = smem_u32(ta_raw), q_s = (raw + 1023u) & ~1023u, ring_s = q_s + NG * Cfg::QBYTES;
    TaShared& s = *reinterpret_cast<TaShared*>(ta_raw + (ring_s - raw) + (size_t)NS * Cfg::SLOT);
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    if (tid == 0u) {
        for (int i = 0; i < 8; ++i) {
            mbar_init(smem_u32(&s.kv_full[i]), FP8 ? PW : PW * 32);   // bf16: every producer thread's copies
            mbar_init(smem_u32(&s.kv_empty[i]), 1);
            mbar_init(smem_u32(&s.exp_full[i]), PW);
            mbar_init(smem_u32(&s.piece_end[i]), PW);
            s.bad[i] = 0u;
        }
        mbar_init(smem_u32(&s.q_full), PW);
        mbar_init(smem_u32(&s.q_empty), 1);
        mbar_init(smem_u32(&s.end), 2);
        mbar_init(smem_u32(&s.o_empty), 4 * NG);
        for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&s.qs_full[i]), PW);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s.scores[i]), 1);
            mbar_init(smem_u32(&s.probs[i]), 4);
            mbar_init(smem_u32(&s.done[i]), 1);
        }
        s.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        ta_fence_async();
    }
    griddep_wait();
    // All of TMEM is taken only when the kernel before has left its own, and the next one may begin only once this block has it: either
    // would otherwise wait for columns that the other holds while it waits for its end.
    if (warp == (uint32_t)Cfg::QK_WARP) tm_alloc(smem_u32(&s.tmem), 512);
    if (a.row_starts && blockIdx.x == 0u) {
        for (uint32_t i = tid; i < c.n_seqs; i += NW * 32) {
            const int32_t x = a.row_starts[i], y = a.row_starts[i + 1u];
            if (x < 0 || y < x || (uint32_t)y > a.n_rows) pg_error(c);
        }
    }
    uint64_t* const pre = reinterpret_cast<uint64_t*>(s.x);
    static_assert(sizeof(s.x) >= NW * 32 * 8 && alignof(TaShared) >= 16, "prefix sums");
    const bool stopped = pg_stopped(c);   // (a barrier of the whole block where there is a status word)
    const uint64_t work = stopped ? 0ull : pg_prefix<NW>(c.n_seqs, pre, s.wsum, [&](uint32_t i) { return ta_work(c, ta_seq<NK, UR>(c, a, i)); });
    __syncthreads();
    griddep_launch();
    tm_fence_after();
    const uint32_t tmem = s.tmem;
    const TaShares shares(work, gridDim.x);
    const uint64_t g0 = shares.border(blockIdx.x), g1 = shares.border(blockIdx.x + 1u);
    TaIter<NK, NW, UR> iter(c, a, pre, g0, g1 - g0);
    __syncthreads();   // the prefix sums have been read
    TaPiece p;

    if (warp > (uint32_t)Cfg::PV_WARP) {   // ---- producers: queries, keys, values into shared memory
        const uint32_t pw = warp - Cfg::PV_WARP - 1u;
        constexpr uint32_t RPW = NK / PW;                  // rows of a tile per warp, one per lane
        constexpr uint32_t CH = FP8 ? HD / 16 : HD / 8;    // 16-byte pieces of a row in the cache
        constexpr uint32_t STEPS = RPW * CH / 32;          // pieces per lane
        uint32_t slot = 0, use = 0, ntile = 0, npiece = 0;
        auto take_slot = [&]() { return use == 0u || ta_wait(&s.kv_empty[slot], (use - 1u) & 1u, s, c.status); };   // until it may be written
        auto next_slot = [&]() {
            if (++slot == NS) {
                slot = 0;
                ++use;
            }
        };
        // Page sizes and tiles are multiples of four rows: rows 4 g .. 4 g + 3 of the warp's share of a tile lie in one page.  The warp looks up
        // a chunk of CT tiles at a time, lane j GPT + g the page of group g of the chunk's tile j, and asks for the next chunk's pages
        // when it begins with one.
        constexpr uint32_t STEP_ROWS = 32 / CH;            // rows that the lanes' pieces of one step make up
        constexpr uint32_t GPT = RPW / 4, CT = 32 / GPT;   // groups of a tile, tiles of a chunk
        const uint32_t reciprocal = 0xffffffffu / c.page + 1u;
        const int32_t* table = nullptr;                    // of the piece's sequence
        int64_t lane_at = 0;                               // of the lane's pieces, behind their rows' group
        const uint32_t lane_row = lane / CH, lane_dst = lane % CH * (FP8 ? 2u : 1u) / 8u * (NK * 128u) + (pw * RPW + lane_row) * 128u +
                                                        ((lane % CH * (FP8 ? 2u : 1u) % 8u ^ (lane_row & 7u)) << 4);
        struct Look { int32_t phys; uint32_t x, off; };    // off == ~0: nothing to read
        auto look_up = [&](uint32_t t) {
            t += lane / GPT;
            Look k = {0, 0u, ~0u};
            if (t >= p.t1) return k;
            k.x = ta_tile_pos(p.q, t, NK) + pw * RPW + 4u * (lane % GPT);
            if (k.x >= p.q.len || (k.x + 3u < p.q.lo && k.x >= a.sinks)) return k;
            uint32_t lp = __umulhi(k.x, reciprocal);       // x / page, or one more
            if (lp * c.page > k.x) --lp;
            k.off = k.x - lp * c.page;
            k.phys = table[lp];
            return k;
        };
        // Of the chunk: where a lane's group lies in either pool (-1: nothing to read) and its scale bytes, with a mask of those that count;
        // groups all of whose rows are read.
        int64_t base = -1, ex = 0;
        uint32_t ex_mask = 0, clean = 0;
        auto read = [&](uint32_t x) { return x < p.q.len && (x >= p.q.lo || x < a.sinks); };
        auto place = [&](const Look& k) {
            base = -1;
            ex_mask = 0u;
            if (k.off != ~0u) {
                if ((uint32_t)k.phys >= c.n_pages) {
                    pg_error(c);
                } else {
                    base = (int64_t)k.phys * c.page_b + (int64_t)k.off * c.row_b;
                    if (FP8) ex = ((int64_t)k.phys * c.nkv + p.h) * c.page + k.off;
#pragma unroll
                    for (uint32_t j = 0; j < 4u; ++j)
                        if (read(k.x + j)) ex_mask |= 0xffu << 8 * j;
                }
            }
            clean = __ballot_sync(0xffffffffu, ex_mask == ~0u);
        };
        auto all_of = [&](uint32_t j) { return (clean >> j * GPT & (GPT == 32u ? ~0u : (1u << GPT % 32u) - 1u)) == (GPT == 32u ? ~0u : (1u << GPT % 32u) - 1u); };
        // Of the lane's piece of step i of the chunk's tile j, which begins at position x (-1: nothing to read).
        auto offset = [&](uint32_t i, uint32_t j, bool all, uint32_t x) {
            const int64_t o = __shfl_sync(0xffffffffu, base, j * GPT + (STEP_ROWS <= 4u ? i * STEP_ROWS / 4u : i * (STEP_ROWS / 4u) + lane_row / 4u));
            const int64_t to = o + lane_at + (i * STEP_ROWS & 3u ? (int64_t)(i * STEP_ROWS & 3u) * c.row_b : 0);
            if (all) return to;
            const uint32_t at = x + pw * RPW + i * STEP_ROWS + lane_row;
            return (o >= 0) & (at < p.q.len) & ((at >= p.q.lo) | (at < a.sinks)) ? to : (int64_t)-1;
        };
        // the unit's queries: row L of the first (second) 128 is row L % R (128 + L) of it
        auto load_queries = [&]() {
            if (npiece > 0u && !ta_wait(&s.q_empty, (npiece - 1u) & 1u, s, c.status)) return false;
            // PT threads to a row: its address is worked out once, and its pieces are under way together
            constexpr uint32_t PT = PW * 32 / 128, QC = HD / 8 / PT, B = FP8 ? 4u : 8u;
            const uint32_t me = pw * 32u + lane, L = me / PT, ch0 = me % PT * QC;
#pragma unroll 1
            for (uint32_t half = 0; half < (p.two ? 2u : 1u); ++half) {
                const uint32_t r = p.two ? half * 128u + L : L & p.R - 1u, gr = p.row0 + r, tok = gr / a.G;
                const uint8_t* src = r < p.rows ? a.q + (int64_t)(p.q.r0 + tok) * a.q_stride + ((size_t)(p.h * a.G + gr - tok * a.G) * HD + ch0 * 8u) * 2u : nullptr;
                float inv = 1.f;
                if constexpr (FP8) {   // as f16, divided by a power of two that brings the row's largest to 2^14 .. 2^15
                    uint32_t big = 0u, odd = 0u;
                    if (src)
#pragma unroll
                        for (uint32_t i = 0; i < QC; ++i) {
                            const uint4 v = reinterpret_cast<const uint4*>(src)[i];
                            big = pg_larger(pg_larger(big, v.x), pg_larger(v.y, pg_larger(v.z, v.w)));
                            odd |= (v.x & 0x7f807f80u) + 0x00800080u | (v.y & 0x7f807f80u) + 0x00800080u | (v.z & 0x7f807f80u) + 0x00800080u | (v.w & 0x7f807f80u) + 0x00800080u;
                        }
                    big = max(big & 0x7fffu, big >> 16 & 0x7fffu);
                    if (odd & 0x80008000u) big = 0x7f80u;   // infinities and NaN stay what they are
#pragma unroll
                    for (uint32_t o = PT / 2u; o > 0u; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
                    const int e = (int)(big >> 7);   // 1 .. 254 for numbers that are not tiny
                    if (e != 255 && e != 0) inv = pg_scale((uint32_t)min(268 - e, 254));
                    if (ch0 == 0u) s.qscale[npiece & 3u][half][L] = 1.f / inv;
                }
#pragma unroll 1
                for (uint32_t i0 = 0; i0 < QC; i0 += B) {
                    uint4 v[B];
#pragma unroll
                    for (uint32_t i = 0; i < B; ++i) v[i] = src ? reinterpret_cast<const uint4*>(src)[i0 + i] : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (uint32_t i = 0; i < B; ++i) {
                        const uint32_t ch = ch0 + i0 + i;
                        if constexpr (FP8) {
                            uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const __half2 h = __floats2half2_rn(bf_lo(w[j]) * inv, bf_hi(w[j]) * inv);
                                w[j] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        ta_st16(q_s + half * Cfg::QBYTES + ch / 8u * (128u * 128u) + L * 128u + ((ch % 8u ^ (L & 7u)) << 4), v[i]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0u) {
                mbar_arrive(smem_u32(&s.q_full));
                if (FP8) mbar_arrive(smem_u32(&s.qs_full[npiece & 3u]));
            }
            return true;
        };
        bool ok = true;
        while (ok && iter.next(c, a, p)) {
            table = c.table + (int64_t)iter.s * c.table_stride;
            lane_at = (int64_t)p.h * c.head_b + (int64_t)(lane_row & 3u) * c.row_b + lane % CH * 16u;
            Look next = look_up(p.t0);
            const int64_t far = ta_far(a, p.q);
            place(next);
            next = look_up(p.t0 + CT);
            uint32_t j = 0;   // tile of the chunk
            bool bad = false;
            if constexpr (!FP8) {
                for (uint32_t t = p.t0; ok && t < p.t1; ++t) {
                    if (j == CT) {
                        place(next);
                        next = look_up(t + CT);
                        j = 0;
                    }
                    const uint32_t x = ta_tile_pos(p.q, t, NK);
                    const bool mixed = ta_mixed(a, p.q, x, NK, far), all = all_of(j);
#pragma unroll 1
                    for (int kv = 0; ok && kv < 2; ++kv) {
                        ok = take_slot();
                        if (!ok) break;
                        const uint32_t dst = ring_s + slot * Cfg::SLOT + lane_dst, bar = smem_u32(&s.kv_full[slot]);
                        const uint8_t* src = kv ? c.v : c.k;
                        if (kv == 0 || !mixed) {
                            if (all) {
#pragma unroll
                                for (uint32_t i = 0; i < STEPS; ++i) ta_cp16((dst ^ (i * STEP_ROWS & 7u) << 4) + i * STEP_ROWS * 128u, src + offset(i, j, true, x), 16u);
                            } else
#pragma unroll
                            for (uint32_t i = 0; i < STEPS; ++i) {
                                const int64_t o = offset(i, j, false, x);
                                ta_cp16((dst ^ (i * STEP_ROWS & 7u) << 4) + i * STEP_ROWS * 128u, src + (o < 0 ? 0 : o), o < 0 ? 0u : 16u);
                            }
                            // every thread's arrival comes when its copies have
                            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                        } else {   // values that some row must not see: what is no number becomes zero here
                            constexpr uint32_t Z = STEPS < 8u ? STEPS : 8u;   // pieces under way
#pragma unroll
                            for (uint32_t i0 = 0; i0 < STEPS; i0 += Z) {
                                uint4 v[Z];
#pragma unroll
                                for (uint32_t z = 0; z < Z; ++z) {
                                    const int64_t o = offset(i0 + z, j, false, x);
                                    v[z] = ta_load_if(o >= 0, src + o);
                                }
#pragma unroll
                                for (uint32_t z = 0; z < Z; ++z) {
                                    const uint32_t i = i0 + z;
                                    auto odd = [](uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; };   // carries where an exponent is all ones
                                    if ((odd(v[z].x) | odd(v[z].y) | odd(v[z].z) | odd(v[z].w)) & 0x80008000u) {
                                        uint32_t w[4] = {v[z].x, v[z].y, v[z].z, v[z].w};
#pragma unroll
                                        for (int j = 0; j < 4; ++j) {
                                            if ((w[j] & 0x7f80u) == 0x7f80u) w[j] &= 0xffff0000u;
                                            if ((w[j] & 0x7f800000u) == 0x7f800000u) w[j] &= 0xffffu;
                                        }
                                        v[z] = make_uint4(w[0], w[1], w[2], w[3]);
                                        bad = true;
                                    }
                                    ta_st16((dst ^ (i * STEP_ROWS & 7u) << 4) + i * STEP_ROWS * 128u, v[z]);
                                }
                            }
                            mbar_arrive(bar);
                        }
                        next_slot();
                    }
                    ++j;
                    // (behind the first tile's copies, which are then under way)
                    if (t == p.t0) ok = ok && load_queries();
                }
            } else {
                // The next tile's loads are under way while one is widened.
                uint4 kraw[STEPS], vraw[STEPS];
                uint32_t ke = 0, ve = 0;
                int64_t at[STEPS];
                auto aim = [&](uint32_t t) {
                    const bool all = all_of(j);
                    const uint32_t x = t < p.t1 ? ta_tile_pos(p.q, t, NK) : 0u;
#pragma unroll
                    for (uint32_t i = 0; i < STEPS; ++i) at[i] = offset(i, j, all, x);
                };
                auto request = [&](const uint8_t* src, uint4 (&to)[STEPS]) {
#pragma unroll
                    for (uint32_t i = 0; i < STEPS; ++i) to[i] = ta_load_if(at[i] >= 0, src + at[i]);
                };
                auto request_scales = [&]() {   // of four rows; a row that nobody sees gets the smallest
                    ke = ve = 0;
                    if (ex_mask) {
                        ke = *reinterpret_cast<const uint32_t*>(c.ke + ex);
                        ve = *reinterpret_cast<const uint32_t*>(c.ve + ex);
                    }
                };
                aim(p.t0);
                request(c.k, kraw);
                request_scales();
                request(c.v, vraw);
                ok = load_queries();   // (while the first tile's loads are under way)
                for (uint32_t t = p.t0; ok && t < p.t1; ++t) {
                    const bool mixed = ta_mixed(a, p.q, ta_tile_pos(p.q, t, NK), NK, far);
                    if (lane / GPT == j) {
                        *reinterpret_cast<uint32_t*>(&s.exps[ntile % TA_RING][0][pw * RPW + lane % GPT * 4u]) = ke & ex_mask;
                        *reinterpret_cast<uint32_t*>(&s.exps[ntile % TA_RING][1][pw * RPW + lane % GPT * 4u]) = ve & ex_mask;
                    }
                    __syncwarp();
                    if (lane == 0u) mbar_arrive(smem_u32(&s.exp_full[ntile % TA_RING]));
                    if (++j == CT) {   // tile t + 1 begins a chunk
                        place(next);
                        request_scales();
                        next = look_up(t + 1u + CT);
                        j = 0;
                    }
                    aim(t + 1u);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        ok = ok && take_slot();
                        if (!ok) break;
                        const uint32_t dst = ring_s + slot * Cfg::SLOT + lane_dst;
#pragma unroll
                        for (uint32_t i = 0; i < STEPS; ++i) {
                            uint4 w[2];
                            if (kv == 0) ta_widen(kraw[i], w, false);
                            else bad |= ta_widen(vraw[i], w, mixed);
                            ta_st16((dst ^ (i * STEP_ROWS & 7u) << 4) + i * STEP_ROWS * 128u, w[0]);
                            ta_st16((dst ^ (i * STEP_ROWS & 7u) << 4 ^ 16u) + i * STEP_ROWS * 128u, w[1]);
                        }
                        __syncwarp();
                        if (lane == 0u) mbar_arrive(smem_u32(&s.kv_full[slot]));
                        next_slot();
                        if (kv == 0) {
                            request(c.k, kraw);
                        } else {
                            request(c.v, vraw);
                        }
                    }
                    ++ntile;
                }
            }
            if (bad) atomicOr(&s.bad[npiece % TA_RING], 1u);
            __syncwarp();
            if (lane == 0u) mbar_arrive(smem_u32(&s.piece_end[npiece % TA_RING]));
            ++npiece;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= (uint32_t)Cfg::QK_WARP) {   // ---- matrix instructions: one warp for Q K^T, one for P V
        // A lone warp takes some five cycles per instruction, and 64 a matrix instruction: hence two warps, descriptors made once per
        // tile, and no loops around the instructions.
        constexpr uint32_t type = FP8 ? 0u : 1u, qk_idesc = ta_idesc(type, NK, false), pv_idesc = ta_idesc(type, HD, true);
        uint32_t tile = 0, npiece = 0, n0 = 0, n1 = 0;   // tiles, units and every stream's tiles so far
        bool ok = true;
        auto landed = [&](uint32_t n) {   // slot of the ring that is the n-th to be filled
            if (!ta_wait(&s.kv_full[n % NS], n / NS & 1u, s, c.status)) return false;
            ta_fence_async();   // what the barrier tells of was written by threads (who do not fence themselves: it would wait for their next loads)
            return true;
        };
        if (warp == (uint32_t)Cfg::QK_WARP) {
            while (ok && iter.next(c, a, p)) {
                ok = ta_wait(&s.q_full, npiece & 1u, s, c.status);
                ta_fence_async();
                for (uint32_t t = p.t0; ok && t < p.t1; ++t, ++tile) {
                    if (!(ok = landed(2u * tile))) break;
                    const uint32_t sl = 2u * tile % NS, b0 = p.two ? 0u : t - p.t0 & 1u, b1 = p.two ? 1u : b0;
                    const uint64_t kd = ta_desc(ring_s + sl * Cfg::SLOT, 16u);
#pragma unroll 1
                    for (uint32_t b = b0; b <= b1; ++b) {
                        uint32_t& n = b ? n1 : n0;
                        if (n > 0u && !(ok = ta_wait(&s.done[b], n - 1u & 1u, s, c.status))) break;   // P on this score buffer has been read
                        ++n;
                        tm_fence_after();
                        if (lane == 0u) {
                            const uint64_t qd = ta_desc(q_s + (p.two ? b : 0u) * Cfg::QBYTES, 16u);
                            const uint32_t to = tmem + b * NK;
#pragma unroll
                            for (uint32_t k = 0; k < HD / 16; ++k)   // 32 bytes along the swizzled rows, then the next 64 columns
                                ta_mma_ss(to, qd + (k / 4u * (128u * 128u / 16u) + k % 4u * 2u), kd + (k / 4u * (NK * 128u / 16u) + k % 4u * 2u), qk_idesc, k > 0u);
                            tm_commit_to(&s.scores[b]);
                            if (b == b1) {
                                tm_commit_to(&s.kv_empty[sl]);
                                if (t + 1u == p.t1) tm_commit_to(&s.q_empty);
                            }
                        }
                        __syncwarp();
                    }
                }
                ++npiece;
            }
        } else {
            while (ok && iter.next(c, a, p)) {
                if (npiece > 0u) ok = ta_wait(&s.o_empty, (npiece - 1u) & 1u, s, c.status);   // the last unit's result has been read
                for (uint32_t t = p.t0; ok && t < p.t1; ++t, ++tile) {
                    const uint32_t sl = (2u * tile + 1u) % NS, b0 = p.two ? 0u : t - p.t0 & 1u, b1 = p.two ? 1u : b0;
                    const uint64_t vd = ta_desc(ring_s + sl * Cfg::SLOT, NK * 128u);
                    const uint32_t acc = t > p.t0 + (p.two || NG == 1 ? 0u : 1u);
                    if (!(ok = landed(2u * tile + 1u))) break;
#pragma unroll 1
                    for (uint32_t b = b0; b <= b1; ++b) {
                        uint32_t& n = b ? n1 : n0;
                        if (!(ok = ta_wait(&s.probs[b], n & 1u, s, c.status))) break;
                        ++n;
                        tm_fence_after();
                        if (lane == 0u) {
                            const uint32_t d = tmem + Cfg::O_COL + (NG == 2 ? b * HD : 0u), pa = tmem + b * NK;
#pragma unroll
                            for (uint32_t k = 0; k < NK / 16; ++k) {
                                ta_mma_ts(d, pa + k * 16u, vd + k * (2048u / 16u), pv_idesc, k > 0u ? 1u : acc);
                                if (!FP8) ta_mma_ts(d, pa + k * 16u + 8u, vd + k * (2048u / 16u), pv_idesc, 1u);
                            }
                            if (b == b1) tm_commit_to(&s.kv_empty[sl]);
                            tm_commit_to(&s.done[b]);
                        }
                        __syncwarp();
                    }
                }
                ++npiece;
            }
        }
        // nothing may still be under way when TMEM is given back
        if (lane == 0u) tm_commit_to(&s.end);
        __syncwarp();
        ta_wait(&s.end, 0u, s, c.status);
    } else {   // ---- softmax and results: thread L of a group owns TMEM lane L
        const uint32_t grp = warp >> 2, L = tid & 127u, lane_base = tmem + ((warp & 3u) * 32u << 16), o_at = lane_base + Cfg::O_COL + grp * HD;
        float(&kf)[128] = s.factor[warp][0];
        float(&vf)[128] = s.factor[warp][1];
        uint32_t tile = 0, npiece = 0, n0 = 0, n1 = 0;   // tiles of the block, units and every stream's tiles so far
        bool ok = true;
        while (ok && iter.next(c, a, p)) {
            const uint32_t R = p.R, r = p.two ? grp * 128u + L : L % R, share = L / R;
            const uint32_t ncol = p.two ? (uint32_t)NK : (uint32_t)NK / p.split, col0 = p.two ? 0u : share * ncol, col1 = col0 + ncol;
            const TaRow row = ta_row(a, p, r);
            const bool active = __any_sync(0xffffffffu, row.T > 0u);
            float m = -INFINITY, l = 0.f, qs = 1.f;
            int ev_ref = -1;   // e4m3: the largest value scale byte so far
            if (FP8) {
                ok = ta_wait(&s.qs_full[npiece & 3u], npiece >> 2 & 1u, s, c.status);
                qs = s.qscale[npiece & 3u][p.two ? grp : 0u][L];
            }
            const float unit_s = FP8 ? qs : a.scale_log2;
            const uint64_t sc2 = ta_pair(unit_s, unit_s), minus = ta_pair(-1.f, -1.f);
            const uint32_t step = p.two || NG == 1 ? 1u : 2u, first = p.two || NG == 1 ? p.t0 : p.t0 + grp;   // this group's tiles
            for (uint32_t t = first; ok && t < p.t1; t += step) {
                const uint32_t b = NG == 2 ? grp : t - p.t0 & 1u, pos = ta_tile_pos(p.q, t, NK), s_at = lane_base + b * NK, nt = tile + (t - p.t0);
                uint32_t& n = b ? n1 : n0;
                if (FP8 && !(ok = ta_wait(&s.exp_full[nt % TA_RING], (nt / TA_RING) & 1u, s, c.status))) break;
                if (!(ok = ta_wait(&s.scores[b], n & 1u, s, c.status))) break;
                ++n;
                tm_fence_after();
                if (active) {
                    float raise = 1.f;   // of O: by a new reference of the values' scales
                    if constexpr (FP8) {
                        const uint32_t kw = *reinterpret_cast<const uint32_t*>(&s.exps[nt % TA_RING][0][lane * 4u % NK]);
                        const uint32_t vw = *reinterpret_cast<const uint32_t*>(&s.exps[nt % TA_RING][1][lane * 4u % NK]);
                        int mx = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) mx = max(mx, (int)(vw >> 8 * j & 0xffu));
                        mx = (int)__reduce_max_sync(0xffffffffu, (unsigned)mx);
                        if (mx > ev_ref) {
                            raise = ev_ref < 0 ? 0.f : ta_exp2((float)(ev_ref - mx));
                            ev_ref = mx;
                        }
                        __syncwarp();
                        if (lane * 4u < (uint32_t)NK) {
                            float k4[4], v4[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                k4[j] = pg_scale(kw >> 8 * j & 0xffu) * a.scale_log2;
                                v4[j] = ta_exp2((float)((int)(vw >> 8 * j & 0xffu) - ev_ref) + TA_HEAD);
                            }
                            *reinterpret_cast<float4*>(&kf[lane * 4u]) = make_float4(k4[0], k4[1], k4[2], k4[3]);
                            *reinterpret_cast<float4*>(&vf[lane * 4u]) = make_float4(v4[0], v4[1], v4[2], v4[3]);
                        }
                        __syncwarp();
                    }
                    auto ta_scale_o = [&](float f) {   // O times f; the last product must have landed (two groups: these scores came behind it)
                        if (NG == 1 && !ta_wait(&s.done[b ^ 1u], (b ? n0 : n1) - 1u & 1u, s, c.status)) return false;
                        tm_fence_after();
#pragma unroll 1
                        for (uint32_t c0 = 0; c0 < (uint32_t)HD; c0 += 16u) {
                            uint32_t x[16];
                            tm_ld16(o_at + c0, x);
                            tm_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) x[j] = __float_as_uint(f == 0.f ? 0.f : __uint_as_float(x[j]) * f);
                            ta_tmem_st16(o_at + c0, x);
                        }
                        return true;
                    };
                    // whether every row of the warp sees all of the tile
                    const bool full = __all_sync(0xffffffffu, row.T == 0u || (pos + NK <= row.base && (int32_t)pos > row.after));
                    // 32 columns at a time: scores to probabilities, on which P is written: of 16 columns the first eight hold the high halves
                    // (f16: all), the others the low ones
                    uint64_t sum[2] = {0ull, 0ull};
                    uint64_t ref2 = ta_pair(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m);
                    if (FP8 && raise != 1.f && t > first) ok = ta_scale_o(raise);
#pragma unroll 1
                    for (uint32_t c0 = col0; ok && c0 < col1; c0 += 32u) {
                        uint32_t x[32];
                        tm_ld32(s_at + c0, x);
                        tm_ld_wait();
                        if (!full) {   // what the row does not see is -infinity
                            const uint32_t sees = ta_sees(a, row, pos + c0);
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(sees >> j & 1u)) x[j] = 0xff800000u;
                        }
                        if constexpr (FP8) {
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {   // (scales are positive: -infinity stays)
                                const ulonglong2 ks = *reinterpret_cast<const ulonglong2*>(&kf[c0 + j]);
#pragma unroll
                                for (int i = 0; i < 4; i += 2) {
                                    float y0, y1;
                                    ta_unpair(ta_mul2(ta_pair(__uint_as_float(x[j + i]), __uint_as_float(x[j + i + 1])), i ? ks.y : ks.x), y0, y1);
                                    x[j + i] = __float_as_uint(y0);
                                    x[j + i + 1] = __float_as_uint(y1);
                                }
                            }
                        }
                        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            top[0] = pg_max3(top[0], __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
                            top[1] = pg_max3(top[1], __uint_as_float(x[j + 2]), __uint_as_float(x[j + 3]));
                        }
                        const float mx = fmaxf(top[0], top[1]) * unit_s;
                        // (scores of 2^22 and more: a step of the reference is as large as the slack, and no score may lie above it)
                        const bool rise = mx > m + (fabsf(m) < 4194304.f ? (float)Cfg::RAISE : 0.f);
                        if (__any_sync(0xffffffffu, rise)) {   // seldom but for the first tile
                            float g = 1.f;
                            if (rise) {
                                if (m == -INFINITY || fabsf(mx) >= 4194304.f) {
                                    g = 0.f;
                                    if (m > -INFINITY) g = ta_exp2(m - mx);
                                    m = fabsf(mx) >= 4194304.f ? fmaf(fabsf(mx), 1.2e-7f, mx) : mx;
                                } else {   // by whole binades: what is written of P stays exact
                                    const float k = ceilf(mx - m);
                                    m += k;
                                    g = ta_exp2(-k);
                                }
                            }
                            ref2 = ta_pair(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m);
                            l *= g;
                            sum[0] = ta_mul2(sum[0], ta_pair(g, g));
                            sum[1] = ta_mul2(sum[1], ta_pair(g, g));
                            for (uint32_t d0 = col0; d0 < c0; d0 += 16u) {   // P of this tile so far
                                uint32_t w[16];
                                tm_ld16(s_at + d0, w);
                                tm_ld_wait();
#pragma unroll
                                for (int j = 0; j < (FP8 ? 8 : 16); ++j) {
                                    if constexpr (FP8) {
                                        const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&w[j]), __float2half2_rn(g));
                                        w[j] = *reinterpret_cast<const uint32_t*>(&h);
                                    } else {
                                        w[j] = pg_mul_bf16x2(w[j], __float_as_uint(g) >> 16 | (__float_as_uint(g) & 0xffff0000u));
                                    }
                                }
                                ta_tmem_st16(s_at + d0, w);
                            }
                            if (t > first && !(ok = ta_scale_o(g))) break;
                        }
                        uint32_t h[FP8 ? 16 : 32];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float y0, y1;
                            ta_unpair(ta_fma2(ta_pair(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), sc2, ref2), y0, y1);
                            const uint64_t e = ta_pair(ta_exp2(y0), ta_exp2(y1));
                            sum[j & 1] = ta_add2(sum[j & 1], e);
                            if constexpr (FP8) {
                                const uint64_t vs = *reinterpret_cast<const uint64_t*>(&vf[c0 + 2 * j]);
                                ta_unpair(ta_mul2(e, vs), y0, y1);
                                h[j] = ta_pack_f16(y0, y1);
                            } else {
                                ta_unpair(e, y0, y1);
                                // the upper 16 bits of p, and what they leave, rounded (no conversion instructions: they run on the unit that has
                                // the exponentials to do)
                                const uint32_t u0 = __float_as_uint(y0), u1 = __float_as_uint(y1);
                                h[j / 8 * 16 + j % 8] = __byte_perm(u0, u1, 0x7632);
                                ta_unpair(ta_fma2(ta_pair(__uint_as_float(u0 & 0xffff0000u), __uint_as_float(u1 & 0xffff0000u)), minus, e), y0, y1);
                                h[j / 8 * 16 + 8 + j % 8] = __byte_perm(__float_as_uint(y0) + 0x8000u, __float_as_uint(y1) + 0x8000u, 0x7632);
                            }
                        }
                        if constexpr (FP8) {
                            const uint32_t h0[8] = {h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]}, h1[8] = {h[8], h[9], h[10], h[11], h[12], h[13], h[14], h[15]};
                            ta_tmem_st8(s_at + c0, h0);
                            ta_tmem_st8(s_at + c0 + 16u, h1);
                        } else {
                            ta_tmem_st32(s_at + c0, h);
                        }
                    }
                    if (!ok) break;
                    if (p.split > 1u) {   // the other copies' columns are zero
                        uint32_t zero[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) zero[j] = 0u;
#pragma unroll 1
                        for (uint32_t c0 = 0; c0 < (uint32_t)NK; c0 += 16u)
                            if (c0 < col0 || c0 >= col1) ta_tmem_st16(s_at + c0, zero);
                    }
                    float s0, s1;
                    ta_unpair(ta_add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    ta_tmem_st_wait();
                }
                tm_fence_before();
                __syncwarp();
                if (lane == 0u) mbar_arrive(smem_u32(&s.probs[b]));
            }
            tile += p.t1 - p.t0;
            const bool any = first < p.t1;   // whether this group had a tile
            if (ok && any) {
                const uint32_t b = NG == 2 ? grp : p.t1 - 1u - p.t0 & 1u;
                ok = ta_wait(&s.done[b], (b ? n1 : n0) - 1u & 1u, s, c.status);
            }
            ok = ok && ta_wait(&s.piece_end[npiece % TA_RING], (npiece / TA_RING) & 1u, s, c.status);
            if (!(ok = ta_named_all(3u, NG * 128u, ok))) break;   // (no softmax warp waits for one that has given up)
            tm_fence_after();
            const bool bad = *(volatile uint32_t*)&s.bad[npiece % TA_RING] != 0u;
            const float unit = FP8 && ev_ref >= 0 ? ta_exp2((float)(ev_ref - 127) - TA_HEAD) : 1.f;   // of the values
            // the parts of a row: one reference, one sum (units of one run: thread g * 128 + j * R + r holds part (g, j) of row r)
            const uint32_t me = grp * 128u + L;
            float mm = m, ll = l;
            s.ml[0][me] = m;
            s.ml[1][me] = l;
            s.ml[2][me] = unit;
            ta_named_sync(3u, NG * 128u);
            if (bad && me == 0u) s.bad[npiece % TA_RING] = 0u;
            if (!p.two) {
                constexpr uint32_t PARTS = NG * 4;   // fewer where a row has fewer copies
                float mk[PARTS], lk[PARTS];
#pragma unroll
                for (uint32_t k = 0; k < PARTS; ++k) {
                    const uint32_t at = k / 4u * 128u + k % 4u * R + r;
                    const bool is = k % 4u < p.split;
                    mk[k] = is ? s.ml[0][at] : -INFINITY;
                    lk[k] = is ? s.ml[1][at] : 0.f;
                }
                mm = mk[0];
#pragma unroll
                for (uint32_t k = 1; k < PARTS; ++k) mm = fmaxf(mm, mk[k]);
                ll = 0.f;
#pragma unroll
                for (uint32_t k = 0; k < PARTS; ++k) ll += mk[k] > -INFINITY ? lk[k] * ta_exp2(mk[k] - mm) : 0.f;
            }
            const bool whole = p.slot == ~0u, valid = r < p.rows;
            const uint32_t tok = row.i, head = p.h * a.G + p.row0 + r - tok * a.G;
            if (valid && (p.two || me == r)) {
                if (whole) {
                    if (a.lse) a.lse[(size_t)(p.q.r0 + tok) * a.nq + head] = ll > 0.f || ll != ll ? (mm + log2f(ll)) * 0.6931471805599453f : -INFINITY;
                } else {
                    a.part_ml[(size_t)p.slot * TA_RECORD + r] = make_float2(mm, ll);
                }
            }
            const float norm = whole ? (ll > 0.f || ll != ll ? 1.f / ll : 0.f) : 1.f;
            __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(a.out + (int64_t)(p.q.r0 + tok) * a.out_stride) + (size_t)head * HD;
            float* const rec = a.part + ((size_t)(whole ? 0u : p.slot) * TA_RECORD + r) * HD;
            auto put = [&](uint32_t at, const float (&y)[8]) {
                if (whole) pg_store8<__nv_bfloat16>(out + at, y);
                else pg_store8<float>(rec + at, y);
            };
            // Units of one run: both groups' O of a lane can be read by either, so each takes half of the columns of both.
            const bool pair = NG == 2 && !p.two, other = pair && p.t1 - p.t0 > 1u;   // (a single tile is the first group's)
            float f[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t w = pair ? k * 128u + L : me;
                f[k] = s.ml[0][w] == -INFINITY ? 0.f : ta_exp2(s.ml[0][w] - mm) * s.ml[2][w] * norm;
            }
            const uint32_t first_o = pair ? lane_base + Cfg::O_COL : o_at, c_end = pair ? (grp + 1u) * (HD / 2) : (uint32_t)HD;
            // The exchange between copies: `wide` columns of every valid row's copies at a time, as many as the group's 8 KB hold; their fours are
            // exchanged so that eight threads' lie in all banks.  (Head size 64: a group has 32 columns.)
            const uint32_t wide = p.rows <= 8u && HD > 64 ? 64u : p.rows <= 16u ? 32u : 16u, turn = wide == 16u ? r >> 1 & 3u : r & 7u;
            float* const xs = s.x + grp * 2048u + (share * (wide == 16u ? R : p.rows) + r) * wide;
            const float* const xr = s.x + grp * 2048u + r * wide;
#pragma unroll 1
            for (uint32_t c0 = pair ? grp * (HD / 2) : 0u; c0 < c_end; c0 += 16u) {
                uint32_t x[16];
                float o[16];
                tm_ld16(first_o + c0, x);
                if (other) {
                    uint32_t y[16];
                    tm_ld16(first_o + HD + c0, y);
                    tm_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = __uint_as_float(x[j]) * f[0] + __uint_as_float(y[j]) * f[1];
                } else {
                    tm_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = __uint_as_float(x[j]) * f[0];
                }
                if (bad && valid) {   // values that are no numbers, for the rows that see them
                    for (uint32_t t = p.t0; t < p.t1; ++t) {
                        const uint32_t pos = ta_tile_pos(p.q, t, NK);
                        if (!ta_mixed(a, p.q, pos, NK, INT32_MAX)) continue;
                        for (uint32_t k0 = col0; k0 < col1; k0 += 32u) {
                            uint32_t sees = ta_sees(a, row, pos + k0);
                            while (sees) {
                                const uint32_t at = pos + k0 + __ffs(sees) - 1u;
                                sees &= sees - 1u;
                                const int32_t phys = pg_physical(c, iter.s, at / c.page);
                                if (phys < 0) continue;
                                const uint8_t* v = c.v + (int64_t)phys * c.page_b + (int64_t)p.h * c.head_b + (int64_t)(at % c.page) * c.row_b;
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    const uint32_t w = FP8 ? v[c0 + j] : reinterpret_cast<const uint16_t*>(v)[c0 + j];
                                    if (FP8 ? (w & 0x7fu) == 0x7fu : (w & 0x7f80u) == 0x7f80u) o[j] += FP8 ? NAN : __uint_as_float(w << 16);
                                }
                            }
                        }
                    }
                }
                if (p.two || p.split == 1u) {
                    if (valid) {
#pragma unroll
                        for (int j = 0; j < 16; j += 8) {
                            const float y[8] = {o[j], o[j + 1], o[j + 2], o[j + 3], o[j + 4], o[j + 5], o[j + 6], o[j + 7]};
                            put(c0 + j, y);
                        }
                    }
                    continue;
                }
                const uint32_t in = c0 % wide;
                if (in == 0u) ta_named_sync(1u + grp, 128u);   // the buffer's last readers are done
                if (valid)
#pragma unroll
                    for (uint32_t j = 0; j < 16u; j += 4u) *reinterpret_cast<float4*>(xs + (((in + j) / 4u ^ turn) << 2)) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                if (in + 16u < wide) continue;
                ta_named_sync(1u + grp, 128u);
                if (valid) {
                    const uint32_t cols = wide / p.split, next = (wide == 16u ? R : p.rows) * wide;
                    for (uint32_t j = share * cols; j < (share + 1u) * cols; j += 4u) {
                        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (uint32_t k = 0; k < 4u; ++k)
                            if (k < p.split) {
                                const float4 z = *reinterpret_cast<const float4*>(xr + k * next + ((j / 4u ^ turn) << 2));
                                y.x += z.x;
                                y.y += z.y;
                                y.z += z.z;
                                y.w += z.w;
                            }
                        if (whole) *reinterpret_cast<uint2*>(out + c0 - in + j) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
                        else *reinterpret_cast<float4*>(rec + c0 - in + j) = y;
                    }
                }
            }
            tm_fence_before();
            __syncwarp();
            if (lane == 0u) mbar_arrive(smem_u32(&s.o_empty));
            ++npiece;
        }
    }
    tm_fence_before();
    __syncthreads();
    if (warp == (uint32_t)Cfg::QK_WARP) tm_dealloc(tmem, 512);
}

// Joins the parts of the units that borders between blocks cut: block (b - 1, y) of the grid has border b, and does nothing unless it is the
// first border inside its unit.  A warp takes a row: weights 2^(m - largest m), sums in the order of the parts.  Bound by latency: prefix sums
// over the sequences, look-up of the unit, then a row's parts, four under way; its launch overlaps the main kernel's end.
constexpr int TA_MERGE_THREADS = 128;
template <int HD, int NK, int UR>
__global__ void __launch_bounds__(TA_MERGE_THREADS) kl_paged_tree_merge_kernel(const PagedView c, const TreeArgs a, const uint32_t blocks) {
    constexpr int NW = TA_MERGE_THREADS / 32, COLS = HD / 32;
    __shared__ uint64_t pre[NW * 32], wsum[NW];
    griddep_launch();
    griddep_wait();
    if (pg_stopped(c)) return;
    const uint64_t work = pg_prefix<NW>(c.n_seqs, pre, wsum, [&](uint32_t i) { return ta_work(c, ta_seq<NK, UR>(c, a, i)); });
    const uint32_t b = blockIdx.x + 1u, warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const TaShares shares(work, blocks);
    const uint64_t g = shares.border(b);
    if (g == 0u || g >= work) return;
    const uint32_t share = pg_find<NW>(pre, g), per = (c.n_seqs + NW * 32u - 1u) / (NW * 32u);
    uint32_t s = share * per;
    uint64_t off = g - pre[share];
    TaSeq q = ta_seq<NK, UR>(c, a, s);
    while (off >= ta_work(c, q)) {
        off -= ta_work(c, q);
        if (++s >= c.n_seqs) return;
        q = ta_seq<NK, UR>(c, a, s);
    }
    const TaUnit u = ta_unit<UR>(a, q, off);
    const uint64_t begin = g - (off - u.begin), end = begin + ((uint64_t)q.tiles << u.twice);
    const uint32_t first = b - 1u;
    if (g == begin || shares.border(first) > begin || u.tile_at(off) == q.tiles) return;   // (the last: the first block has the whole unit)
    const uint32_t first_slot = 2u * first + (shares.border(first) < begin ? 1u : 0u);
    uint32_t last = min(blocks - 1u, (uint32_t)pg_div(end * blocks - 1u, (uint32_t)min(work, (uint64_t)0xffffffffu)));   // nearly: the last block whose share begins before the unit's end
    last = max(last, b);
    while (last > b && shares.border(last) >= end) --last;
    while (last + 1u < blocks && shares.border(last + 1u) < end) ++last;
    auto slot_of = [&](uint32_t k) { return k == first ? first_slot : 2u * k; };
    auto tile_at = [&](uint64_t at) { return u.tile_at(min(max(at, begin), end) - begin + u.begin); };
    auto holds = [&](uint32_t k) { return tile_at(shares.border(k)) < tile_at(shares.border(k + 1u)); };   // blocks without a tile left nothing
    const bool mine = first + lane <= last && holds(first + lane);   // of the first 32
    for (uint32_t r = blockIdx.y * NW + warp; r < u.rows; r += gridDim.y * NW) {
        float m = -INFINITY, l = 0.f, sum[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) sum[j] = 0.f;
        for (uint32_t k0 = first; k0 <= last; k0 += 32u) {   // 32 parts at a time, each lane with the reference and sum of one
            float2 ml = make_float2(-INFINITY, 0.f);
            if (k0 == first ? mine : k0 + lane <= last && holds(k0 + lane)) ml = a.part_ml[(size_t)slot_of(k0 + lane) * TA_RECORD + r];
            float mx = fmaxf(m, ml.x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float old = m == -INFINITY ? 0.f : ta_exp2(m - mx), w = ml.x == -INFINITY ? 0.f : ta_exp2(ml.x - mx);
            m = mx;
            l *= old;
#pragma unroll
            for (int j = 0; j < COLS; ++j) sum[j] *= old;
            const float wl = w * ml.y;
            uint32_t todo = __ballot_sync(0xffffffffu, w > 0.f);
            while (todo) {   // four parts' loads under way
                float x[4][COLS], wk[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    wk[z] = 0.f;
                    const uint32_t k = todo ? __ffs(todo) - 1u : 0u;
                    const float wz = __shfl_sync(0xffffffffu, w, k), lz = __shfl_sync(0xffffffffu, wl, k);
                    if (!todo) {
#pragma unroll
                        for (int j = 0; j < COLS; ++j) x[z][j] = 0.f;
                        continue;
                    }
                    todo &= todo - 1u;
                    wk[z] = wz;
                    l += lz;
                    const float* src = a.part + ((size_t)slot_of(k0 + k) * TA_RECORD + r) * HD + lane * COLS;
                    if constexpr (COLS == 2) {
                        const float2 v = *reinterpret_cast<const float2*>(src);
                        x[z][0] = v.x; x[z][1] = v.y;
                    } else {
#pragma unroll
                        for (int j = 0; j < COLS / 4; ++j) {
                            const float4 v = reinterpret_cast<const float4*>(src)[j];
                            x[z][4 * j] = v.x; x[z][4 * j + 1] = v.y; x[z][4 * j + 2] = v.z; x[z][4 * j + 3] = v.w;
                        }
                    }
                }
#pragma unroll
                for (int z = 0; z < 4; ++z)
#pragma unroll
                    for (int j = 0; j < COLS; ++j) sum[j] += wk[z] * x[z][j];
            }
        }
        const uint32_t gr = u.row0 + r, tok = gr / a.G, head = u.h * a.G + gr - tok * a.G;
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
        if (a.lse && lane == 0u) a.lse[(size_t)(q.r0 + tok) * a.nq + head] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        uint32_t* out = reinterpret_cast<uint32_t*>(a.out + (int64_t)(q.r0 + tok) * a.out_stride + ((size_t)head * HD + lane * COLS) * 2u);
        uint32_t o[COLS / 2];
#pragma unroll
        for (int j = 0; j < COLS / 2; ++j) o[j] = pack_bf16(sum[2 * j] * inv, sum[2 * j + 1] * inv);
        if constexpr (COLS == 2) *out = o[0];
        else if constexpr (COLS == 4) *reinterpret_cast<uint2*>(out) = make_uint2(o[0], o[1]);
        else *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace kl
