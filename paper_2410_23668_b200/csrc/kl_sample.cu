// Sampling from given random numbers: temperature, top-k, top-p and min-p per row of logits (contract in include/kl.h).
//
// w_i = exp((x_i - max) / T).  Tokens in order of falling logit (the lower token first among equals): those of rank < k stay, of
// these those with less than p of their mass in front of them, of these those with w >= min_p; then the first token, in order of
// its number, at which the cumulative mass exceeds u times the mass of all that stayed.  Which token that is hangs on comparisons
// of sums of up to some 10^5 weights: weights and sums are held in 64 bits, so that it is the token of the definition (32 bits
// would err in one of ten draws from a flat row of 128256).
//
// One cluster of thread blocks = one row, whose logits are read once and stay in the blocks' shared memory.  A row is not sorted:
//   * a histogram over (max - x) / T, 64 bins to the unit, finds the bin that a cut falls into -- by counts for top-k, by mass for
//     top-p (a bin's members differ by 1.6 % at most, so their weights relative to the bin's largest fit whole numbers of 16 bits) --
//     and only that bin's members are put in order, by the first block;
//   * approximate masses only say which bin to look at: the mass in front of it and its own are then summed in 64 bits, and the
//     neighbouring bin is taken where they say so;
//   * a bin of too many members (equal logits) is cut again by their bits, until it is small or holds equal logits alone;
//   * for k up to SP_LIST all that can stay goes to the first block, which finishes alone.
//
// What bounds it: latency.  A row's way is load, largest logit, histogram, cut, sums, draw, with an exchange of the cluster between
// most of them, and two blocks to an SM are what its shared memory holds: one row of 128256 with k = 50 takes 12.4 us, 32 rows of mixed
// settings 41, 256 rows of 32000 with p = 0.9 79 (issue slots 46 % and 64-bit pipe 11 % busy), 160 rows of 128256 with min_p 69 (82 MB: 12.5 at the copy
// rate).  More blocks to a row while the GPU is not full, fewer where it is: see kl_sample.  A sort of the row, or several passes over memory,
// would cost more than the whole call (the same in library calls: 430 us for the one row).
#include "kl_device.cuh"

#include <atomic>

#include "../../include/kl.h"

using namespace kl;

namespace {

constexpr int SP_THREADS = 512, SP_WARPS = SP_THREADS / 32;
constexpr int SP_BINS = 2048;             // 64 to the unit of (max - x) / T; the last one holds all that lies further down
constexpr float SP_BINS_PER_UNIT = 64.f;
constexpr uint32_t SP_LIST = 2048;        // members of a bin that are put in order; also the largest k that one block finishes alone
constexpr uint32_t SP_SLICE = 40960;      // most logits of a block
constexpr int SP_POW = 64;                // entries of the table of powers of two
constexpr int SP_MAX_CLUSTER = 8;
constexpr uint32_t SP_SLICE_FEW = 16384;  // logits of a block beyond which a row is spread over more blocks

struct SampleArgs {
    const float* logits;
    int64_t stride;
    uint32_t n_rows, vocab, slice;
    const float *uniforms, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t *tokens, *positions;
    float* logprobs;
};

// Shared memory in front of the slice of logits.
struct alignas(16) SampleShared {
    uint64_t list[SP_LIST];               // members of a bin, (complement of the key, token): a block's own, in the first block all of them
    union {
        double listw[SP_LIST];
        uint64_t bins[SP_BINS];           // a histogram of the whole row
    };
    uint32_t hist[SP_BINS];               // a block's own
    double pow2[SP_POW];                  // 2^(j / SP_POW)
    // written by every block of the cluster; two of each in turn, so that a block may go on while another still reads
    double sums[2][SP_MAX_CLUSTER][3];
    uint64_t best[2][SP_MAX_CLUSTER];
    double warp_sum[SP_WARPS];
    uint64_t warp_u64[SP_WARPS];
    uint64_t cut;                         // first block: what the other blocks read
    uint64_t found64[2];
    uint32_t found, n_list, n_own;
};

__device__ __forceinline__ uint32_t cl_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cl_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cl_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of this block's shared variable in block `rank` of the cluster.
__device__ __forceinline__ uint32_t cl_map(const void* p, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void cl_st64(uint32_t a, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }
__device__ __forceinline__ void cl_st128(uint32_t a, uint64_t v, uint64_t w) {
    asm volatile("st.shared::cluster.v2.u64 [%0], {%1, %2};" ::"r"(a), "l"(v), "l"(w) : "memory");
}
__device__ __forceinline__ uint64_t cl_ld64(uint32_t a) { uint64_t v; asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory"); return v; }
__device__ __forceinline__ uint4 cl_ld128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
// Whole numbers in the order of the floats they stand for, and back.
__device__ __forceinline__ uint32_t sp_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float sp_unkey(uint32_t k) { return __uint_as_float(k ^ ((int32_t)k < 0 ? 0x80000000u : 0xffffffffu)); }
// Places in the order of falling logits: the lower the number, the earlier.
__device__ __forceinline__ uint64_t sp_place(float x, uint32_t token) { return (uint64_t)(~sp_key(x)) << 32 | token; }

struct Sampler {
    float* x;                 // this block's slice
    SampleShared& s;
    uint32_t base, n;         // first token of the slice, and how many
    uint32_t rank, C, tid, warp, lane;
    float m, scale;
    double c64;               // 64 log2(e) / T
    double md;                // m
    uint32_t turn;            // of the cluster's exchanges

    // exp((v - m) / T), by Tang's table method: t = 64 (v - m) log2(e) / T = n + r, 2^(n / 64) from a table of 64 powers and the exponent, 2^(r / 64)
    // from six terms of its series (|r| <= 1/2: the seventh is below 2^-54).  What is wrong with t counts most, 2^-46 at t = -80 * 92.
    __device__ __forceinline__ double weight(float v) const {
        const double t = ((double)v - md) * c64;
        if (!(t > -7400.0)) return 0.0;   // (an empty token's t is -infinity; the rest is less than 2^-115 of the largest)
        const double shifted = t + 6755399441055744.0;   // 1.5 * 2^52: the sum's last bit is 1
        const double r = t - (shifted - 6755399441055744.0);
        const int32_t n = __double2loint(shifted);
        constexpr double L = 0.010830424696249145;   // ln 2 / 64
        double q = L * L * L * L * L / 120;
        q = fma(q, r, L * L * L * L / 24);
        q = fma(q, r, L * L * L / 6);
        q = fma(q, r, L * L / 2);
        q = fma(q, r, L);
        q = fma(q, r, 1.0);
        q *= s.pow2[n & 63];
        return __hiloint2double(__double2hiint(q) + (n >> 6) * (1 << 20), __double2loint(q));
    }
    uint32_t i0, i1;          // this thread's run of the slice: of odd length, so that the runs of a warp lie in different banks
    __device__ __forceinline__ float at(float v) const { return (m - v) * scale; }   // in bins; infinite where there is no token
    __device__ __forceinline__ uint32_t bin(float v) const { return (uint32_t)fminf(at(v), (float)(SP_BINS - 1)); }

    // f(logit, place in the slice) for this thread's run
    template <class F>
    __device__ __forceinline__ void over_run(F&& f) const {
        uint32_t i = i0;
        for (; i + 8u <= i1; i += 8u) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = x[i + j];
#pragma unroll
            for (int j = 0; j < 8; ++j) f(v[j], i + j);
        }
        for (; i < i1; ++i) f(x[i], i);
    }
    // ... for those of it that `in` names: found first, so that a warp does f as often as its fullest run has some
    template <class In, class F>
    __device__ __forceinline__ void over_some(In&& in, F&& f) const {
        for (uint32_t i = i0; i < i1; i += 32u) {
            uint32_t todo = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < 32u; ++j)
                if (i + j < i1 && in(x[i + j])) todo |= 1u << j;
            for (; todo; todo &= todo - 1u) {
                const uint32_t a = i + __ffs(todo) - 1u;
                f(x[a], a);
            }
        }
    }
    __device__ __forceinline__ double block_sum(double v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0u) s.warp_sum[warp] = v;
        __syncthreads();
        double all = 0;
#pragma unroll
        for (int w = 0; w < SP_WARPS; ++w) all += s.warp_sum[w];
        return all;
    }
    // Inclusive sum over the threads of the block, what lies before this thread, and all of it.
    __device__ __forceinline__ double block_scan(double v, double& before, double& total) {
        double incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= (uint32_t)o) incl += y;
        }
        __syncthreads();
        if (lane == 31u) s.warp_sum[warp] = incl;
        __syncthreads();
        double b = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < SP_WARPS; ++w) {
            if (w < (int)warp) b += s.warp_sum[w];
            total += s.warp_sum[w];
        }
        before = b + (incl - v);
        return b + incl;
    }
    // Three sums over the cluster, the same in every block.
    __device__ __forceinline__ void cluster_sums(double& a, double& b, double& c) {
        a = block_sum(a);
        b = block_sum(b);
        c = block_sum(c);
        const uint32_t half = turn++ & 1u;
        if (tid < C) {
            const uint32_t to = cl_map(&s.sums[half][rank][0], tid);
            cl_st64(to, __double_as_longlong(a));
            cl_st64(to + 8u, __double_as_longlong(b));
            cl_st64(to + 16u, __double_as_longlong(c));
        }
        cl_sync();
        a = b = c = 0;
        for (uint32_t r = 0; r < C; ++r) {
            a += s.sums[half][r][0];
            b += s.sums[half][r][1];
            c += s.sums[half][r][2];
        }
    }
    __device__ __forceinline__ uint64_t block_min(uint64_t v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = min(v, (uint64_t)__shfl_xor_sync(0xffffffffu, (unsigned long long)v, o));
        __syncthreads();
        if (lane == 0u) s.warp_u64[warp] = v;
        __syncthreads();
        uint64_t all = s.warp_u64[0];
#pragma unroll
        for (int w = 1; w < SP_WARPS; ++w) all = min(all, s.warp_u64[w]);
        return all;
    }
    __device__ __forceinline__ uint64_t cluster_min(uint64_t v) {
        v = block_min(v);
        const uint32_t half = turn++ & 1u;
        if (tid < C) cl_st64(cl_map(&s.best[half][rank], tid), v);
        cl_sync();
        for (uint32_t r = 0; r < C; ++r) v = min(v, s.best[half][r]);
        return v;
    }

    // Histogram over the whole row, in every thread's hands: thread t gets bins 4 t .. 4 t + 3.
    // each(add) calls add(bin, amount) for what this thread contributes.
    template <class Each>
    __device__ __forceinline__ void histogram(Each&& each, uint64_t (&mine)[4]) {
        static_assert(SP_BINS == 4 * SP_THREADS, "four bins to a thread");
        __syncthreads();
        reinterpret_cast<uint4*>(s.hist)[tid] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        each([&](uint32_t b, uint32_t v) { atomicAdd(&s.hist[b], v); });
        if (C > 1u) {
            cl_sync();
            // every block adds up its share of the bins and hands the sums to all
            const uint32_t per = SP_BINS / C, b4 = rank * per + 4u * tid;
            if (4u * tid < per) {
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[i] = 0;
                for (uint32_t r = 0; r < C; ++r) {
                    const uint4 h = cl_ld128(cl_map(&s.hist[b4], r));
                    mine[0] += h.x; mine[1] += h.y; mine[2] += h.z; mine[3] += h.w;
                }
                for (uint32_t r = 0; r < C; ++r) {
                    const uint32_t to = cl_map(&s.bins[b4], r);
                    cl_st128(to, mine[0], mine[1]);
                    cl_st128(to + 16u, mine[2], mine[3]);
                }
            }
            cl_sync();
            const ulonglong2 a = reinterpret_cast<const ulonglong2*>(s.bins)[2 * tid], b = reinterpret_cast<const ulonglong2*>(s.bins)[2 * tid + 1];
            mine[0] = a.x; mine[1] = a.y; mine[2] = b.x; mine[3] = b.y;
        } else {
            __syncthreads();
            const uint4 h = reinterpret_cast<const uint4*>(s.hist)[tid];
            mine[0] = h.x; mine[1] = h.y; mine[2] = h.z; mine[3] = h.w;
        }
    }

    // A list of tokens, in any order: every block's own (list_begin, then list_add), joined in the first block's by list_end, which returns
    // how many there are in all (more than SP_LIST: some are missing).  Between two lists lies another exchange of the cluster.
    __device__ __forceinline__ void list_begin() {
        if (tid == 0u) s.n_own = 0u;
        __syncthreads();
    }
    __device__ __forceinline__ void list_add(float v, uint32_t token) {
        const uint32_t at = atomicAdd(&s.n_own, 1u);
        if (at < SP_LIST) s.list[at] = sp_place(v, token);
    }
    template <class In>
    __device__ __forceinline__ uint32_t gather(In&& in) {   // those that `in` names
        list_begin();
        over_run([&](float v, uint32_t i) {
            if (in(v, base + i)) list_add(v, base + i);
        });
        return list_end();
    }
    __device__ __forceinline__ uint32_t list_end() {
        if (C == 1u) {
            __syncthreads();
            return s.n_own;
        }
        __syncthreads();
        const uint32_t own = s.n_own, half = turn++ & 1u;
        if (tid < C) cl_st64(cl_map(&s.best[half][rank], tid), own);
        cl_sync();
        uint32_t before = 0, all = 0;
        for (uint32_t r = 0; r < C; ++r) {
            const uint32_t c = (uint32_t)s.best[half][r];
            if (r < rank) before += c;
            all += c;
        }
        if (rank > 0u && all <= SP_LIST) {
            const uint32_t to = cl_map(&s.list[before], 0);
            for (uint32_t i = tid; i < own; i += SP_THREADS) cl_st64(to + i * 8u, s.list[i]);
        }
        cl_sync();
        return all;
    }
    // The first cnt entries of the list in ascending order (first block; cnt <= SP_LIST, all different).
    __device__ __forceinline__ void sort_list(uint32_t cnt) {
        if (cnt <= 2 * SP_THREADS) {   // every thread counts what comes before its own entries
            const uint64_t own = tid < cnt ? s.list[tid] : ~0ull, second = tid + SP_THREADS < cnt ? s.list[tid + SP_THREADS] : ~0ull;
            const uint32_t at = count_before(own, cnt), at2 = cnt > SP_THREADS ? count_before(second, cnt) : 0u;
            __syncthreads();
            if (tid < cnt) s.list[at] = own;
            if (tid + SP_THREADS < cnt) s.list[at2] = second;
            __syncthreads();
            return;
        }
        uint32_t len = 2;   // bitonic
        while (len < cnt) len <<= 1;
        for (uint32_t i = cnt + tid; i < len; i += SP_THREADS) s.list[i] = ~0ull;
        __syncthreads();
        for (uint32_t k = 2; k <= len; k <<= 1)
            for (uint32_t j = k >> 1; j > 0; j >>= 1) {
                for (uint32_t t = tid; t < len / 2; t += SP_THREADS) {
                    const uint32_t i = 2 * t - (t & (j - 1)), l = i + j;
                    const uint64_t a = s.list[i], b = s.list[l];
                    if ((a > b) == ((i & k) == 0u)) {
                        s.list[i] = b;
                        s.list[l] = a;
                    }
                }
                __syncthreads();
            }
    }
    __device__ __forceinline__ uint32_t count_before(uint64_t own, uint32_t cnt) const {
        uint32_t at = 0;
        if (__any_sync(0xffffffffu, own != ~0ull)) {
#pragma unroll 4
            for (uint32_t j = 0; j + 1u < cnt; j += 2u) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&s.list[j]);
                at += (v.x < own) + (v.y < own);
            }
            if (cnt & 1u) at += s.list[cnt - 1u] < own;
        }
        return at;
    }
    __device__ __forceinline__ uint64_t broadcast(uint64_t v) {   // of the first block's thread 0
        if (rank == 0u && tid == 0u) s.cut = v;
        cl_sync();
        v = cl_ld64(cl_map(&s.cut, 0));
        cl_sync();
        return v;
    }
};

// The bin whose running sum first reaches `want` (> 0), the sum in front of it and its own; bins are four to a thread.  Whole block.
__device__ __forceinline__ bool sp_find(Sampler& q, const uint64_t (&mine)[4], uint64_t want, uint32_t& bin, uint64_t& before, uint64_t& own) {
    SampleShared& s = q.s;
    const uint64_t sum = mine[0] + mine[1] + mine[2] + mine[3];
    uint64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, (unsigned long long)incl, o);
        if (q.lane >= (uint32_t)o) incl += y;
    }
    __syncthreads();
    if (q.lane == 31u) s.warp_u64[q.warp] = incl;
    if (q.tid == 0u) s.found = SP_BINS;
    __syncthreads();
    uint64_t b = 0;
    for (uint32_t w = 0; w < q.warp; ++w) b += s.warp_u64[w];
    uint64_t at = b + incl - sum;
    if (at < want && want <= at + sum) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at < want && want <= at + mine[i]) {
                s.found = 4 * q.tid + i;
                s.found64[0] = at;
                s.found64[1] = mine[i];
            }
            at += mine[i];
        }
    }
    __syncthreads();
    bin = s.found;
    before = s.found64[0];
    own = s.found64[1];
    __syncthreads();
    return bin < SP_BINS;
}

// The tokens that stay: those before the place (x, token) and it.
struct SampleCut {
    float x;              // -infinity: all that are tokens
    uint32_t end;         // of the tokens with this logit, those below
    __device__ __forceinline__ bool stays(float v, uint32_t token) const { return v > x || (v == x && token < end); }
    __device__ __forceinline__ uint64_t place() const { return end ? sp_place(x, end - 1u) : ~0ull - 1ull; }
};
__device__ __forceinline__ SampleCut sp_cut_at(uint64_t place) { return {sp_unkey(~(uint32_t)(place >> 32)), (uint32_t)place + 1u}; }

// A run of places that a cut falls into: a bin of the row's first histogram, or the places lo .. hi.
struct SampleRegion {
    float from, to;       // the bin, as the least and the largest number of bins; from < 0: lo and hi say it
    uint64_t lo, hi;
    // -1: the token comes before the region, 0: it belongs to it, 1: behind it
    __device__ __forceinline__ int side(const Sampler& q, float x, uint32_t token) const {
        if (from >= 0.f) {
            const float t = q.at(x);
            return t < from ? -1 : t > to;
        }
        const uint64_t place = sp_place(x, token);
        return place < lo ? -1 : place > hi;
    }
};
__device__ __forceinline__ SampleRegion sp_bin(uint32_t b) {   // (the number below b + 1, as a float; the last bin has no end)
    return {(float)b, b + 1u < (uint32_t)SP_BINS ? __uint_as_float(__float_as_uint((float)(b + 1u)) - 1u) : INFINITY, 0, 0};
}

// A region of too many tokens is cut into SP_BINS runs of places, 2^shift each from the first place that it holds.
__device__ __forceinline__ void sp_split(Sampler& q, const SampleRegion& g, uint64_t& lo, uint64_t& hi, uint32_t& shift) {
    uint64_t first = ~0ull, last = ~0ull;   // last: its complement
    for (uint32_t i = q.tid; i < q.n; i += SP_THREADS) {
        if (!(q.x[i] > -INFINITY)) continue;
        const uint64_t p = sp_place(q.x[i], q.base + i);
        if (g.side(q, q.x[i], q.base + i) == 0) {
            first = min(first, p);
            last = min(last, ~p);
        }
    }
    lo = q.cluster_min(first);
    hi = ~q.cluster_min(last);
    shift = 0;
    while (((hi - lo) >> shift) >= SP_BINS) ++shift;
}

// The place of rank k - 1 (ranks from zero): the last one that stays.
__device__ __forceinline__ SampleCut sp_cut_by_rank(Sampler& q, SampleRegion g, uint64_t before, uint64_t own, uint64_t k) {
    while (own > SP_LIST) {
        uint64_t lo, hi, mine[4], b4;
        uint32_t shift, bin;
        sp_split(q, g, lo, hi, shift);
        q.histogram([&](auto&& add) {
            for (uint32_t i = q.tid; i < q.n; i += SP_THREADS) {
                const uint64_t p = sp_place(q.x[i], q.base + i);
                if (q.x[i] > -INFINITY && p >= lo && p <= hi) add((uint32_t)((p - lo) >> shift), 1u);
            }
        }, mine);
        if (!sp_find(q, mine, k - before, bin, b4, own)) return sp_cut_at(hi);
        before += b4;
        g.from = -1.f;
        g.lo = lo + ((uint64_t)bin << shift);
        g.hi = min(hi, g.lo + (((uint64_t)1 << shift) - 1u));
    }
    const uint32_t cnt = q.gather([&](float x, uint32_t token) { return x > -INFINITY && g.side(q, x, token) == 0; });
    uint64_t cut = 0;
    if (q.rank == 0u) {   // own >= k - before >= 1
        q.sort_list(cnt);
        cut = q.s.list[min((uint32_t)(k - before), cnt) - 1u];
    }
    return sp_cut_at(q.broadcast(cut));
}

// What stays of `cut` when those stay with less than p of its mass in front of them.  g: the region that the new cut falls into, run_front:
// the mass of this thread's run that lies in front of it; hits: how many of the run belong to it, hit: the first of them.
__device__ __forceinline__ SampleCut sp_cut_by_mass(Sampler& q, const SampleCut cut, double p, SampleRegion& g, double& run_front, uint32_t& hits, uint32_t& hit) {
    SampleShared& s = q.s;
    uint64_t mine[4], before, own;
    uint32_t bin;
    // approximate masses, in units of 2^-43 of the largest weight: sums of at most 2^19 tokens stay below 2^62
    q.histogram([&](auto&& add) {
#pragma unroll 4
        for (uint32_t i = q.tid; i < q.n; i += SP_THREADS) {
            const float x = q.x[i];
            if (!cut.stays(x, q.base + i)) continue;
            // bins and their fraction f; the weight relative to the bin's largest is exp(-f / 64), to third order
            const uint32_t u = (uint32_t)(fminf(q.at(x), (float)SP_BINS - 0.01f) * 65536.f), f = u & 0xffffu;
            add(u >> 16, 65536u - (f >> 6) + (f * f >> 29));
        }
    }, mine);
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[i] = (uint64_t)((float)mine[i] * exp2f((4 * q.tid + i) * (-1.4426950408889634f / SP_BINS_PER_UNIT) + 27.f));
    {
        const double part = (double)(mine[0] + mine[1] + mine[2] + mine[3]);   // (rounded: approximate anyway)
        all = (uint64_t)q.block_sum(part);
    }
    uint64_t want = (uint64_t)(p * (double)all);
    if (want < 1ull) want = 1ull;
    if (!sp_find(q, mine, want, bin, before, own)) bin = 0u;
    double total = 0, goal = 0, front, inside;
    g = sp_bin(bin);
    uint64_t lo = 0, hi = 0;   // of the runs of places that a region has been cut into, if it has
    uint32_t shift = 0, last = SP_BINS - 1;
    int went = 0;
    bool settled = false;
    for (;;) {
        // the masses in front of the region, in it and behind it, and a list of its members
        double behind = 0;
        front = inside = 0;
        hits = 0;
        q.list_begin();
        q.over_run([&](float x, uint32_t i) {
            if (!cut.stays(x, q.base + i)) return;
            const int side = g.side(q, x, q.base + i);
            if (side > 0 && goal > 0) return;
            const double w = q.weight(x);
            if (side < 0) {
                front += w;
            } else if (side == 0) {
                inside += w;
                if (hits++ == 0u) hit = i;
                q.list_add(x, q.base + i);
            } else {
                behind += w;
            }
        });
        run_front = front;
        double sum = front + inside + behind;
        q.cluster_sums(sum, front, inside);
        if (goal == 0) {
            total = sum;
            goal = p * total;
        }
        // towards the region where the mass in front first reaches the goal; where two neighbours point at each other (their sums
        // round apart) the one that was left again is taken
        const int go = front >= goal ? -1 : front + inside < goal ? 1 : 0;
        if (!settled && go != 0 && (go < 0 ? bin > 0u : bin < last)) {
            settled = go == -went;
            went = go;
            bin += go;
        } else {
            const uint32_t cnt = q.list_end();
            if (cnt <= SP_LIST) {
                uint64_t end = 0;
                if (q.rank == 0u) {
                    q.sort_list(cnt);
                    double w[SP_LIST / SP_THREADS], sum4 = 0, ahead, all4;
#pragma unroll
                    for (uint32_t i = 0; i < SP_LIST / SP_THREADS; ++i) {
                        const uint32_t at = q.tid * (SP_LIST / SP_THREADS) + i;
                        w[i] = at < cnt ? q.weight(sp_unkey(~(uint32_t)(s.list[at] >> 32))) : 0.0;
                        sum4 += w[i];
                    }
                    q.block_scan(sum4, ahead, all4);
                    uint32_t stay = 0;
#pragma unroll
                    for (uint32_t i = 0; i < SP_LIST / SP_THREADS; ++i) {
                        const uint32_t at = q.tid * (SP_LIST / SP_THREADS) + i;
                        if (at < cnt && front + ahead < goal) stay = at + 1u;
                        ahead += w[i];
                    }
                    const uint32_t most = (uint32_t)~q.block_min(~(uint64_t)stay);
                    end = cnt ? s.list[most ? most - 1u : 0u] : cut.place();
                }
                return sp_cut_at(q.broadcast(end));
            }
            sp_split(q, g, lo, hi, shift);
            hi = min(hi, cut.place());
            went = 0;
            settled = false;
            const float first = sp_unkey(~(uint32_t)(lo >> 32));
            q.histogram([&](auto&& add) {
                for (uint32_t i = q.tid; i < q.n; i += SP_THREADS) {
                const float x = q.x[i];
                const uint64_t place = sp_place(x, q.base + i);
                if (!(x > -INFINITY) || place < lo || place > hi) continue;
                add((uint32_t)((place - lo) >> shift), (uint32_t)(65536.f * exp2f((float)(((double)x - (double)first) * q.c64) * (1.f / 64.f))));
                }
            }, mine);
            last = (uint32_t)((hi - lo) >> shift);
            const double unit = q.weight(first) / 65536.0;
            want = unit > 0 ? (uint64_t)fmax(fmin((goal - front) / unit, 9e18), 1.0) : 1ull;
            if (!sp_find(q, mine, want, bin, before, own)) bin = last;
        }
        if (hi) {
            g.from = -1.f;
            g.lo = lo + ((uint64_t)bin << shift);
            g.hi = min(hi, g.lo + (((uint64_t)1 << shift) - 1u));
        } else {
            g = sp_bin(bin);
        }
    }
}

__device__ __forceinline__ void sp_write(const SampleArgs& a, uint32_t row, int32_t token, double w, double total) {
    a.tokens[row] = token;
    if (a.logprobs) a.logprobs[row] = token < 0 ? -INFINITY : (float)log(w / total);
    if (a.positions && token >= 0) ++a.positions[row];
}

// The first block alone: `cnt` tokens in its list, of which the first k by rank stay.
__device__ __forceinline__ void sp_finish_list(Sampler& q, const SampleArgs& a, uint32_t row, uint32_t cnt, uint32_t k, double p, double min_p, double u) {
    SampleShared& s = q.s;
    if (cnt <= SP_THREADS) {   // a token to a thread; orders by counting
        const uint64_t own = q.tid < cnt ? s.list[q.tid] : ~0ull;
        const double w = q.tid < cnt ? q.weight(sp_unkey(~(uint32_t)(own >> 32))) : 0.0;
        const uint32_t rank = q.count_before(own, cnt), most = min(cnt, k);
        if (q.tid < cnt) s.listw[rank] = w;
        __syncthreads();
        const double in_order = q.tid < most ? s.listw[q.tid] : 0.0;
        double ahead, mass, total;
        q.block_scan(in_order, ahead, mass);
        // (what stays is the beginning of the order)
        const uint32_t stay = (uint32_t)__syncthreads_count(q.tid < most && (q.tid == 0u || ((p >= 1.0 || ahead < p * mass) && in_order >= min_p)));
        const uint32_t token = q.tid < cnt && rank < stay ? (uint32_t)own : ~0u;
        uint32_t* tokens = s.hist;
        if (q.tid < (cnt + 3u) / 4u * 4u) tokens[q.tid] = token;
        __syncthreads();
        uint32_t at = 0;
        if (q.warp * 32u < cnt)
#pragma unroll 4
            for (uint32_t j = 0; j < cnt; j += 4u) {
                const uint4 v = *reinterpret_cast<const uint4*>(&tokens[j]);
                at += (v.x < token) + (v.y < token) + (v.z < token) + (v.w < token);
            }
        if (token != ~0u) {
            s.listw[SP_THREADS + at] = w;
            s.hist[SP_THREADS + at] = token;
        }
        __syncthreads();
        const double mine = q.tid < stay ? s.listw[SP_THREADS + q.tid] : 0.0;
        const double up_to = q.block_scan(mine, ahead, total), goal = u * total;
        // the first token at which the running mass exceeds the goal; the last one of any mass where rounding lets none
        const uint64_t first = q.block_min(mine > 0 && up_to > goal ? q.tid : ~0ull), last = ~q.block_min(mine > 0 ? ~(uint64_t)q.tid : ~0ull);
        if (q.tid == (uint32_t)(first != ~0ull ? first : last)) sp_write(a, row, (int32_t)s.hist[SP_THREADS + q.tid], mine, total);
        return;
    }
    constexpr uint32_t PER = SP_LIST / SP_THREADS;
    q.sort_list(cnt);
    cnt = min(cnt, k);
    double w[PER], sum = 0, ahead;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t at = q.tid * PER + i;
        w[i] = at < cnt ? q.weight(sp_unkey(~(uint32_t)(s.list[at] >> 32))) : 0.0;
        sum += w[i];
    }
    double mass, total;
    q.block_scan(sum, ahead, mass);
    uint64_t item[PER];
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t at = q.tid * PER + i;
        const bool stays = at < cnt && (at == 0u || ((p >= 1.0 || ahead < p * mass) && w[i] >= min_p));
        item[i] = (uint64_t)(stays ? (uint32_t)s.list[at] : ~0u) << 32 | at;   // (what does not stay: behind all tokens)
        ahead += w[i];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t at = q.tid * PER + i;
        if (at < cnt) {
            s.list[at] = item[i];
            s.listw[at] = w[i];
        }
    }
    __syncthreads();
    q.sort_list(cnt);   // by token
    sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t at = q.tid * PER + i;
        item[i] = at < cnt ? s.list[at] : ~0ull;
        w[i] = item[i] >> 32 != 0xffffffffull ? s.listw[(uint32_t)item[i]] : 0.0;
        sum += w[i];
    }
    q.block_scan(sum, ahead, total);
    const double goal = u * total;
    // the first token at which the running mass exceeds the goal; the last one of any mass where rounding lets none
    uint64_t first = ~0ull, last = ~0ull;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        ahead += w[i];
        if (w[i] > 0) {
            if (ahead > goal) first = min(first, item[i]);
            last = min(last, ~item[i]);
        }
    }
    first = q.block_min(first);
    last = ~q.block_min(last);
    if (q.tid == 0u) {
        const uint64_t it = first != ~0ull ? first : last;
        sp_write(a, row, (int32_t)(it >> 32), s.listw[(uint32_t)it], total);
    }
}

__global__ void __launch_bounds__(SP_THREADS, 2) kl_sample_kernel(const SampleArgs a) {
    extern __shared__ __align__(16) uint8_t sp_smem[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(sp_smem);
    const uint32_t C = cl_size(), row = blockIdx.x / C;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // every block of the cluster has begun: see the wait
    griddep_launch();
    griddep_wait();
    Sampler q = {reinterpret_cast<float*>(sp_smem + sizeof(SampleShared)), s};
    q.rank = cl_rank();
    q.C = C;
    q.tid = threadIdx.x;
    q.warp = threadIdx.x >> 5;
    q.lane = threadIdx.x & 31u;
    q.base = q.rank * a.slice;
    q.n = q.base < a.vocab ? min(a.slice, a.vocab - q.base) : 0u;
    q.turn = 0;
    const uint32_t run = (q.n + SP_THREADS - 1u) / SP_THREADS | 1u;
    q.i0 = min(q.n, q.tid * run);
    q.i1 = min(q.n, q.i0 + run);
    const bool idle = a.positions && a.positions[row] < 0;   // an empty slot of the batch: the same for the whole cluster
    const float T = a.temperature ? a.temperature[row] : 1.f;
    const float top_p = a.top_p ? a.top_p[row] : 1.f, min_pf = a.min_p ? a.min_p[row] : 0.f;
    int32_t top_k = a.top_k ? a.top_k[row] : 0;
    const double p = top_p < 1.f ? (double)top_p : 1.0, min_p = min_pf > 0.f ? (double)min_pf : 0.0;
    if (!(T > 0.f) || p <= 0.0 || min_p > 1.0) top_k = 1;
    const double u = a.uniforms[row] > 0.f ? (double)fminf(a.uniforms[row], 1.f) : 0.0;

    if (q.tid < SP_POW) s.pow2[q.tid] = exp2((double)q.tid / SP_POW);
    // NaN is no token; -0 counts as 0.  This thread's largest logit, the lowest token among equals.
    float most = -INFINITY;
    uint32_t most_at = 0;
    auto keep = [&](float v, uint32_t i) {
        const float y = v == v ? v + 0.f : -INFINITY;
        if (y > most) {
            most = y;
            most_at = i;
        }
        return y;
    };
    if (!idle) {
        const float* src = a.logits + (int64_t)row * a.stride + q.base;
        const uint32_t n4 = ((uintptr_t)src & 15u) == 0 ? q.n / 4u : 0u;   // pieces of 16 bytes
        constexpr int U = 8;
        for (uint32_t i0 = q.tid; i0 < n4; i0 += SP_THREADS * U) {
            float4 v[U];
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (i0 + j * SP_THREADS < n4) v[j] = reinterpret_cast<const float4*>(src)[i0 + j * SP_THREADS];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const uint32_t i = i0 + j * SP_THREADS;
                if (i < n4) {
                    const float4 y = make_float4(keep(v[j].x, 4 * i), keep(v[j].y, 4 * i + 1), keep(v[j].z, 4 * i + 2), keep(v[j].w, 4 * i + 3));
                    reinterpret_cast<float4*>(q.x)[i] = y;
                }
            }
        }
        for (uint32_t i0 = 4 * n4 + q.tid; i0 < q.n; i0 += SP_THREADS * 2 * U) {
            float v[2 * U];
#pragma unroll
            for (int j = 0; j < 2 * U; ++j)
                if (i0 + j * SP_THREADS < q.n) v[j] = src[i0 + j * SP_THREADS];
#pragma unroll
            for (int j = 0; j < 2 * U; ++j) {
                const uint32_t i = i0 + j * SP_THREADS;
                if (i < q.n) q.x[i] = keep(v[j], i);
            }
        }
    }
    uint64_t best = most > -INFINITY ? sp_place(most, q.base + most_at) : ~0ull;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (idle) return;
    best = q.cluster_min(best);
    if (best == ~0ull || top_k == 1) {   // nothing to choose from, or nothing to choose
        if (q.rank == 0u && q.tid == 0u) sp_write(a, row, best == ~0ull ? -1 : (int32_t)(uint32_t)best, 1.0, 1.0);
        return;
    }
    q.m = sp_unkey(~(uint32_t)(best >> 32));
    if (q.m == INFINITY) {   // equal chances for the infinite ones, none for the rest
        for (uint32_t i = q.tid; i < q.n; i += SP_THREADS) q.x[i] = q.x[i] == INFINITY ? 0.f : -INFINITY;
        most = most == INFINITY ? 0.f : -INFINITY;
        q.m = 0.f;
        __syncthreads();
    }
    q.scale = fminf(SP_BINS_PER_UNIT / T, 3e38f);
    q.md = (double)q.m;
    q.c64 = 92.33248261893449 / (double)T;   // 64 log2(e)

    SampleCut cut = {-INFINITY, 0u};
    if (top_k > 0 && (uint32_t)top_k < a.vocab) {
        uint64_t mine[4], before, own;
        uint32_t bin;
        // The k-th largest of the threads' largest logits is a lower bound of the k-th largest of all, and few others lie above it.
        if ((uint32_t)top_k <= C * (SP_THREADS / 4)) {
            q.histogram([&](auto&& add) {
                if (most > -INFINITY) add(q.bin(most), 1u);
            }, mine);
            if (sp_find(q, mine, (uint64_t)top_k, bin, before, own)) {
                const float to = sp_bin(bin).to;
                const uint32_t cnt = q.gather([&](float x, uint32_t) { return x > -INFINITY && q.at(x) <= to; });
                if (cnt <= SP_LIST) {
                    if (q.rank == 0u) sp_finish_list(q, a, row, cnt, (uint32_t)top_k, p, min_p, u);
                    return;
                }
            }
        }
        q.histogram([&](auto&& add) {
            for (uint32_t i = q.tid; i < q.n; i += SP_THREADS)
                if (q.x[i] > -INFINITY) add(q.bin(q.x[i]), 1u);
        }, mine);
        const bool enough = sp_find(q, mine, (uint64_t)top_k, bin, before, own);
        if (enough && before + own <= SP_LIST) {
            const float to = sp_bin(bin).to;
            const uint32_t cnt = q.gather([&](float x, uint32_t) { return x > -INFINITY && q.at(x) <= to; });
            if (q.rank == 0u) sp_finish_list(q, a, row, cnt, (uint32_t)top_k, p, min_p, u);
            return;
        }
        if (enough) cut = sp_cut_by_rank(q, sp_bin(bin), before, own, (uint64_t)top_k);
    }
    SampleRegion g;
    double run_front = 0;
    uint32_t hits = 0, hit = 0;
    if (p < 1.0) cut = sp_cut_by_mass(q, cut, p, g, run_front, hits, hit);

    // The draw: every thread sums up its run, then the run that the goal falls into is looked at once more.
    // What is certainly below min_p need not be weighed: 32 bits with room to spare.
    const float sure = min_p > 0 ? q.m + 1.0001f * T * logf(min_pf) - 1e-5f * fabsf(q.m) : -INFINITY, least = fmaxf(cut.x, sure);
    auto weight = [&](float x, uint32_t i) {
        if (!cut.stays(x, q.base + i)) return 0.0;
        const double w = q.weight(x);
        return w >= min_p ? w : 0.0;
    };
    double mine = 0, before, own;
    if (p < 1.0 && !(min_p > 0)) {   // the mass in front of the cut's region is known
        mine = run_front;
        if (hits == 1u) {
            if (cut.stays(q.x[hit], q.base + hit)) mine += q.weight(q.x[hit]);
        } else if (hits) {
            q.over_run([&](float x, uint32_t i) {
                if (x >= cut.x && cut.stays(x, q.base + i) && g.side(q, x, q.base + i) == 0) mine += q.weight(x);
            });
        }
    } else {
        auto add = [&](float x, uint32_t i) { mine += weight(x, i); };
        if (least > -INFINITY) q.over_some([&](float x) { return x >= least; }, add);
        else q.over_run(add);
    }
    q.block_scan(mine, before, own);
    const uint32_t half = q.turn++ & 1u;
    if (C > 1u) {
        if (q.tid < C) cl_st64(cl_map(&s.sums[half][q.rank][0], q.tid), __double_as_longlong(own));
        cl_sync();
    } else {
        if (q.tid == 0u) s.sums[half][0][0] = own;
        __syncthreads();
    }
    double total = 0;
    for (uint32_t r = 0; r < C; ++r) total += s.sums[half][r][0];
    const double goal = u * total;
    // the first block whose end lies beyond the goal, else the last one that has any mass
    double at = 0, front = 0;
    uint32_t who = C;
    bool beyond = false;
    for (uint32_t r = 0; r < C; ++r) {
        const double x = s.sums[half][r][0];
        if (x > 0 && !beyond) {
            who = r;
            front = at;
            beyond = at + x > goal;
        }
        at += x;
    }
    if (who != q.rank) return;
    // the same among the threads' runs
    const uint64_t first = q.block_min(mine > 0 && front + before + mine > goal ? q.tid : ~0ull), last = ~q.block_min(mine > 0 ? ~(uint64_t)q.tid : ~0ull);
    const uint32_t t = (uint32_t)(first != ~0ull ? first : last);
    if (q.tid == t) s.found64[0] = __double_as_longlong(front + before);
    __syncthreads();
    if (q.warp != 0u) return;
    // and among the tokens of that run, 32 at a time
    double start = __longlong_as_double(s.found64[0]);
    const uint32_t k0 = min(q.n, t * run), k1 = min(q.n, k0 + run);
    uint32_t token = 0;
    double w_token = 1;
    for (uint32_t k = k0; k < k1; k += 32u) {
        const double w = k + q.lane < k1 ? weight(q.x[k + q.lane], k + q.lane) : 0.0;
        double incl = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, incl, o);
            if (q.lane >= (uint32_t)o) incl += y;
        }
        const uint32_t any = __ballot_sync(0xffffffffu, w > 0), over = __ballot_sync(0xffffffffu, w > 0 && start + incl > goal);
        if (any) {
            const uint32_t l = over ? __ffs(over) - 1 : 31 - __clz(any);
            token = q.base + k + l;
            w_token = __shfl_sync(0xffffffffu, w, l);
        }
        if (over) break;
        start += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (q.lane == 0u) sp_write(a, row, (int32_t)token, w_token, total);
}

}  // namespace

extern "C" kl_status kl_sample(const float* logits_d, int64_t row_stride, uint32_t n_rows, uint32_t vocab, const float* uniforms_d,
                               const float* temperature_d, const int32_t* top_k_d, const float* top_p_d, const float* min_p_d, int32_t* tokens_d,
                               float* logprobs_d, int32_t* positions_d, void* stream) {
    if (n_rows == 0) return KL_OK;
    if (!logits_d || !uniforms_d || !tokens_d || vocab == 0) return KL_ERR_INVALID_ARG;
    for (const void* x : {(const void*)logits_d, (const void*)uniforms_d, (const void*)temperature_d, (const void*)top_k_d, (const void*)top_p_d, (const void*)min_p_d,
                          (const void*)tokens_d, (const void*)logprobs_d, (const void*)positions_d})
        if ((uintptr_t)x & 3u) return KL_ERR_INVALID_ARG;
    if (n_rows > 1 && (row_stride < (int64_t)vocab || row_stride > (INT64_MAX >> 27))) return KL_ERR_INVALID_ARG;   // 2^24 rows of it are counted in 64 bits of bytes
    if (vocab > SP_SLICE * SP_MAX_CLUSTER || n_rows > (1u << 24)) return KL_ERR_UNSUPPORTED_SHAPE;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return KL_ERR_CUDA;
    // blocks of a row: as many as hold it, and while the GPU is not full, twice as many as long as each has SP_SLICE_FEW / 8 logits to do
    uint32_t C = 1;
    while (C < SP_MAX_CLUSTER && vocab > (uint64_t)C * SP_SLICE_FEW) C *= 2;
    while (C < SP_MAX_CLUSTER && (uint64_t)n_rows * C * 2 <= (uint64_t)sms && vocab >= C * 2 * (SP_SLICE_FEW / 8)) C *= 2;
    SampleArgs a;
    a.logits = logits_d;
    a.stride = row_stride;
    a.n_rows = n_rows;
    a.vocab = vocab;
    a.slice = (vocab + 4 * C - 1) / (4 * C) * 4;   // pieces of 16 bytes
    a.uniforms = uniforms_d;
    a.temperature = temperature_d;
    a.top_p = top_p_d;
    a.min_p = min_p_d;
    a.top_k = top_k_d;
    a.tokens = tokens_d;
    a.positions = positions_d;
    a.logprobs = logprobs_d;
    static std::atomic<uint64_t> done{0};   // one bit per device whose kernel attribute is set
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (!bit || !(done.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(kl_sample_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(SampleShared) + SP_SLICE * 4)) != cudaSuccess)
            return KL_ERR_CUDA;
        done.fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_rows * C);
    cfg.blockDim = dim3(SP_THREADS);
    cfg.dynamicSmemBytes = sizeof(SampleShared) + (size_t)a.slice * 4;
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kl_sample_kernel, a) == cudaSuccess ? KL_OK : KL_ERR_CUDA;
}
