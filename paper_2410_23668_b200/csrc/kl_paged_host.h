// What the host sides of the paged operators share: launches, checks of descriptors, their form for the kernels.
#pragma once

#include <atomic>
#include <utility>

#include "kl_paged_common.cuh"
#include "kl_paged_internal.h"

namespace kl {

// With `early` a kernel is launched with programmatic stream serialisation (see griddep_wait): its set-up overlaps the end of the
// stream's previous kernel.
template <typename... KArgs, typename... Args>
kl_status launch(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, PagedOrder order, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = reinterpret_cast<cudaStream_t>(order.stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = order.early ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...) == cudaSuccess ? KL_OK : KL_ERR_CUDA;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline uint32_t elem(int type) { return type == KL_F32 ? 4u : 2u; }

// The descriptor's own consistency (rows: whether the call touches k_d, v_d and the scales).
inline kl_status check_cache(const kl_paged_cache* c, bool rows) {
    if (!c) return KL_ERR_INVALID_ARG;
    if (!c->n_kv_heads || (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)) return KL_ERR_UNSUPPORTED_SHAPE;
    if (c->page_size < 4 || c->page_size > 1024 || c->page_size % 4) return KL_ERR_UNSUPPORTED_SHAPE;
    if (c->n_kv_heads > 65535u || c->n_pages > 0x7fffffffu) return KL_ERR_UNSUPPORTED_SHAPE;
    if (c->kv_type != KL_KV_BF16 && c->kv_type != KL_KV_E4M3) return KL_ERR_INVALID_ARG;
    if (!aligned16(c->bounds_d)) return KL_ERR_INVALID_ARG;
    if (!rows) return KL_OK;
    const int64_t bytes = c->kv_type == KL_KV_BF16 ? 2 : 1;
    const int64_t st[3] = {c->page_stride, c->head_stride, c->row_stride};
    for (int64_t x : st)
        if (x < 0 || x > (INT64_MAX >> 34) || (x * bytes) % 16) return KL_ERR_INVALID_ARG;
    if (!c->k_d || !c->v_d || !aligned16(c->k_d) || !aligned16(c->v_d)) return KL_ERR_INVALID_ARG;
    if (c->kv_type == KL_KV_E4M3 && (!c->k_exp_d || !c->v_exp_d || !aligned16(c->k_exp_d) || !aligned16(c->v_exp_d))) return KL_ERR_INVALID_ARG;
    return KL_OK;
}
inline kl_status check_seqs(const kl_paged_cache* c, const kl_paged_seqs* s) {
    if (!s) return KL_ERR_INVALID_ARG;
    if (s->n_seqs == 0) return KL_OK;
    if (!s->positions_d || !s->page_table_d) return KL_ERR_INVALID_ARG;
    if (!s->table_pages || s->table_stride < (int64_t)s->table_pages || s->table_stride > (INT64_MAX >> 34)) return KL_ERR_INVALID_ARG;
    if ((uint64_t)s->table_pages * c->page_size > 0x7fffffffull || s->n_seqs > 0x7fffffffu) return KL_ERR_UNSUPPORTED_SHAPE;
    return KL_OK;
}

inline PagedView view(const kl_paged_cache* c, const kl_paged_seqs* s, int32_t* status_d) {
    PagedView v;
    const int64_t bytes = c->kv_type == KL_KV_BF16 ? 2 : 1;
    v.k = (uint8_t*)c->k_d; v.v = (uint8_t*)c->v_d;
    v.ke = c->k_exp_d; v.ve = c->v_exp_d;
    v.bounds = (__nv_bfloat16*)c->bounds_d;
    v.page_b = c->page_stride * bytes; v.head_b = c->head_stride * bytes; v.row_b = c->row_stride * bytes;
    v.nkv = c->n_kv_heads; v.hd = c->head_dim; v.page = c->page_size; v.n_pages = c->n_pages; v.fp8 = c->kv_type == KL_KV_E4M3;
    v.positions = s->positions_d; v.table = s->page_table_d; v.table_stride = s->table_stride;
    v.table_pages = s->table_pages; v.n_seqs = s->n_seqs;
    v.status = status_d;
    return v;
}

inline kl_status check_rows(const kl_paged_cache* c, const kl_paged_seqs* s, const int32_t* row_starts_d, uint32_t n_rows, const void* k,
                     const void* v, int type, int64_t ks, int64_t vs) {
    if (type != KL_F32 && type != KL_BF16) return KL_ERR_INVALID_ARG;
    if (!row_starts_d && n_rows != s->n_seqs) return KL_ERR_INVALID_ARG;
    if (n_rows > 0x7fffffffu) return KL_ERR_UNSUPPORTED_SHAPE;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return KL_ERR_INVALID_ARG;
    const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
    if (n_rows > 1)   // the stride of a single row means nothing
        for (int64_t x : {ks, vs})
            if (x < width || x > (INT64_MAX >> 34) || (x * elem(type)) % 16) return KL_ERR_INVALID_ARG;
    return KL_OK;
}

inline PagedRows rows_of(const int32_t* row_starts_d, uint32_t n_rows, const void* k, const void* v, int type, int64_t ks, int64_t vs) {
    PagedRows r;
    r.row_starts = row_starts_d;
    r.n_rows = n_rows;
    r.k = (uint8_t*)const_cast<void*>(k);
    r.v = (uint8_t*)const_cast<void*>(v);
    r.k_stride = ks * elem(type);
    r.v_stride = vs * elem(type);
    return r;
}

inline kl_status check_queries(const kl_paged_cache* c, const void* q, int type, int64_t stride, uint32_t n_q_heads, uint32_t n_seqs) {
    if (!q || (type != KL_F32 && type != KL_BF16)) return KL_ERR_INVALID_ARG;
    if (!n_q_heads || n_q_heads % c->n_kv_heads) return KL_ERR_UNSUPPORTED_SHAPE;
    if ((uint64_t)n_q_heads * c->head_dim > 0x7fffffffull || n_q_heads > 65535u) return KL_ERR_UNSUPPORTED_SHAPE;
    if (!aligned16(q)) return KL_ERR_INVALID_ARG;
    if (n_seqs > 1 && (stride < (int64_t)n_q_heads * c->head_dim || stride > (INT64_MAX >> 34) || (stride * elem(type)) % 16)) return KL_ERR_INVALID_ARG;
    return KL_OK;
}

// Function attributes hold per device: set them on a kernel's first launch there (`done`: one bit per device; devices
// beyond 63 set them every time).
inline kl_status prepare(const void* f, int smem, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return KL_ERR_CUDA;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return KL_OK;
    if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return KL_ERR_CUDA;
    done.fetch_or(bit, std::memory_order_relaxed);
    return KL_OK;
}

}  // namespace kl
