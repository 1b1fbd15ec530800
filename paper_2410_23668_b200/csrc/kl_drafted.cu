// Host side of the operators for drafted tokens on a paged cache (contracts in include/kl.h, kernels in kl_drafted.cuh).
#include "kl_drafted.cuh"

#include <math.h>

#include "kl_paged_host.h"

using namespace kl;

namespace {

template <class T, int HD, int THREADS>
kl_status launch_rotate_of(const PagedView& v, const PagedRows& r, const RotateArgs& a, unsigned blocks, PagedOrder order) {
    constexpr size_t smem = rt_smem_bytes<HD, THREADS>();
    auto go = [&](auto* f, std::atomic<uint64_t>& done) {
        const kl_status rc = prepare((const void*)f, (int)smem, done);
        return rc != KL_OK ? rc : launch(f, dim3(blocks), THREADS, smem, order, v, r, a);
    };
    static std::atomic<uint64_t> done8{0}, done16{0};
    return v.fp8 ? go(kl_paged_append_rotated_kernel<T, HD, true, THREADS>, done8) : go(kl_paged_append_rotated_kernel<T, HD, false, THREADS>, done16);
}
// One row of every sequence: blocks of 256 threads begin sooner (one row 4.3 us, with 512 threads 6.3); several: twice as many rows share a
// block's angles (32 x 8 rows 7.8 us instead of 10.5, 8191 rows with 32 query heads 60 instead of 66).
template <class T, int HD>
kl_status launch_rotate(const PagedView& v, const PagedRows& r, const RotateArgs& a, unsigned blocks, PagedOrder order) {
    return r.row_starts ? launch_rotate_of<T, HD, RT_MANY>(v, r, a, blocks, order) : launch_rotate_of<T, HD, RT_FEW>(v, r, a, blocks, order);
}

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms;
}

// Workspace of kl_paged_tree_attention (byte offsets): two parts of a unit for every block.
struct TreeSpace { size_t part_ml, bytes; };
TreeSpace tree_space(uint32_t head_dim) {
    TreeSpace s;
    s.part_ml = (size_t)2 * TA_MAX_BLOCKS * TA_RECORD * head_dim * 4;
    s.bytes = s.part_ml + (size_t)2 * TA_MAX_BLOCKS * TA_RECORD * 8;
    if (s.bytes < paged_attention_bytes(head_dim)) s.bytes = paged_attention_bytes(head_dim);   // (single tokens)
    return s;
}

template <int HD, bool FP8>
kl_status launch_tree(const PagedView& v, const TreeArgs& a, unsigned blocks, PagedOrder order) {
    using Cfg = TaCfg<HD, FP8>;
    auto* f = kl_paged_tree_kernel<HD, FP8>;
    constexpr size_t smem = ta_smem<HD, FP8>();
    static_assert(smem <= 227 * 1024, "shared memory of a block");
    static std::atomic<uint64_t> done{0};
    kl_status rc = prepare((const void*)f, (int)smem, done);
    if (rc != KL_OK || (rc = launch(f, dim3(blocks), Cfg::NW * 32, smem, order, v, a)) != KL_OK) return rc;
    // tables of one tile leave no unit to cut
    if ((uint64_t)v.table_pages * v.page <= (uint64_t)Cfg::NK || blocks < 2) return KL_OK;
    return launch(kl_paged_tree_merge_kernel<HD, Cfg::NK, Cfg::NG * 128>, dim3(blocks - 1, 16), TA_MERGE_THREADS, 0, order, v, a, (uint32_t)blocks);
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

}  // namespace

extern "C" {

kl_status kl_paged_append_rotated(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows,
                                  const void* k_rows_d, const void* v_rows_d, int row_type, int64_t k_row_stride, int64_t v_row_stride,
                                  const double* freqs_d, const int32_t* row_positions_d, const void* q_d, void* q_out_d, int64_t q_row_stride,
                                  int64_t q_out_row_stride, uint32_t n_q_heads, int32_t* status_d, void* stream) {
    kl_status rc;
    if ((rc = check_cache(cache, true)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0 || n_rows == 0) return KL_OK;
    if ((rc = check_rows(cache, seqs, row_starts_d, n_rows, k_rows_d, v_rows_d, row_type, k_row_stride, v_row_stride)) != KL_OK) return rc;
    if (!freqs_d || ((uintptr_t)freqs_d & 7u) || !aligned4(row_starts_d) || !aligned4(row_positions_d) || (q_d != nullptr) != (q_out_d != nullptr)) return KL_ERR_INVALID_ARG;
    if (q_d && q_d == q_out_d && n_rows > 1 && q_row_stride != q_out_row_stride) return KL_ERR_INVALID_ARG;   // a row would be written before it is read
    if (q_d) {
        if ((rc = check_queries(cache, q_d, row_type, q_row_stride, n_q_heads, n_rows)) != KL_OK) return rc;
        if ((rc = check_queries(cache, q_out_d, row_type, q_out_row_stride, n_q_heads, n_rows)) != KL_OK) return rc;
    }
    const int sms = sm_count();
    if (sms <= 0) return KL_ERR_CUDA;
    const uint64_t units = row_starts_d ? (uint64_t)n_rows / cache->page_size + 2ull * seqs->n_seqs : seqs->n_seqs;
    RotateArgs a = {};
    a.freqs = freqs_d;
    a.row_positions = row_positions_d;
    // kv heads of a block: up to eight share the angles of their rows, fewer where that leaves SMs without a block
    a.heads = 8;
    while (a.heads > 1 && (a.heads > cache->n_kv_heads || units * ((cache->n_kv_heads + a.heads - 1) / a.heads) < (uint64_t)sms / 2)) a.heads /= 2;
    a.head_groups = (cache->n_kv_heads + a.heads - 1) / a.heads;
    uint64_t blocks = units * a.head_groups;
    a.q_groups = 1;
    if (q_d) {
        a.q = (const uint8_t*)q_d;
        a.q_out = (uint8_t*)q_out_d;
        a.q_stride = q_row_stride * elem(row_type);
        a.q_out_stride = q_out_row_stride * elem(row_type);
        a.nq = n_q_heads;
        const uint64_t runs = (n_rows + RT_ROWS - 1) / RT_ROWS;
        a.q_heads = n_q_heads;
        while (a.q_heads > 4 && runs * ((n_q_heads + a.q_heads - 1) / a.q_heads) < 2ull * sms) a.q_heads = (a.q_heads + 1) / 2;
        a.q_groups = (n_q_heads + a.q_heads - 1) / a.q_heads;
        blocks += runs * a.q_groups;
    }
    if (blocks > 0x7fffffffull) return KL_ERR_UNSUPPORTED_SHAPE;
    a.kv_blocks = (uint32_t)(units * a.head_groups);
    const PagedView v = view(cache, seqs, status_d);
    const PagedRows r = rows_of(row_starts_d, n_rows, k_rows_d, v_rows_d, row_type, k_row_stride, v_row_stride);
    const PagedOrder order = {stream, true};
    const bool f32 = row_type == KL_F32;
    if (v.hd == 64) return f32 ? launch_rotate<float, 64>(v, r, a, (unsigned)blocks, order) : launch_rotate<__nv_bfloat16, 64>(v, r, a, (unsigned)blocks, order);
    if (v.hd == 128) return f32 ? launch_rotate<float, 128>(v, r, a, (unsigned)blocks, order) : launch_rotate<__nv_bfloat16, 128>(v, r, a, (unsigned)blocks, order);
    return f32 ? launch_rotate<float, 256>(v, r, a, (unsigned)blocks, order) : launch_rotate<__nv_bfloat16, 256>(v, r, a, (unsigned)blocks, order);
}

kl_status kl_paged_tree_workspace_bytes(const kl_paged_cache* cache, uint32_t n_q_heads, size_t* bytes) {
    if (!bytes) return KL_ERR_INVALID_ARG;
    const kl_status rc = check_cache(cache, false);
    if (rc != KL_OK) return rc;
    if (!n_q_heads || n_q_heads % cache->n_kv_heads) return KL_ERR_UNSUPPORTED_SHAPE;
    *bytes = tree_space(cache->head_dim).bytes;
    return KL_OK;
}

kl_status kl_paged_tree_attention(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows, const void* q_d,
                                  void* out_d, int q_type, int64_t q_row_stride, int64_t out_row_stride, uint32_t n_q_heads, float scale, uint32_t window,
                                  uint32_t n_sinks, const int32_t* row_positions_d, const uint32_t* mask_d, uint32_t mask_words, float* lse_d,
                                  void* workspace_d, size_t workspace_bytes, int32_t* status_d, void* stream) {
    kl_status rc;
    if ((rc = check_cache(cache, true)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0 || n_rows == 0) return KL_OK;
    if (!row_starts_d && n_rows != seqs->n_seqs) return KL_ERR_INVALID_ARG;
    if (q_type != KL_F32 && q_type != KL_BF16) return KL_ERR_INVALID_ARG;
    if (q_type != KL_BF16 || n_rows > 0x7fffffffu) return KL_ERR_UNSUPPORTED_SHAPE;
    if ((rc = check_queries(cache, q_d, q_type, q_row_stride, n_q_heads, n_rows)) != KL_OK) return rc;
    if ((rc = check_queries(cache, out_d, q_type, out_row_stride, n_q_heads, n_rows)) != KL_OK) return rc;
    if ((uint64_t)n_rows * (n_q_heads / cache->n_kv_heads) > 0x7fffffffull) return KL_ERR_UNSUPPORTED_SHAPE;   // (token, head) pairs are counted in 32 bits
    if (!aligned4(row_starts_d) || !aligned4(row_positions_d) || !aligned4(mask_d) || !aligned4(lse_d)) return KL_ERR_INVALID_ARG;
    if (!(scale < INFINITY) || (mask_d != nullptr) != (mask_words != 0) || mask_words > (1u << 26)) return KL_ERR_INVALID_ARG;
    const TreeSpace sp = tree_space(cache->head_dim);
    if (!workspace_d || ((uintptr_t)workspace_d & 255u) || workspace_bytes < sp.bytes) return KL_ERR_INVALID_ARG;
    const float scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.4426950408889634f;
    // One token per sequence, which sees what its place says, for up to eight query heads to a kv head: the kernel of kl_paged_attention, whose
    // warps each hold all of a tile's way (32 sequences, window 2048, eight kv heads of 128, four query heads to each: e4m3 36 us instead of 83,
    // bf16 55 instead of 75).  It reads the cache once per eight query heads.
    if (!row_starts_d && !mask_d && (!row_positions_d || !window) && n_q_heads / cache->n_kv_heads <= 8)
        return paged_attention_sinks(cache, seqs, q_d, out_d, q_row_stride, out_row_stride, n_q_heads, scale_log2, window, n_sinks, lse_d, workspace_d, workspace_bytes,
                                     status_d, {stream, true});
    const int sms = sm_count();
    if (sms <= 0) return KL_ERR_CUDA;
    const unsigned blocks = (unsigned)(sms < TA_MAX_BLOCKS ? sms : TA_MAX_BLOCKS);
    const PagedView v = view(cache, seqs, status_d);
    TreeArgs a = {};
    a.row_starts = row_starts_d;
    a.n_rows = n_rows;
    a.q = (const uint8_t*)q_d;
    a.out = (uint8_t*)out_d;
    a.q_stride = q_row_stride * 2;
    a.out_stride = out_row_stride * 2;
    a.nq = n_q_heads;
    a.G = n_q_heads / cache->n_kv_heads;
    a.scale_log2 = scale_log2;
    a.window = window;
    a.sinks = n_sinks;
    a.row_positions = row_positions_d;
    a.mask = mask_d;
    a.mask_words = mask_words;
    a.lse = lse_d;
    a.part = (float*)workspace_d;
    a.part_ml = (float2*)((uint8_t*)workspace_d + sp.part_ml);
    const PagedOrder order = {stream, true};
    if (v.hd == 64) return v.fp8 ? launch_tree<64, true>(v, a, blocks, order) : launch_tree<64, false>(v, a, blocks, order);
    if (v.hd == 128) return v.fp8 ? launch_tree<128, true>(v, a, blocks, order) : launch_tree<128, false>(v, a, blocks, order);
    return v.fp8 ? launch_tree<256, true>(v, a, blocks, order) : launch_tree<256, false>(v, a, blocks, order);
}

}  // extern "C"
