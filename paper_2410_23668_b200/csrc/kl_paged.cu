// Host side of the paged key-value cache operators (contracts in include/kl.h, kernels in kl_paged.cuh).
#include "kl_paged.cuh"

#include <math.h>
#include <string.h>

#include <atomic>
#include <utility>

#include "kl_paged_host.h"
#include "kl_paged_internal.h"

using namespace kl;

namespace {

// Workspace of kl_paged_select; false where no address space holds it.
bool score_bytes(const kl_paged_cache* c, uint64_t n_seqs, uint64_t table_pages, size_t* bytes) {
    const uint64_t pairs = n_seqs * c->n_kv_heads;   // below 2^48
    if (table_pages && pairs > (1ull << 56) / table_pages) return false;
    *bytes = (size_t)((pairs * table_pages * 8 + 255) / 256 * 256);
    return true;
}

// Workspace of kl_paged_attention (byte offsets): room for PA_MAX_BLOCKS blocks of PA_MAX_WARPS warps.
struct AttnSpace { size_t part, part_ml, head, head_ml, meta, bytes; };
AttnSpace attn_space(uint32_t head_dim) {
    AttnSpace s;
    const size_t rec = (size_t)8 * head_dim * 4, ml = 8 * 8;
    s.part = 0;
    s.head = s.part + 2 * PA_MAX_BLOCKS * rec;
    s.part_ml = s.head + PA_MAX_WARPS * PA_MAX_BLOCKS * rec;
    s.head_ml = s.part_ml + 2 * PA_MAX_BLOCKS * ml;
    s.meta = s.head_ml + PA_MAX_WARPS * PA_MAX_BLOCKS * ml;
    s.bytes = s.meta + PA_MAX_BLOCKS * sizeof(int4);
    return s;
}

// Blocks of the attention grid: one per SM.
int attn_blocks() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms < PA_MAX_BLOCKS ? sms : PA_MAX_BLOCKS;
}

template <int HD>
kl_status launch_append(int type, const PagedView& v, const PagedRows& r, dim3 grid, size_t smem, PagedOrder order) {
    if (v.fp8)
        return type == KL_F32 ? launch(kl_paged_append_kernel<float, HD, true>, grid, PW_THREADS, smem, order, v, r)
                              : launch(kl_paged_append_kernel<__nv_bfloat16, HD, true>, grid, PW_THREADS, smem, order, v, r);
    return type == KL_F32 ? launch(kl_paged_append_kernel<float, HD, false>, grid, PW_THREADS, smem, order, v, r)
                          : launch(kl_paged_append_kernel<__nv_bfloat16, HD, false>, grid, PW_THREADS, smem, order, v, r);
}
template <int HD>
kl_status launch_read(int type, const PagedView& v, const PagedRows& r, dim3 grid, PagedOrder order) {
    if (v.fp8)
        return type == KL_F32 ? launch(kl_paged_read_kernel<float, HD, true>, grid, PG_THREADS, 0, order, v, r)
                              : launch(kl_paged_read_kernel<__nv_bfloat16, HD, true>, grid, PG_THREADS, 0, order, v, r);
    return type == KL_F32 ? launch(kl_paged_read_kernel<float, HD, false>, grid, PG_THREADS, 0, order, v, r)
                          : launch(kl_paged_read_kernel<__nv_bfloat16, HD, false>, grid, PG_THREADS, 0, order, v, r);
}

template <int HD, bool F32>
kl_status launch_score_as(const PagedView& v, const PagedSelect& a, int sms, PagedOrder order) {
    using Cfg = PsCfg<HD>;
    auto* f = kl_paged_score_kernel<HD, F32>;
    static std::atomic<uint64_t> done{0};
    const kl_status rc = prepare((const void*)f, (int)Cfg::SMEM, done);
    return rc != KL_OK ? rc : launch(f, dim3((unsigned)sms), Cfg::NW * 32, Cfg::SMEM, order, v, a);
}
kl_status launch_score(const PagedView& v, const PagedSelect& a, int sms, PagedOrder order) {
    if (v.hd == 64) return a.q_f32 ? launch_score_as<64, true>(v, a, sms, order) : launch_score_as<64, false>(v, a, sms, order);
    if (v.hd == 128) return a.q_f32 ? launch_score_as<128, true>(v, a, sms, order) : launch_score_as<128, false>(v, a, sms, order);
    return a.q_f32 ? launch_score_as<256, true>(v, a, sms, order) : launch_score_as<256, false>(v, a, sms, order);
}

template <int HD, bool FP8, int UR, bool EX>
kl_status launch_attn_as(const PagedView& v, const PagedAttn& a, int blocks, PagedOrder order) {
    using Cfg = PaCfg<HD, FP8, EX>;
    auto* f = kl_paged_attn_kernel<HD, FP8, UR, EX>;
    static std::atomic<uint64_t> done{0};
    const kl_status rc = prepare((const void*)f, (int)Cfg::SMEM, done);
    if (rc != KL_OK) return rc;
    return launch(f, dim3((unsigned)blocks), Cfg::NW * 32, Cfg::SMEM, order, v, a);
}
template <int HD, bool FP8>
kl_status launch_attn_hd(const PagedView& v, const PagedAttn& a, int blocks, PagedOrder order) {
    // pages are looked up in units of 16 rows where they consist of such units, else of four
    const bool whole = v.page % 16 == 0, ex = a.out_mode != PA_BF16;
    if (ex) return whole ? launch_attn_as<HD, FP8, 16, true>(v, a, blocks, order) : launch_attn_as<HD, FP8, 4, true>(v, a, blocks, order);
    return whole ? launch_attn_as<HD, FP8, 16, false>(v, a, blocks, order) : launch_attn_as<HD, FP8, 4, false>(v, a, blocks, order);
}
// Positions per tile of the kernel that a call takes.
uint32_t attn_tile(const PagedView& v, uint32_t out_mode) {
    const bool ex = out_mode != PA_BF16;
    if (v.hd == 64) return v.fp8 ? PaCfg<64, true, false>::TP : PaCfg<64, false, false>::TP;
    if (v.hd == 128) return v.fp8 ? (ex ? PaCfg<128, true, true>::TP : PaCfg<128, true, false>::TP) : PaCfg<128, false, false>::TP;
    return v.fp8 ? PaCfg<256, true, false>::TP : PaCfg<256, false, false>::TP;
}
kl_status launch_attn(const PagedView& v, const PagedAttn& a, int blocks, PagedOrder order) {
    if (v.hd == 64) return v.fp8 ? launch_attn_hd<64, true>(v, a, blocks, order) : launch_attn_hd<64, false>(v, a, blocks, order);
    if (v.hd == 128) return v.fp8 ? launch_attn_hd<128, true>(v, a, blocks, order) : launch_attn_hd<128, false>(v, a, blocks, order);
    return v.fp8 ? launch_attn_hd<256, true>(v, a, blocks, order) : launch_attn_hd<256, false>(v, a, blocks, order);
}

// Both ways into the attention kernels.
kl_status run_attention(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, void* out_d, int q_type, uint32_t out_mode,
                        int64_t q_row_stride, int64_t out_row_stride, uint32_t n_q_heads, float scale_log2, uint32_t window, uint32_t n_sinks,
                        const int32_t* selected_d, uint32_t n_select, float* lse_d, void* workspace_d, size_t workspace_bytes,
                        int32_t* status_d, uint64_t* launches, PagedOrder order, bool leave_empty = false) {
    if ((selected_d != nullptr) != (n_select != 0) || n_select > 0x7fffffffu) return KL_ERR_INVALID_ARG;
    const AttnSpace sp = attn_space(cache->head_dim);
    if (!workspace_d || ((uintptr_t)workspace_d & 255u) || workspace_bytes < sp.bytes) return KL_ERR_INVALID_ARG;
    const int blocks = attn_blocks();
    if (blocks <= 0) return KL_ERR_CUDA;
    uint8_t* ws = (uint8_t*)workspace_d;
    const PagedView v = view(cache, seqs, status_d);
    PagedAttn a;
    a.q = (const uint8_t*)q_d;
    a.out = (uint8_t*)out_d;
    a.q_stride = q_row_stride * elem(q_type);
    a.out_stride = out_row_stride * elem(q_type);
    a.out_mode = out_mode;
    a.nq = n_q_heads;
    a.G = n_q_heads / cache->n_kv_heads;
    a.HT = (a.G + 7) / 8;
    a.scale_log2 = scale_log2;
    a.window = window;
    a.sinks = n_sinks;
    a.leave_empty = leave_empty;
    a.selected = selected_d;
    a.n_select = n_select;
    a.lse = lse_d;
    a.part = (float*)(ws + sp.part);
    a.part_ml = (float*)(ws + sp.part_ml);
    a.head = (float*)(ws + sp.head);
    a.head_ml = (float*)(ws + sp.head_ml);
    a.meta = (int4*)(ws + sp.meta);
    // the longest a pair can be, by the page table, the page list and the window
    uint64_t most = (uint64_t)seqs->table_pages * cache->page_size;
    if (selected_d && (uint64_t)n_select * cache->page_size < most) most = (uint64_t)n_select * cache->page_size;
    if (!selected_d && window && (uint64_t)window + 64 < most) most = (uint64_t)window + 64;   // a window may begin inside a tile
    if (!selected_d && window && n_sinks) most += (uint64_t)n_sinks + 64;
    const bool many = (uint64_t)seqs->n_seqs * cache->n_kv_heads * a.HT >= (uint64_t)blocks;
    a.whole_pairs = most <= (uint64_t)(many ? PA_WHOLE_MANY : PA_WHOLE_FEW) * attn_tile(v, out_mode);
    if (launches) *launches = a.whole_pairs ? 1 : 2;
    const kl_status rc = launch_attn(v, a, blocks, order);
    if (rc != KL_OK || a.whole_pairs) return rc;
    return launch(kl_paged_merge_kernel, dim3((unsigned)blocks, a.G < 8 ? a.G : 8), PA_MERGE_THREADS, 0, order, v, a);
}

}  // namespace

namespace kl {
kl_status paged_check(const kl_paged_cache* cache, const kl_paged_seqs* seqs) {
    const kl_status rc = check_cache(cache, true);
    return rc != KL_OK ? rc : check_seqs(cache, seqs);
}

kl_status paged_append(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows,
                       const void* k_rows_d, const void* v_rows_d, int row_type, int64_t k_row_stride, int64_t v_row_stride,
                       int32_t* status_d, PagedOrder order) {
    kl_status rc;
    if ((rc = check_cache(cache, true)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0 || n_rows == 0) return KL_OK;
    if ((rc = check_rows(cache, seqs, row_starts_d, n_rows, k_rows_d, v_rows_d, row_type, k_row_stride, v_row_stride)) != KL_OK) return rc;
    const uint64_t units = row_starts_d ? (uint64_t)n_rows / cache->page_size + 2ull * seqs->n_seqs : seqs->n_seqs;
    if (units > 0x7fffffffull) return KL_ERR_UNSUPPORTED_SHAPE;
    const PagedView v = view(cache, seqs, status_d);
    const PagedRows r = rows_of(row_starts_d, n_rows, k_rows_d, v_rows_d, row_type, k_row_stride, v_row_stride);
    const size_t smem = cache->bounds_d ? (size_t)(PW_THREADS / (cache->head_dim / 8) / 2) * 2 * cache->head_dim * 4 : 0;
    const dim3 grid((unsigned)units, cache->n_kv_heads);
    if (v.hd == 64) return launch_append<64>(row_type, v, r, grid, smem, order);
    if (v.hd == 128) return launch_append<128>(row_type, v, r, grid, smem, order);
    return launch_append<256>(row_type, v, r, grid, smem, order);
}

kl_status paged_select(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, int q_type, int64_t q_row_stride,
                       uint32_t n_q_heads, uint32_t keep_first, uint32_t keep_last, uint32_t n_select, int32_t* selected_d,
                       void* workspace_d, size_t workspace_bytes, int32_t* status_d, PagedOrder order) {
    kl_status rc;
    if ((rc = check_cache(cache, false)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0) return KL_OK;
    if ((rc = check_queries(cache, q_d, q_type, q_row_stride, n_q_heads, seqs->n_seqs)) != KL_OK) return rc;
    if (!cache->bounds_d || !selected_d) return KL_ERR_INVALID_ARG;
    if (!n_select || (uint64_t)keep_first + keep_last > n_select || n_select > 0x7fffffffu) return KL_ERR_INVALID_ARG;
    size_t need;
    if (seqs->n_seqs > 65535u || !score_bytes(cache, seqs->n_seqs, seqs->table_pages, &need)) return KL_ERR_UNSUPPORTED_SHAPE;
    if (!workspace_d || ((uintptr_t)workspace_d & 255u) || workspace_bytes < need) return KL_ERR_INVALID_ARG;
    const PagedView v = view(cache, seqs, status_d);
    PagedSelect a;
    a.q = (const uint8_t*)q_d;
    a.q_stride = q_row_stride * elem(q_type);
    a.q_f32 = q_type == KL_F32;
    a.G = n_q_heads / cache->n_kv_heads;
    a.keep_first = keep_first; a.keep_last = keep_last; a.n_select = n_select;
    a.selected = selected_d;
    a.scores = (float2*)workspace_d;
    const int sms = attn_blocks();
    if (sms <= 0) return KL_ERR_CUDA;
    if ((rc = launch_score(v, a, sms, order)) != KL_OK) return rc;
    // keys in shared memory up to PT_KEYS pages, else in the workspace
    const dim3 grid(cache->n_kv_heads, seqs->n_seqs);
    if (seqs->table_pages > PT_KEYS) return launch(kl_paged_topk_kernel<false>, grid, PT_THREADS, 0, order, v, a);
    static std::atomic<uint64_t> done{0};
    if ((rc = prepare((const void*)kl_paged_topk_kernel<true>, (int)PT_KEYS * 4, done)) != KL_OK) return rc;
    return launch(kl_paged_topk_kernel<true>, grid, PT_THREADS, (size_t)seqs->table_pages * 4, order, v, a);
}

kl_status paged_attention_operand(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const float* q_d, __nv_bfloat16* operand_d,
                                  uint32_t n_q_heads, const int32_t* selected_d, uint32_t n_select, void* workspace_d,
                                  size_t workspace_bytes, int32_t* status_d, uint64_t* launches, PagedOrder order) {
    const int64_t width = (int64_t)n_q_heads * cache->head_dim;
    return run_attention(cache, seqs, q_d, operand_d, KL_F32, PA_OPERAND, width, width, n_q_heads, 1.f, 0, 0, selected_d, n_select, nullptr, workspace_d,
                         workspace_bytes, status_d, launches, order);
}
size_t paged_attention_bytes(uint32_t head_dim) { return attn_space(head_dim).bytes; }

kl_status paged_attention_sinks(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, void* out_d, int64_t q_row_stride, int64_t out_row_stride,
                                uint32_t n_q_heads, float scale_log2, uint32_t window, uint32_t n_sinks, float* lse_d, void* workspace_d,
                                size_t workspace_bytes, int32_t* status_d, PagedOrder order) {
    const uint32_t most = seqs->table_pages * cache->page_size;   // (below 2^31)
    return run_attention(cache, seqs, q_d, out_d, KL_BF16, PA_BF16, q_row_stride, out_row_stride, n_q_heads, scale_log2, window, n_sinks < most ? n_sinks : most,
                         nullptr, 0, lse_d, workspace_d, workspace_bytes, status_d, nullptr, order, true);
}
}  // namespace kl

extern "C" {

kl_status kl_paged_append(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows,
                          const void* k_rows_d, const void* v_rows_d, int row_type, int64_t k_row_stride, int64_t v_row_stride,
                          int32_t* status_d, void* stream) {
    return paged_append(cache, seqs, row_starts_d, n_rows, k_rows_d, v_rows_d, row_type, k_row_stride, v_row_stride, status_d, {stream, true});
}

kl_status kl_paged_read(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows,
                        void* k_out_d, void* v_out_d, int row_type, int64_t k_row_stride, int64_t v_row_stride,
                        int32_t* status_d, void* stream) {
    kl_status rc;
    if ((rc = check_cache(cache, true)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0 || n_rows == 0) return KL_OK;
    if ((rc = check_rows(cache, seqs, row_starts_d, n_rows, k_out_d, v_out_d, row_type, k_row_stride, v_row_stride)) != KL_OK) return rc;
    const PagedView v = view(cache, seqs, status_d);
    const PagedOrder order = {stream, true};
    const PagedRows r = rows_of(row_starts_d, n_rows, k_out_d, v_out_d, row_type, k_row_stride, v_row_stride);
    const uint32_t per = pr_rows(cache->n_kv_heads, cache->head_dim / 8), chunks = (n_rows + per - 1) / per;
    const int sms = attn_blocks();
    if (sms <= 0) return KL_ERR_CUDA;
    const dim3 grid(chunks < 4u * (unsigned)sms ? chunks : 4u * (unsigned)sms);   // as many blocks as the SMs hold
    if (v.hd == 64) return launch_read<64>(row_type, v, r, grid, order);
    if (v.hd == 128) return launch_read<128>(row_type, v, r, grid, order);
    return launch_read<256>(row_type, v, r, grid, order);
}

kl_status kl_paged_workspace_bytes(const kl_paged_cache* cache, uint32_t n_q_heads, uint32_t n_seqs, uint32_t table_pages, size_t* bytes) {
    if (!bytes) return KL_ERR_INVALID_ARG;
    const kl_status rc = check_cache(cache, false);
    if (rc != KL_OK) return rc;
    if (!n_q_heads || n_q_heads % cache->n_kv_heads) return KL_ERR_UNSUPPORTED_SHAPE;
    size_t sel;
    if (!score_bytes(cache, n_seqs, table_pages, &sel)) return KL_ERR_UNSUPPORTED_SHAPE;
    const size_t att = attn_space(cache->head_dim).bytes;
    *bytes = sel > att ? sel : att;
    return KL_OK;
}

kl_status kl_paged_select(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, int q_type, int64_t q_row_stride,
                          uint32_t n_q_heads, uint32_t keep_first, uint32_t keep_last, uint32_t n_select, int32_t* selected_d,
                          void* workspace_d, size_t workspace_bytes, int32_t* status_d, void* stream) {
    return paged_select(cache, seqs, q_d, q_type, q_row_stride, n_q_heads, keep_first, keep_last, n_select, selected_d, workspace_d, workspace_bytes,
                        status_d, {stream, true});
}

kl_status kl_paged_attention(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, void* out_d, int q_type,
                             int64_t q_row_stride, int64_t out_row_stride, uint32_t n_q_heads, float scale, uint32_t window,
                             const int32_t* selected_d, uint32_t n_select, float* lse_d, void* workspace_d, size_t workspace_bytes,
                             int32_t* status_d, void* stream) {
    kl_status rc;
    if ((rc = check_cache(cache, true)) != KL_OK || (rc = check_seqs(cache, seqs)) != KL_OK) return rc;
    if (seqs->n_seqs == 0) return KL_OK;
    if ((rc = check_queries(cache, q_d, q_type, q_row_stride, n_q_heads, seqs->n_seqs)) != KL_OK) return rc;
    if ((rc = check_queries(cache, out_d, q_type, out_row_stride, n_q_heads, seqs->n_seqs)) != KL_OK) return rc;
    if (!(scale < INFINITY)) return KL_ERR_INVALID_ARG;
    const float scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.4426950408889634f;
    return run_attention(cache, seqs, q_d, out_d, q_type, q_type == KL_F32 ? PA_F32 : PA_BF16, q_row_stride, out_row_stride, n_q_heads, scale_log2,
                         window, 0, selected_d, n_select, lse_d, workspace_d, workspace_bytes, status_d, nullptr, {stream, true});
}

}  // extern "C"
