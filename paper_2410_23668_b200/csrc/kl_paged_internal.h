// What the decode step on a paged cache (kl.cu) needs of the paged operators (kl_paged.cu) beyond their public entry points.
#pragma once

#include <cuda_bf16.h>

#include "../../include/kl.h"

namespace kl {

// Where an operator's kernels are launched, and whether each may start while the kernel in front of it still runs (the operators'
// public entry points: always; a step: as kl_set_dependent_launch says).
struct PagedOrder {
    void* stream;
    bool early;
};

// kl_paged_append and kl_paged_select.
kl_status paged_append(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const int32_t* row_starts_d, uint32_t n_rows, const void* k_rows_d,
                       const void* v_rows_d, int row_type, int64_t k_row_stride, int64_t v_row_stride, int32_t* status_d, PagedOrder order);
kl_status paged_select(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const void* q_d, int q_type, int64_t q_row_stride,
                       uint32_t n_q_heads, uint32_t keep_first, uint32_t keep_last, uint32_t n_select, int32_t* selected_d, void* workspace_d,
                       size_t workspace_bytes, int32_t* status_d, PagedOrder order);

// kl_paged_attention for the step: fp32 queries [n_seqs][n_q_heads * head_dim] that carry the factor log2(e) / sqrt(head_dim)
// already, and the result as the operand of a batched projection ([64][n_q_heads * head_dim]: rows 0..31 the bf16 hi halves,
// rows 32..63 the lo halves).  At most 32 sequences.  *launches: the kernels it launched.
kl_status paged_attention_operand(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const float* q_d, __nv_bfloat16* operand_d,
                                  uint32_t n_q_heads, const int32_t* selected_d, uint32_t n_select, void* workspace_d,
                                  size_t workspace_bytes, int32_t* status_d, uint64_t* launches, PagedOrder order);

// What every operator that touches rows checks of its descriptors.
kl_status paged_check(const kl_paged_cache* cache, const kl_paged_seqs* seqs);

}  // namespace kl
