// What the decode step on a paged cache (kl.cu) needs of the paged operators (kl_paged.cu) beyond their public entry points.
#pragma once

#include <cuda_bf16.h>

#include "../../include/kl.h"

namespace kl {

// kl_paged_attention for the step: fp32 queries [n_seqs][n_q_heads * head_dim] that carry the factor log2(e) / sqrt(head_dim)
// already, and the result as the operand of a batched projection ([64][n_q_heads * head_dim]: rows 0..31 the bf16 hi halves,
// rows 32..63 the lo halves).  At most 32 sequences.  *launches: the kernels it launched.
kl_status paged_attention_operand(const kl_paged_cache* cache, const kl_paged_seqs* seqs, const float* q_d, __nv_bfloat16* operand_d,
                                  uint32_t n_q_heads, const int32_t* selected_d, uint32_t n_select, void* workspace_d,
                                  size_t workspace_bytes, int32_t* status_d, uint64_t* launches, void* stream);

// What every operator that touches rows checks of its descriptors.
kl_status paged_check(const kl_paged_cache* cache, const kl_paged_seqs* seqs);

}  // namespace kl
