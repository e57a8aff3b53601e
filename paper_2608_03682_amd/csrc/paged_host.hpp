// The checked launches of the paged cache, for the C entry points and for the model
// paths that run on it.  They throw Fail (errors.hpp).
#pragma once

#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "phyai.h"

namespace phyai {

// Checks the cache and gives one layer of it to a kernel.
PagePool page_pool(const phyai_paged_cache* cache, int layer);
int pool_kind(const phyai_paged_cache* cache);

void enqueue_norm_rope(const phyai_head_rows* q, const phyai_head_rows* k, const phyai_head_rows* q_out,
                       const phyai_head_rows* k_out, const float* q_gain, const float* k_gain, float eps,
                       float rope_base, const int32_t* past_len, const int32_t* new_len, int batch, int rows,
                       int head_dim, int dtype, int32_t* status, hipStream_t s);
void enqueue_append(const phyai_paged_cache* cache, int layer, const phyai_head_rows* k, const phyai_head_rows* v,
                    float rope_base, const int32_t* past_len, const int32_t* new_len, int rows, int dtype,
                    int32_t* status, hipStream_t s);
int64_t attention_workspace(const phyai_paged_cache* cache, int n_q_heads, int rows, int max_kv_len);
void enqueue_attention(const phyai_paged_cache* cache, int layer, const phyai_head_rows* q, const phyai_head_rows* out,
                       const int32_t* kv_len, const int32_t* new_len, int max_kv_len, float scale, int causal,
                       int window, int rows, int dtype, void* workspace, int64_t workspace_bytes, int32_t* status,
                       hipStream_t s);

}  // namespace phyai
