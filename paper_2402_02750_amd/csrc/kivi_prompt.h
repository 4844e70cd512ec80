// Attention of prompts inside the library: arguments of its kernel (kivi_prompt_attention.hip).
#pragma once

#include "kivi_head_rows.h"

namespace kivi {

struct PromptParams {
    head_rows::TensorParams q, k, v, out;
    const int32_t *q_starts, *k_starts;            // null: max_q, max_k rows per sequence
    int32_t batch, n_q_heads, n_kv_heads, bf16;
    int32_t max_q, max_k, q_rows, k_rows;
    int32_t window, sinks;
    float softmax_scale;
};
hipError_t launch_prompt_attention(const PromptParams& p, void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t prompt_workspace_bytes(const PromptParams& p);

}  // namespace kivi
