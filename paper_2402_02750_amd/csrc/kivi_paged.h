// The paged cache inside the library (include/kivi.h describes it): what its two kernels share.
#pragma once

#include "kivi_head_rows.h"

namespace kivi {

constexpr int record_bytes(int bits) { return 1024 + 2 * kTileTokens * kHeadDim * bits / 8; }

struct PagedParams {
    char* pages;
    __half *k_resid, *v_resid;
    const int32_t* page_table;
    const int32_t* lengths;
    const int32_t* slots;              // null: sequence b has the fp16 rows b
    int64_t page_table_stride;
    int32_t batch, max_pages, n_pages, max_sequences;
    int32_t n_q_heads, n_kv_heads, bits, residual, cap_r;
    int32_t page_shift;                // log2(records per page and kv-head)
};

// records of a sequence of n tokens
__host__ __device__ inline int packed_records(int n, int residual) { return n > residual ? (n - residual) / kTileTokens : 0; }

struct PagedAppendParams : PagedParams {
    head_rows::TensorParams k, v, q, q_out;        // q_out.data null: no queries
    const int32_t* starts;                         // null: max_new rows per sequence
    int32_t n_rows, max_new, bf16;
    int32_t rotates;
    head_rows::RotationParams rotation;            // positions null: the place in the sequence
};
hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t stream);

struct PagedAttentionParams : PagedParams {
    const __half* q;
    void* out;
    int32_t out_bf16, window, sinks;
    float softmax_scale;
    int32_t* counters;                 // workspace, see kivi_paged_attention.hip
    float *part_ml, *part_o;
};
hipError_t launch_paged_attention(const PagedAttentionParams& p, hipStream_t stream);
size_t paged_workspace_bytes();

}  // namespace kivi
