// Implementation of the second half of include/kivi.h: argument checks of the operators around the cache, and the hand-over to their
// launchers.  Nothing is enqueued before every check has passed.
#include "kivi_paged.h"
#include "kivi_prompt.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

using namespace kivi;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? KIVI_OK : e == hipErrorNotSupported ? KIVI_ERR_UNSUPPORTED : e == hipErrorInvalidValue ? KIVI_ERR_INVALID_ARG : KIVI_ERR_HIP; }
bool known_type(int t) { return t == KIVI_TYPE_FP16 || t == KIVI_TYPE_BF16; }

// a product of counts, if it is at most `limit`
bool fits(int64_t limit, std::initializer_list<int64_t> counts) {
    __int128 product = 1;
    for (const int64_t n : counts) {
        product *= n;
        if (product > limit) return false;
    }
    return true;
}
constexpr int64_t kMaxBytes = (int64_t)1 << 62;

// a tensor that is read; strides may be 0 (broadcast)
int check_read(const kivi_tensor_t& t) {
    if (!t.data || !aligned16(t.data)) return KIVI_ERR_INVALID_ARG;
    if (t.stride_b < 0 || t.stride_h < 0 || t.stride_t < 0 || ((t.stride_b | t.stride_h | t.stride_t) & 7)) return KIVI_ERR_INVALID_ARG;
    return KIVI_OK;
}
// ... that is written: no two heads, rows or batch entries at one place (whichever of the three is the innermost, each steps over all of the one inside)
int check_written(const kivi_tensor_t& t, int64_t batch, int64_t heads, int64_t rows) {
    if (const int st = check_read(t)) return st;
    std::pair<int64_t, int64_t> dims[3] = {{t.stride_b, batch}, {t.stride_h, heads}, {t.stride_t, rows}};
    std::sort(dims, dims + 3);
    __int128 span = kHeadDim;
    for (const auto& [stride, n] : dims)
        if (n > 1) {
            if (stride < span) return KIVI_ERR_INVALID_ARG;
            span += (__int128)stride * (n - 1);
        }
    return KIVI_OK;
}
int check_rotation(const kivi_rotation_t* r, bool positions_needed) {
    if (!r) return KIVI_OK;
    if (!r->table || !aligned16(r->table) || r->n_positions < 1) return KIVI_ERR_INVALID_ARG;
    if ((positions_needed && !r->positions) || !aligned4(r->positions)) return KIVI_ERR_INVALID_ARG;
    if (r->interleaved != 0 && r->interleaved != 1) return KIVI_ERR_INVALID_ARG;
    if (r->rotary_dim < 1 || r->rotary_dim > kHeadDim) return KIVI_ERR_INVALID_ARG;
    if (r->rotary_dim % 16 != 0) return KIVI_ERR_UNSUPPORTED;
    return KIVI_OK;
}
head_rows::RotationParams rotation_params(const kivi_rotation_t* r) {
    if (!r) return head_rows::RotationParams{nullptr, nullptr, 1, 0, 0};
    return head_rows::RotationParams{r->table, r->positions, r->n_positions, r->rotary_dim / 2, r->interleaved};
}
head_rows::TensorParams tensor_params(const kivi_tensor_t& t) {
    return head_rows::TensorParams{static_cast<__half*>(t.data), t.stride_b, t.stride_h, t.stride_t};
}

int check_prompt(const kivi_prompt_t* p) {
    if (!p || p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) return KIVI_ERR_INVALID_ARG;
    if (p->max_q < 0 || p->max_k < 0 || p->window < 0 || p->sinks < 0 || !std::isfinite(p->softmax_scale)) return KIVI_ERR_INVALID_ARG;
    if (!aligned4(p->q_starts) || !aligned4(p->k_starts) || (p->q_starts && p->q_rows < 0) || (p->k_starts && p->k_rows < 0)) return KIVI_ERR_INVALID_ARG;
    if (p->head_dim != kHeadDim || !known_type(p->type)) return KIVI_ERR_UNSUPPORTED;
    // (counted in 32 bits)
    if (!fits(0x7fffffff, {p->batch, p->n_kv_heads}) || !fits(0x3fffffff, {p->max_q, p->n_q_heads / p->n_kv_heads})) return KIVI_ERR_UNSUPPORTED;
    return KIVI_OK;
}
PromptParams prompt_params(const kivi_prompt_t* p) {
    PromptParams r{};
    r.q_starts = p->q_starts; r.k_starts = p->k_starts;
    r.batch = p->batch; r.n_q_heads = p->n_q_heads; r.n_kv_heads = p->n_kv_heads; r.bf16 = p->type == KIVI_TYPE_BF16;
    r.max_q = p->max_q; r.max_k = p->max_k; r.q_rows = p->q_rows; r.k_rows = p->k_rows;
    r.window = p->window < p->max_k ? p->window : 0;       // (one that no sequence is longer than hides nothing)
    r.sinks = p->sinks; r.softmax_scale = p->softmax_scale;
    return r;
}

int check_paged_layout(const kivi_paged_layout_t* l) {
    if (!l || l->max_sequences < 1 || l->n_q_heads < 1 || l->n_kv_heads < 1 || l->n_q_heads % l->n_kv_heads != 0) return KIVI_ERR_INVALID_ARG;
    if (l->residual < 0 || l->n_pages < 1 || l->cap_r_tokens < 0) return KIVI_ERR_INVALID_ARG;
    if (l->head_dim != kHeadDim || (l->bits != 2 && l->bits != 4) || l->group != kTileTokens) return KIVI_ERR_UNSUPPORTED;
    if (l->residual % kTileTokens != 0 || l->cap_r_tokens % kTileTokens != 0 || l->cap_r_tokens < (int64_t)l->residual + kTileTokens) return KIVI_ERR_INVALID_ARG;
    if (l->page_tokens < kTileTokens || l->page_tokens > 4096 || (l->page_tokens & (l->page_tokens - 1))) return KIVI_ERR_INVALID_ARG;
    if (l->n_q_heads / l->n_kv_heads > kMaxRepTotal || l->cap_r_tokens > 1 << 20) return KIVI_ERR_UNSUPPORTED;
    if (!fits(kMaxBytes, {l->n_pages, l->n_kv_heads, l->page_tokens / kTileTokens, record_bytes(l->bits)}) ||
        !fits(kMaxBytes, {l->max_sequences, l->n_kv_heads, l->cap_r_tokens, kHeadDim * 2}))
        return KIVI_ERR_UNSUPPORTED;
    return KIVI_OK;
}
int check_paged(const kivi_paged_layout_t* l, const kivi_paged_cache_t* c, const kivi_paged_batch_t* b) {
    if (const int st = check_paged_layout(l)) return st;
    if (!c || !b || !c->pages || !c->k_resid || !c->v_resid || !aligned16(c->pages) || !aligned16(c->k_resid) || !aligned16(c->v_resid)) return KIVI_ERR_INVALID_ARG;
    if (b->batch < 1 || b->max_pages < 0 || b->page_table_stride < b->max_pages || !b->lengths) return KIVI_ERR_INVALID_ARG;
    if ((b->max_pages > 0 && !b->page_table) || !aligned4(b->page_table) || !aligned4(b->lengths) || !aligned4(b->slots)) return KIVI_ERR_INVALID_ARG;
    if ((int64_t)b->max_pages * l->page_tokens > 0x7fffffff) return KIVI_ERR_INVALID_ARG;
    if (!fits(0x7fffffff, {b->batch, l->n_q_heads})) return KIVI_ERR_UNSUPPORTED;
    return KIVI_OK;
}
void paged_params(const kivi_paged_layout_t* l, const kivi_paged_cache_t* c, const kivi_paged_batch_t* b, PagedParams& p) {
    p.pages = static_cast<char*>(c->pages);
    p.k_resid = static_cast<__half*>(c->k_resid);
    p.v_resid = static_cast<__half*>(c->v_resid);
    p.page_table = b->page_table; p.lengths = b->lengths; p.slots = b->slots;
    p.page_table_stride = b->page_table_stride;
    p.batch = b->batch; p.max_pages = b->max_pages; p.n_pages = l->n_pages; p.max_sequences = l->max_sequences;
    p.n_q_heads = l->n_q_heads; p.n_kv_heads = l->n_kv_heads; p.bits = l->bits; p.residual = l->residual; p.cap_r = l->cap_r_tokens;
    p.page_shift = __builtin_ctz((unsigned)l->page_tokens / kTileTokens);
}

}  // namespace

extern "C" {

int kivi_norm_rotate(const kivi_norm_rotate_job_t* jobs, int32_t n_jobs, int32_t n_rows, float eps, const kivi_rotation_t* rotation, void* stream) {
    if (!jobs || n_jobs < 1 || n_jobs > 2 || n_rows < 0 || !std::isfinite(eps) || eps < 0.f) return KIVI_ERR_INVALID_ARG;
    if (n_rows == 0) return KIVI_OK;                   // (tensors without rows may be null)
    if (const int st = check_rotation(rotation, true)) return st;
    NormRotateParams p{};
    int64_t heads = 0;
    for (int i = 0; i < n_jobs; ++i) {
        const kivi_norm_rotate_job_t& j = jobs[i];
        if (j.n_heads < 1 || !aligned16(j.weight) || !std::isfinite(j.weight_offset)) return KIVI_ERR_INVALID_ARG;
        if (const int st = check_read(j.src)) return st;
        if (const int st = check_written(j.dst, 1, j.n_heads, n_rows)) return st;
        if (!known_type(j.src_type) || !known_type(j.dst_type)) return KIVI_ERR_UNSUPPORTED;
        p.job[i] = NormRotateParams::Job{tensor_params(j.src), tensor_params(j.dst), static_cast<const __half*>(j.weight), j.weight_offset,
                                         j.src_type == KIVI_TYPE_BF16, j.dst_type == KIVI_TYPE_BF16};
        heads += j.n_heads;
    }
    if (heads > 65536) return KIVI_ERR_INVALID_ARG;
    p.heads0 = jobs[0].n_heads;
    p.heads = (int32_t)heads;
    p.n_rows = n_rows;
    p.eps = eps;
    p.rotation = rotation_params(rotation);
    return hip_status(launch_norm_rotate(p, static_cast<hipStream_t>(stream)));
}

int kivi_prompt_workspace_bytes(const kivi_prompt_t* prompt, size_t* bytes) {
    if (!bytes) return KIVI_ERR_INVALID_ARG;
    if (const int st = check_prompt(prompt)) return st;
    *bytes = prompt_workspace_bytes(prompt_params(prompt));
    return KIVI_OK;
}

int kivi_prompt_attention(const kivi_prompt_t* prompt, const kivi_tensor_t* q, const kivi_tensor_t* k, const kivi_tensor_t* v, const kivi_tensor_t* out,
                          void* workspace, size_t workspace_bytes, void* stream) {
    if (const int st = check_prompt(prompt)) return st;
    if (!q || !k || !v || !out || !aligned16(workspace)) return KIVI_ERR_INVALID_ARG;
    if (prompt->max_q == 0 || (prompt->q_starts && prompt->q_rows == 0)) return KIVI_OK;
    const bool no_keys = prompt->max_k == 0 || (prompt->k_starts && prompt->k_rows == 0);      // (then the tensors may be null)
    for (const kivi_tensor_t* t : {q, k, v})
        if (t == q || t->data || !no_keys)
            if (const int st = check_read(*t)) return st;
    if (const int st = check_written(*out, prompt->q_starts ? 1 : prompt->batch, prompt->n_q_heads, prompt->q_starts ? prompt->q_rows : prompt->max_q)) return st;
    PromptParams p = prompt_params(prompt);
    p.q = tensor_params(*q); p.k = tensor_params(*k); p.v = tensor_params(*v); p.out = tensor_params(*out);
    if (workspace && workspace_bytes < prompt_workspace_bytes(p)) return KIVI_ERR_WORKSPACE;
    return hip_status(launch_prompt_attention(p, workspace, workspace ? workspace_bytes : 0, static_cast<hipStream_t>(stream)));
}

int kivi_paged_sizes(const kivi_paged_layout_t* layout, kivi_paged_sizes_t* sizes) {
    if (!sizes) return KIVI_ERR_INVALID_ARG;
    if (const int st = check_paged_layout(layout)) return st;
    sizes->pages = (size_t)layout->n_pages * layout->n_kv_heads * (layout->page_tokens / kTileTokens) * record_bytes(layout->bits);
    sizes->k_resid = sizes->v_resid = (size_t)layout->max_sequences * layout->n_kv_heads * layout->cap_r_tokens * kHeadDim * 2;
    sizes->workspace = paged_workspace_bytes();
    return KIVI_OK;
}

int kivi_paged_append(const kivi_paged_layout_t* layout, const kivi_paged_cache_t* cache, const kivi_paged_batch_t* batch, const kivi_paged_rows_t* rows, void* stream) {
    if (const int st = check_paged(layout, cache, batch)) return st;
    if (!rows || rows->max_new < 0 || rows->n_rows < 0 || !aligned4(rows->starts)) return KIVI_ERR_INVALID_ARG;
    if (!rows->starts && (int64_t)batch->batch * rows->max_new > rows->n_rows) return KIVI_ERR_INVALID_ARG;
    if (rows->max_new == 0 || rows->n_rows == 0) return KIVI_OK;
    if (const int st = check_read(rows->k)) return st;
    if (const int st = check_read(rows->v)) return st;
    if ((rows->q.data == nullptr) != (rows->q_out.data == nullptr)) return KIVI_ERR_INVALID_ARG;
    if (rows->q.data) {
        if (const int st = check_read(rows->q)) return st;
        if (const int st = check_written(rows->q_out, 1, layout->n_q_heads, rows->n_rows)) return st;
    }
    if (!known_type(rows->type)) return KIVI_ERR_UNSUPPORTED;
    if (const int st = check_rotation(rows->rotation, false)) return st;
    PagedAppendParams p{};
    paged_params(layout, cache, batch, p);
    p.k = tensor_params(rows->k); p.v = tensor_params(rows->v);
    p.q = tensor_params(rows->q); p.q_out = tensor_params(rows->q_out);
    p.starts = rows->starts;
    p.n_rows = rows->n_rows;
    p.max_new = rows->max_new;
    p.bf16 = rows->type == KIVI_TYPE_BF16;
    p.rotates = rows->rotation != nullptr;
    p.rotation = rotation_params(rows->rotation);
    return hip_status(launch_paged_append(p, static_cast<hipStream_t>(stream)));
}

int kivi_paged_attention(const kivi_paged_layout_t* layout, const kivi_paged_cache_t* cache, const kivi_paged_batch_t* batch, const kivi_paged_query_t* query,
                         void* workspace, size_t workspace_bytes, void* stream) {
    if (const int st = check_paged(layout, cache, batch)) return st;
    if (!query || !query->q || !query->out || !aligned16(query->q) || !aligned16(query->out)) return KIVI_ERR_INVALID_ARG;
    if (query->window < 0 || query->sinks < 0 || !std::isfinite(query->softmax_scale)) return KIVI_ERR_INVALID_ARG;
    if (!known_type(query->out_type)) return KIVI_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < paged_workspace_bytes()) return KIVI_ERR_WORKSPACE;
    PagedAttentionParams p{};
    paged_params(layout, cache, batch, p);
    p.q = static_cast<const __half*>(query->q);
    p.out = query->out;
    p.out_bf16 = query->out_type == KIVI_TYPE_BF16;
    p.window = query->window;
    p.sinks = query->sinks;
    p.softmax_scale = query->softmax_scale;
    p.counters = static_cast<int32_t*>(workspace);
    return hip_status(launch_paged_attention(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
