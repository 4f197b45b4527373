// afx_paged_attn: checks and the choice of the kernel.
#include "afx_paged_few.cuh"
#include "afx_paged_prompt.cuh"

namespace afx {

static afx_status attn_args(const afx_paged_kv* kv, int n_heads, int32_t* dev_status, PagedAttnArgs* a) {
    const afx_status rc = paged_view(kv, dev_status, &a->w);
    if (rc != AFX_OK) return rc;
    if (n_heads < 1 || n_heads % kv->n_kv_heads != 0) return AFX_ERR_INVALID_ARG;
    if (n_heads > 8192 || static_cast<int64_t>(kv->n_tokens) * n_heads > 0x7FFFFFFF) return AFX_ERR_CAPACITY;
    a->heads = n_heads;
    a->rep = n_heads / kv->n_kv_heads;
    return AFX_OK;
}

}  // namespace afx

extern "C" size_t afx_paged_attn_workspace_bytes(const afx_paged_kv* kv, int n_heads) {
    afx::PagedAttnArgs a = {};
    if (afx::attn_args(kv, n_heads, nullptr, &a) != AFX_OK) return 0;
    if (kv->n_seqs <= 1 && kv->max_new > afx::few_most_tokens(a.rep, afx::kFewMostGroups)) return 0;
    return (afx::few_workspace_bytes(kv->head_dim) + 255) / 256 * 256;
}

afx_status afx::paged_attn(const afx_paged_kv* kv, const void* q, int q_dtype, int64_t ldq, int n_heads, float scale, int window,
                           int sinks, void* out, int out_dtype, float* lse, void* workspace, size_t workspace_bytes,
                           int limit, bool past_final, int32_t* dev_status, void* stream) {
    PagedAttnArgs a = {};
    const afx_status rc = attn_args(kv, n_heads, dev_status, &a);
    if (rc != AFX_OK) return rc;
    const int D = kv->head_dim;
    if (q == nullptr || out == nullptr || ldq < static_cast<int64_t>(n_heads) * D || window < 0 || sinks < 0 || scale != scale)
        return AFX_ERR_INVALID_ARG;
    if (out_dtype != AFX_F16 && out_dtype != AFX_BF16) return AFX_ERR_UNSUPPORTED;
    if (q_dtype != kv->dtype && q_dtype != AFX_F32) return AFX_ERR_UNSUPPORTED;
    if (q_dtype == AFX_F32 && kv->max_new > AFX_MAX_T) return AFX_ERR_UNSUPPORTED;
    if ((ldq & 7) != 0 || !aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0 ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
        return AFX_ERR_ALIGNMENT;
    const size_t need = afx_paged_attn_workspace_bytes(kv, n_heads);
    if (need != 0 && workspace == nullptr) return AFX_ERR_INVALID_ARG;
    if (workspace_bytes < need) return AFX_ERR_CAPACITY;
    if (a.w.n_seqs == 0 || a.w.n_tokens == 0) return AFX_OK;
    // no position reaches 2^30: what is larger says the same, and differences of positions stay inside 32 bits
    a.mask.window = window < (1 << 30) ? window : 1 << 30;
    a.mask.sinks = sinks < (1 << 30) ? sinks : 1 << 30;
    a.q = static_cast<const char*>(q);
    a.ldq = ldq;
    a.q_type = q_dtype;
    a.scale = (scale == 0.0f ? 1.0f / sqrtf(static_cast<float>(D)) : scale) * 1.4426950408889634f;
    a.out = static_cast<uint16_t*>(out);
    a.out_type = out_dtype;
    a.lse = lse;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Sequences with few new tokens are split over their positions; the tiles of 128 rows are for those with more.  A batch may
    // have both (a few prompts' chunks beside sequences that decode): one kernel after the other, each leaving out what is the other's.
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const int64_t groups = sms / (static_cast<int64_t>(a.w.n_seqs) * a.w.n_kv);
    const int most = few_most_tokens(a.rep, static_cast<int>(groups < kFewMostGroups ? groups : kFewMostGroups));
    const bool prompts = kv->max_new > most;
    if (!prompts || kv->n_seqs > 1) {
        PagedFewArgs f = {};
        f.a = a;
        f.most = most;
        f.limit = limit;
        f.past_final = past_final && kv->n_seqs == 1;
        f.joins = static_cast<FewJoin*>(workspace);
        f.slots = reinterpret_cast<float*>(static_cast<char*>(workspace) + few_slots_at());
        const afx_status few = launch_paged_few(kv->dtype, D, f, st);
        if (few != AFX_OK || !prompts) return few;
    }
    return launch_paged_prompt(kv->dtype, D, a, kv->n_seqs > 1 ? most : 0, st);
}

extern "C" afx_status afx_paged_attn(const afx_paged_kv* kv, const void* q, int q_dtype, int64_t ldq, int n_heads,
                                     float scale, int window, int sinks, void* out, int out_dtype, float* lse,
                                     void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    return afx::paged_attn(kv, q, q_dtype, ldq, n_heads, scale, window, sinks, out, out_dtype, lse, workspace, workspace_bytes,
                           1 << 30, false, dev_status, stream);
}
