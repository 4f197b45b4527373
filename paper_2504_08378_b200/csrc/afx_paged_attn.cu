// afx_paged_attn: checks and the choice of the kernel.
#include "afx_paged_few.cuh"

namespace afx {

// One warp per (token row, query head), positions one after the other.
template <int D, int CT>
__global__ void __launch_bounds__(128) paged_rows_kernel(PagedAttnArgs a) {
    constexpr int E = D / 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int b = blockIdx.z, lane = lane_id();
    const int h = blockIdx.x * 4 + warp_id();
    const SeqSpan s = paged_span(a.w, b, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0);
    if (h >= a.heads) return;
    for (int i = blockIdx.y; i < s.n; i += gridDim.y) {
        const int p = s.first + i, t = s.row0 + i, g = h / a.rep;
        float q[E];
        for (int e = 0; e < E; ++e)
            q[e] = a.scale * typed_value(a.q, a.q_type, t * a.ldq + static_cast<int64_t>(h) * D + lane * E + e);
        RowState<D> st;
        for (int e = 0; e < E; ++e) st.acc[e] = 0.0f;
        if (p >= 0) {
            const int low = paged_low(a.mask, p);
            attend_row<D, CT>(a.w, b, g, q, 0, paged_few(a.mask, low), st);
            attend_row<D, CT>(a.w, b, g, q, low, p + 1, st);
        }
        const int64_t at = static_cast<int64_t>(t) * a.heads + h;
        for (int e = 0; e < E; ++e)
            a.out[at * D + lane * E + e] = typed_bits(st.l == 0.0f ? 0.0f : st.acc[e] / st.l, a.out_type);
        if (a.lse != nullptr && lane == 0) a.lse[at] = st.l == 0.0f ? -INFINITY : (st.m + log2f(st.l)) * kLn2;
    }
}

template <int D, int CT>
static afx_status launch_rows(const PagedAttnArgs& a, cudaStream_t st) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((a.heads + 3) / 4, a.w.max_new < 65535 ? a.w.max_new : 65535, a.w.n_seqs);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, paged_rows_kernel<D, CT>, a) != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

static afx_status attn_args(const afx_paged_kv* kv, int n_heads, int32_t* dev_status, PagedAttnArgs* a) {
    const afx_status rc = paged_view(kv, dev_status, &a->w);
    if (rc != AFX_OK) return rc;
    if (n_heads < 1 || n_heads % kv->n_kv_heads != 0) return AFX_ERR_INVALID_ARG;
    if (n_heads > 8192) return AFX_ERR_CAPACITY;
    a->heads = n_heads;
    a->rep = n_heads / kv->n_kv_heads;
    return AFX_OK;
}

}  // namespace afx

extern "C" size_t afx_paged_attn_workspace_bytes(const afx_paged_kv* kv, int n_heads) {
    afx::PagedAttnArgs a = {};
    if (afx::attn_args(kv, n_heads, nullptr, &a) != AFX_OK) return 0;
    if (kv->max_new > AFX_MAX_T) return 0;
    return (afx::few_workspace_bytes(kv->head_dim) + 255) / 256 * 256;
}

extern "C" afx_status afx_paged_attn(const afx_paged_kv* kv, const void* q, int q_dtype, int64_t ldq, int n_heads,
                                     float scale, int window, int sinks, void* out, int out_dtype, float* lse,
                                     void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    using namespace afx;
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
    a.mask.window = window;
    a.mask.sinks = sinks;
    a.q = static_cast<const char*>(q);
    a.ldq = ldq;
    a.q_type = q_dtype;
    a.scale = (scale == 0.0f ? 1.0f / sqrtf(static_cast<float>(D)) : scale) * 1.4426950408889634f;
    a.out = static_cast<uint16_t*>(out);
    a.out_type = out_dtype;
    a.lse = lse;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (kv->max_new <= AFX_MAX_T) {
        PagedFewArgs f = {};
        f.a = a;
        f.joins = static_cast<FewJoin*>(workspace);
        f.slots = reinterpret_cast<float*>(static_cast<char*>(workspace) + few_slots_at());
        return launch_paged_few(kv->dtype, D, f, st);
    }
    if (D == 128)
        return kv->dtype == AFX_F16 ? launch_rows<128, AFX_F16>(a, st) : launch_rows<128, AFX_BF16>(a, st);
    return kv->dtype == AFX_F16 ? launch_rows<64, AFX_F16>(a, st) : launch_rows<64, AFX_BF16>(a, st);
}
