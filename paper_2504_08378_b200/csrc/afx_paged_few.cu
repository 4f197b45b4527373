// Launcher of the attention of few new tokens over the paged cache (afx_paged_few.cuh).
#include "afx_launch.cuh"
#include "afx_paged_few.cuh"

namespace afx {

template <int D, int CT, bool PACK, bool QF32>
static afx_status launch_few(const PagedFewArgs& f, int max_items, cudaStream_t st) {
    const auto kern = paged_few_kernel<D, CT, PACK, QF32>;
    constexpr size_t dyn = FewCfg<D>::kDyn;
    if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), dyn)) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const int blocks = 2 * sms < kFewMaxBlocks ? 2 * sms : kFewMaxBlocks;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = dyn;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, f);
    if (e == cudaSuccess) {
        cfg.gridDim = dim3(f.a.w.n_seqs * max_items);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, paged_join_kernel<D>, f, blocks, max_items);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

template <int D, int CT>
static afx_status launch_few_dt(const PagedFewArgs& f, int max_items, bool pack, cudaStream_t st) {
    const bool f32 = f.a.q_type == AFX_F32;
    if (pack) return f32 ? launch_few<D, CT, true, true>(f, max_items, st) : launch_few<D, CT, true, false>(f, max_items, st);
    return f32 ? launch_few<D, CT, false, true>(f, max_items, st) : launch_few<D, CT, false, false>(f, max_items, st);
}

afx_status launch_paged_few(int dtype, int D, PagedFewArgs& f, cudaStream_t st) {
    const bool pack = few_packed(f.a.w.max_new, f.a.rep);
    f.rows_per_group = pack ? 8 : kFewRows;
    const int64_t items = static_cast<int64_t>(f.a.w.n_kv) * ((static_cast<int64_t>(f.a.w.max_new) * f.a.rep + f.rows_per_group - 1) / f.rows_per_group);
    if (items * f.a.w.n_seqs > 0x7FFFFFFF) return AFX_ERR_CAPACITY;
    const int n = static_cast<int>(items);
    if (D == 128) return dtype == AFX_F16 ? launch_few_dt<128, AFX_F16>(f, n, pack, st) : launch_few_dt<128, AFX_BF16>(f, n, pack, st);
    return dtype == AFX_F16 ? launch_few_dt<64, AFX_F16>(f, n, pack, st) : launch_few_dt<64, AFX_BF16>(f, n, pack, st);
}

}  // namespace afx
