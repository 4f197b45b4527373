// Launcher of the attention of few new tokens over the paged cache (afx_paged_few.cuh).
#include "afx_launch.cuh"
#include "afx_paged_few.cuh"

namespace afx {

template <int D, int CT, bool PACK, bool QF32>
static afx_status launch_few(const PagedFewArgs& f, cudaStream_t st) {
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
        cfg.gridDim = dim3(blocks, f.rows_per_group * D / (4 * kFewThreads));
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, paged_join_kernel<D>, f);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

template <int D, int CT>
static afx_status launch_few_dt(const PagedFewArgs& f, bool pack, cudaStream_t st) {
    const bool f32 = f.a.q_type == AFX_F32;
    if (pack) return f32 ? launch_few<D, CT, true, true>(f, st) : launch_few<D, CT, true, false>(f, st);
    return f32 ? launch_few<D, CT, false, true>(f, st) : launch_few<D, CT, false, false>(f, st);
}

afx_status launch_paged_few(int dtype, int D, PagedFewArgs& f, cudaStream_t st) {
    const bool pack = few_packed(f.a.w.max_new, f.a.rep);
    f.rows_per_group = pack ? 8 : kFewRows;
    f.rep_mul = static_cast<uint32_t>((uint64_t{1} << 32) / f.a.rep) + 1u;
    if (D == 128) return dtype == AFX_F16 ? launch_few_dt<128, AFX_F16>(f, pack, st) : launch_few_dt<128, AFX_BF16>(f, pack, st);
    return dtype == AFX_F16 ? launch_few_dt<64, AFX_F16>(f, pack, st) : launch_few_dt<64, AFX_BF16>(f, pack, st);
}

}  // namespace afx
