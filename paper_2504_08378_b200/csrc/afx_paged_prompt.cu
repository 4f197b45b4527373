// Launcher of the attention of many new tokens over the paged cache (afx_paged_prompt.cuh).
#include "afx_launch.cuh"
#include "afx_paged_prompt.cuh"

namespace afx {

template <int D, int CT>
static afx_status launch_prompt(const PagedAttnArgs& a, cudaStream_t st) {
    const auto kern = paged_prompt_kernel<D, CT>;
    constexpr size_t dyn = PrCfg<D>::kDyn;
    if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), dyn)) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    // sums of rows rounded up to pairs of row tiles, at most
    const int64_t pairs = static_cast<int64_t>(a.w.n_tokens) * a.rep / (kPrTiles * kPrRows) + a.w.n_seqs;
    if (pairs * a.w.n_kv > 0x7FFFFFFF) return AFX_ERR_CAPACITY;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(pairs * a.w.n_kv));
    cfg.blockDim = dim3(kPrThreads);
    cfg.dynamicSmemBytes = dyn;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, a) != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

afx_status launch_paged_prompt(int dtype, int D, const PagedAttnArgs& a, cudaStream_t st) {
    if (D == 128) return dtype == AFX_F16 ? launch_prompt<128, AFX_F16>(a, st) : launch_prompt<128, AFX_BF16>(a, st);
    return dtype == AFX_F16 ? launch_prompt<64, AFX_F16>(a, st) : launch_prompt<64, AFX_BF16>(a, st);
}

}  // namespace afx
