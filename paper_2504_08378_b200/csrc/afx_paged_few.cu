// Launcher of the attention of few new tokens over the paged cache (afx_paged_few.cuh).
#include "afx_launch.cuh"
#include "afx_paged_few.cuh"

namespace afx {

// One sequence: items side by side, as many blocks to an item as find a tile and are resident at once.  *taken: it is
// the faster way.  It saves the list and the joining launch (3 us: a sequence of 37 positions 5.9 and 7.9 us, 32 kv heads x 2049
// positions 12.3 and 14.4), but seldom fills the machine: clusters of 10 for 8 kv heads, 80 blocks, read 4.9 TB/s
// where the list reads 6.2 (131072 positions 110 and 93 us).  So it is taken where the blocks reach four fifths of
// the SMs, or where what the table (or the window) lets a sequence have is below the 64 MB at which the two meet.
template <int D, int CT, bool PACK, bool QF32>
static afx_status launch_one(const PagedFewArgs& f, int items, int sms, bool* taken, cudaStream_t st) {
    *taken = false;
    const auto kern = paged_few_kernel<D, CT, PACK, QF32, true>;
    const void* k = reinterpret_cast<const void*>(kern);
    constexpr size_t dyn = FewCfg<D>::kOneDyn;
    if (!ensure_dyn_smem(k, dyn)) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    int64_t longest = f.a.w.cap;
    if (f.a.mask.window > 0) {
        const int64_t seen = static_cast<int64_t>(f.a.mask.window) + f.a.mask.sinks + f.a.w.max_new;
        longest = seen < longest ? seen : longest;
    }
    const int tile = kOneWarps * kFewChunk;
    const int64_t most = (longest + tile - 1) / tile;
    int S = most < kOneCluster ? static_cast<int>(most) : kOneCluster;
    if (S > 8 && cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        S = 8;
    }
    while (S > 1 && max_active_clusters(k, S, dyn, kOneWarps * 32) < items) --S;
    if (5 * S * items < 4 * sms && longest * f.a.w.n_kv * D * 4 > (int64_t{64} << 20)) return AFX_OK;
    *taken = true;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(S, items);
    cfg.blockDim = dim3(kOneWarps * 32);
    cfg.dynamicSmemBytes = dyn;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kern, f) != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

template <int D, int CT, bool PACK, bool QF32>
static afx_status launch_few(const PagedFewArgs& f, cudaStream_t st) {
    const int new_tokens = f.a.w.max_new < f.most ? f.a.w.max_new : f.most;
    const int items = f.a.w.n_kv * ((new_tokens * f.a.rep + f.rows_per_group - 1) / f.rows_per_group);
    const int sms = sm_count() > 0 ? sm_count() : 148;
    if (f.a.w.n_seqs == 1 && items <= sms) {
        bool taken;
        const afx_status rc = launch_one<D, CT, PACK, QF32>(f, items, sms, &taken, st);
        if (rc != AFX_OK || taken) return rc;
    }
    const auto kern = paged_few_kernel<D, CT, PACK, QF32, false>;
    constexpr size_t dyn = FewCfg<D>::kDyn;
    if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), dyn)) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
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
    const int new_tokens = f.a.w.max_new < f.most ? f.a.w.max_new : f.most;
    const bool pack = few_packed(new_tokens, f.a.rep);
    f.rows_per_group = pack ? 8 : kFewRows;
    f.rep_mul = static_cast<uint32_t>((uint64_t{1} << 32) / f.a.rep) + 1u;
    if (D == 128) return dtype == AFX_F16 ? launch_few_dt<128, AFX_F16>(f, pack, st) : launch_few_dt<128, AFX_BF16>(f, pack, st);
    return dtype == AFX_F16 ? launch_few_dt<64, AFX_F16>(f, pack, st) : launch_few_dt<64, AFX_BF16>(f, pack, st);
}

}  // namespace afx
