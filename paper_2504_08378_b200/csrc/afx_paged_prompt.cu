// Launcher of the attention of many new tokens over the paged cache (afx_paged_prompt.cuh).
#include "afx_launch.cuh"
#include "afx_paged_prompt.cuh"

namespace afx {

typedef CUresult (*TensorMapEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                    const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                    CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static TensorMapEncode tensor_map_encode() {
    static const TensorMapEncode fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<TensorMapEncode>(p);
    }();
    return fn;
}

// The pool as a tensor [page][kv head][position in the page][dim], read in boxes of `box` positions and 64 dims.
static bool pool_map(CUtensorMap* map, void* pages, int dtype, int D, const PagedView& w, int box) {
    const TensorMapEncode encode = tensor_map_encode();
    if (encode == nullptr) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(w.page_size), static_cast<cuuint64_t>(w.n_kv),
                                static_cast<cuuint64_t>(w.n_pages)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(w.pos_stride) * 2, static_cast<cuuint64_t>(w.head_stride) * 2,
                                   static_cast<cuuint64_t>(w.page_stride) * 2};
    const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(box), 1, 1}, steps[4] = {1, 1, 1, 1};
    return encode(map, dtype == AFX_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, pages, dims, strides, boxes,
                  steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int CT>
static afx_status launch_prompt(const PagedAttnArgs& a, int skip, cudaStream_t st) {
    const auto kern = paged_prompt_kernel<D, CT>;
    constexpr size_t dyn = PrCfg<D>::kDyn;
    if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), dyn)) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    // Both row tiles to a work, where that many works are more than half of the SMs: they share what is loaded, and one's weights
    // are made while the tensor cores work for the other.  Fewer: a row tile to a work, so that twice as many SMs
    // take part (100 new tokens of 32 / 8 heads: 12.8 and 11.4 us, 512 of 8 / 1 heads 13.8 and 12.3).  (Works: at most; the rows
    // of a sequence that takes part, of more than `skip` tokens, are rounded up.)
    const int most_seqs = a.w.n_tokens / (skip + 1), parts = most_seqs < a.w.n_seqs ? most_seqs : a.w.n_seqs;
    auto works = [&](int rows) { return (static_cast<int64_t>(a.w.n_tokens) * a.rep / rows + parts) * a.w.n_kv; };
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const int rows = 2 * works(kPrTiles * kPrRows) > sms ? kPrTiles * kPrRows : kPrRows;
    if (works(rows) > 0x7FFFFFFF) return AFX_ERR_CAPACITY;
    if (works(rows) == 0) return AFX_OK;  // (fewer tokens than a sequence that takes part has)
    PagedPromptArgs args = {a, 1, skip, rows};
    CUtensorMap maps[2] = {};
    // (with a window the positions begin on a box's border, and the first ones end on one: small boxes leave less to mask)
    const int most = a.mask.window > 0 ? 16 : kPrPos;
    int box = 1;
    while (box < most && a.w.page_size % (2 * box) == 0) box *= 2;
    // (what the encoder refuses -- strides of 2^40 bytes, no such entry point -- is read row by row)
    if (box >= 16 && pool_map(&maps[0], a.w.k, CT, D, a.w, box) && pool_map(&maps[1], a.w.v, CT, D, a.w, box)) args.box = box;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(works(rows)));
    cfg.blockDim = dim3(kPrThreads);
    cfg.dynamicSmemBytes = dyn;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, args, maps[0], maps[1]) != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

afx_status launch_paged_prompt(int dtype, int D, const PagedAttnArgs& a, int skip, cudaStream_t st) {
    if (D == 128) return dtype == AFX_F16 ? launch_prompt<128, AFX_F16>(a, skip, st) : launch_prompt<128, AFX_BF16>(a, skip, st);
    return dtype == AFX_F16 ? launch_prompt<64, AFX_F16>(a, skip, st) : launch_prompt<64, AFX_BF16>(a, skip, st);
}

}  // namespace afx
