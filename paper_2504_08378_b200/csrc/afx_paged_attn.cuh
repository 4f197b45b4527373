// Attention over the paged cache: arguments, and one token row on the fp32 pipe.
#pragma once

#include "afx_attn.cuh"
#include "afx_paged.cuh"

namespace afx {

struct PagedAttnArgs {
    PagedView w;
    PagedMask mask;
    const char* q;   // q_type rows of heads * D values
    int64_t ldq;     // in values
    int q_type;
    int heads, rep;  // rep = heads / n_kv
    float scale;     // of the scores, times log2(e)
    uint16_t* out;
    int out_type;
    float* lse;      // or NULL
};

// afx_paged_attn (afx_paged_attn.cu).  past_final: the kernel in front of it in the stream is the afx_paged_append of the same
// tokens, and was itself let in by a kernel that waits for all before it.  limit: tokens at positions from there on take no part (only
// where max_new <= AFX_MAX_T).
afx_status paged_attn(const afx_paged_kv* kv, const void* q, int q_dtype, int64_t ldq, int n_heads, float scale, int window,
                      int sinks, void* out, int out_dtype, float* lse, void* workspace, size_t workspace_bytes, int limit, bool past_final,
                      int32_t* dev_status, void* stream);

constexpr float kLn2 = 0.6931471805599453f;

template <int CT>
__device__ __forceinline__ float2 pair_values(uint32_t r) {
    if constexpr (CT == AFX_F16) return __half22float2(*reinterpret_cast<const __half2*>(&r));
    return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xFFFF0000u));
}

// The sign's places of the halves that are infinite or NaN.  (An exponent of ones carries there.)
template <int CT>
__device__ __forceinline__ uint32_t not_finite(uint32_t pair) {
    return ((pair & 0x7FFF7FFFu) + (CT == AFX_F16 ? 0x04000400u : 0x00800080u)) & 0x80008000u;
}
template <int CT>
__device__ __forceinline__ uint32_t not_finite(const uint4& x) {
    return not_finite<CT>(x.x) | not_finite<CT>(x.y) | not_finite<CT>(x.z) | not_finite<CT>(x.w);
}

// C += A B of 16 x 16 and 16 x 8 values, fp32 sums.
template <int CT>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (CT == AFX_F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of which a lane holds two neighbours of a row, the other way round.
__device__ __forceinline__ uint32_t transposed_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Whether one of the values at positions [from, to) of (sequence b, kv head g) is infinite or NaN; the same for the warp.
template <int D, int CT>
__device__ __forceinline__ bool any_value_not_finite(const PagedView& w, int b, int g, int from, int to) {
    constexpr int E = D / 32;
    uint32_t found = 0;
#pragma unroll 4
    for (int p = from; p < to; ++p) {
        const int64_t at = paged_row(w, b, p, g);
        if (at < 0) continue;
#pragma unroll
        for (int i = 0; i < E / 2; ++i)
            found |= not_finite<CT>(reinterpret_cast<const uint32_t*>(w.v + at)[lane_id() * (E / 2) + i]);
    }
    return __any_sync(0xFFFFFFFFu, found != 0u);
}

}  // namespace afx
