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

__device__ __forceinline__ float typed_value(const char* p, int type, int64_t i) {
    if (type == AFX_F32) return reinterpret_cast<const float*>(p)[i];
    const uint16_t b = reinterpret_cast<const uint16_t*>(p)[i];
    return type == AFX_F16 ? bits_to_float<AFX_F16>(b) : bits_to_float<AFX_BF16>(b);
}
__device__ __forceinline__ uint16_t typed_bits(float v, int type) {
    return type == AFX_F16 ? float_to_bits<AFX_F16>(v) : float_to_bits<AFX_BF16>(v);
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

// Running softmax of one row in a warp: a lane owns D / 32 neighbouring dims.
template <int D>
struct RowState {
    float m = -INFINITY, l = 0.0f, acc[D / 32];
};

// Positions [from, to) of (sequence b, kv head g) added to the row with query q (times scale * log2 e), four on their way at
// once.  Nothing more is added once every sum is infinite or NaN: none becomes finite again.
template <int D, int CT>
__device__ __forceinline__ void attend_row(const PagedView& w, int b, int g, const float (&q)[D / 32], int from, int to,
                                           RowState<D>& s) {
    constexpr int E = D / 32, U = 4;
    const int lane = lane_id();
    for (int p0 = from; p0 < to; p0 += U) {
        uint32_t kr[U][E / 2], vr[U][E / 2];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = p0 + u < to ? paged_row(w, b, p0 + u, g) : -1;
            in[u] = at >= 0;
            if (at < 0 && p0 + u < to && lane == 0) report_status(w.status, AFX_ERR_INVALID_ARG);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                kr[u][i] = in[u] ? reinterpret_cast<const uint32_t*>(w.k + at)[lane * (E / 2) + i] : 0u;
                vr[u][i] = in[u] ? reinterpret_cast<const uint32_t*>(w.v + at)[lane * (E / 2) + i] : 0u;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            float d = 0.0f, v[E];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const float2 kk = pair_values<CT>(kr[u][i]), vv = pair_values<CT>(vr[u][i]);
                d = fmaf(q[2 * i], kk.x, d);
                d = fmaf(q[2 * i + 1], kk.y, d);
                v[2 * i] = vv.x;
                v[2 * i + 1] = vv.y;
            }
            d = warp_sum(d);
            const float mn = fmaxf(s.m, d);
            const float ref = mn == -INFINITY ? 0.0f : mn;
            const float f = fast_exp2(s.m - ref), pw = fast_exp2(d - ref);
            s.m = mn;
            s.l = fmaf(s.l, f, pw);
#pragma unroll
            for (int i = 0; i < E; ++i) s.acc[i] = fmaf(s.acc[i], f, pw * v[i]);
        }
        if (to - from > U) {
            bool some = false;
#pragma unroll
            for (int i = 0; i < E; ++i) some |= fabsf(s.acc[i]) <= 3.402823466e38f;
            if (!__any_sync(0xFFFFFFFFu, some)) return;
        }
    }
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
