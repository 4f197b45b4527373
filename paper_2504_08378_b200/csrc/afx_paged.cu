// afx_paged_append (norm of each head, rotation, rows into the pages) and the checks of the paged cache's descriptor.
#include "afx_paged.cuh"

namespace afx {

afx_status paged_view(const afx_paged_kv* kv, int32_t* dev_status, PagedView* out) {
    if (kv == nullptr) return AFX_ERR_INVALID_ARG;
    const afx_paged_kv& d = *kv;
    if (d.dtype != AFX_F16 && d.dtype != AFX_BF16) return AFX_ERR_UNSUPPORTED;
    if (d.head_dim != 64 && d.head_dim != 128) return AFX_ERR_UNSUPPORTED;
    if (d.n_kv_heads < 1 || d.page_size < 1 || d.n_pages < 1 || d.n_seqs < 0 || d.n_tokens < 0 || d.max_new < 1 ||
        d.table_stride < 1)
        return AFX_ERR_INVALID_ARG;
    if (d.n_kv_heads > 1024 || d.page_size > (1 << 20) || d.n_seqs > 65535 || d.n_tokens > (1 << 24)) return AFX_ERR_CAPACITY;
    if (d.k_pages == nullptr || d.v_pages == nullptr || d.page_table == nullptr || d.seq_len == nullptr) return AFX_ERR_INVALID_ARG;
    if (d.tok_start == nullptr && (d.max_new != 1 || d.n_tokens < d.n_seqs)) return AFX_ERR_INVALID_ARG;
    if (d.page_stride < d.head_dim || d.pos_stride < d.head_dim || d.head_stride < d.head_dim) return AFX_ERR_INVALID_ARG;
    if (((d.page_stride | d.pos_stride | d.head_stride) & 7) != 0 || !aligned16(d.k_pages) || !aligned16(d.v_pages) ||
        (reinterpret_cast<uintptr_t>(d.page_table) & 3u) != 0 || (reinterpret_cast<uintptr_t>(d.seq_len) & 3u) != 0 ||
        (reinterpret_cast<uintptr_t>(d.tok_start) & 3u) != 0 || (reinterpret_cast<uintptr_t>(dev_status) & 3u) != 0)
        return AFX_ERR_ALIGNMENT;
    PagedView w = {};
    w.k = static_cast<uint16_t*>(d.k_pages);
    w.v = static_cast<uint16_t*>(d.v_pages);
    w.table = d.page_table;
    w.len = d.seq_len;
    w.start = d.tok_start;
    w.status = dev_status;
    w.page_stride = d.page_stride;
    w.pos_stride = d.pos_stride;
    w.head_stride = d.head_stride;
    w.table_stride = d.table_stride;
    w.n_kv = d.n_kv_heads;
    w.n_pages = d.n_pages;
    w.n_seqs = d.n_seqs;
    w.n_tokens = d.n_tokens;
    w.max_new = d.max_new;
    w.page_size = d.page_size;
    const int64_t limit = (int64_t{1} << 30);  // positions of a sequence: sums of two stay inside 32 bits
    w.cap = static_cast<int>(d.table_stride >= limit / d.page_size ? limit : d.table_stride * d.page_size);
    if (d.table_stride >= limit / d.page_size) w.cap = static_cast<int>(limit / d.page_size * d.page_size);
    // Division by an invariant d for 31-bit numerators: with l = ceil(log2 d), mul = ceil(2^(31+l) / d) < 2^32 exceeds
    // 2^(31+l) / d by less than 2^l / d, so that p * mul / 2^(31+l) exceeds p / d by less than 1 / d.
    int l = 0;
    while ((1 << l) < d.page_size) ++l;
    w.shift = l;
    w.mul = static_cast<uint32_t>(((uint64_t{1} << (31 + l)) + d.page_size - 1) / d.page_size);
    *out = w;
    return AFX_OK;
}

// -------------------------------------------------------------------------------- afx_paged_append

struct AppendArgs {
    PagedView w;
    const char *q, *k, *v;        // x_dtype rows; q may be NULL
    int64_t ldq, ldk, ldv;        // in values
    char* q_out;
    int q_type, cache_type, heads;
    float eps;
    int style, half;              // half = rotary_dim / 2 (0: no rotation)
    int rope_len;
    const float *g_q, *g_k, *cos, *sin;
    int passes;                   // passes over rows that a block makes
};

constexpr int kAppendThreads = 256;

template <int XT>
struct Piece {  // eight values of a row as they lie in memory
    uint4 raw[XT == AFX_F32 ? 2 : 1];
};
template <int XT>
__device__ __forceinline__ void load_piece(Piece<XT>& p, const char* row, int piece) {
    const uint4* at = reinterpret_cast<const uint4*>(row) + piece * (XT == AFX_F32 ? 2 : 1);
    p.raw[0] = at[0];
    if constexpr (XT == AFX_F32) p.raw[1] = at[1];
}
template <int XT>
__device__ __forceinline__ void piece_values(const Piece<XT>& p, float (&x)[8]) {
    if constexpr (XT == AFX_F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(p.raw[i].x);
            x[4 * i + 1] = __uint_as_float(p.raw[i].y);
            x[4 * i + 2] = __uint_as_float(p.raw[i].z);
            x[4 * i + 3] = __uint_as_float(p.raw[i].w);
        }
    } else {
        f32x2 pr[4];
        unpack8_pairs<XT>(p.raw[0], pr);
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_f32x2(pr[i], x[2 * i], x[2 * i + 1]);
    }
}
__device__ __forceinline__ void store_piece(char* row, int type, int piece, const float (&x)[8]) {
    if (type == AFX_F32) {
        float4* at = reinterpret_cast<float4*>(row) + 2 * piece;
        at[0] = make_float4(x[0], x[1], x[2], x[3]);
        at[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else if (type == AFX_F16) {
        reinterpret_cast<uint4*>(row)[piece] = make_uint4(pack2_bits<AFX_F16>(x[0], x[1]), pack2_bits<AFX_F16>(x[2], x[3]),
                                                          pack2_bits<AFX_F16>(x[4], x[5]), pack2_bits<AFX_F16>(x[6], x[7]));
    } else {
        reinterpret_cast<uint4*>(row)[piece] = make_uint4(pack2_bits<AFX_BF16>(x[0], x[1]), pack2_bits<AFX_BF16>(x[2], x[3]),
                                                          pack2_bits<AFX_BF16>(x[4], x[5]), pack2_bits<AFX_BF16>(x[6], x[7]));
    }
}

// grid (tokens, chunks of a token's q | k | v heads).  D / 16 lanes share a head's row; a lane owns two pieces of eight
// values that hold both members of its rotary pairs (halves: pieces l and l + half / 8; pairs: 2 l and 2 l + 1; what
// is not rotated in pairs of pieces behind), so that the rotation needs no exchange and its cosines are loaded once
// per token.  A row's norm is a sum over its lanes (shuffles).  Everything is held in fp32 and rounded once when it is stored.
template <int D, int XT>
__global__ void __launch_bounds__(kAppendThreads, 4) append_kernel(AppendArgs a) {
    constexpr int GL = D / 16, RPP = kAppendThreads / GL, XB = XT == AFX_F32 ? 4 : 2;
    __shared__ float4 rot[2][D / 8];  // of the token's position
    __shared__ int found[2][kAppendThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t = blockIdx.x, l = threadIdx.x % GL;
    const int kv = a.w.n_kv, nq = a.q != nullptr ? a.heads : 0, rows = nq + 2 * kv;
    const int r_end = min(rows, (static_cast<int>(blockIdx.y) + 1) * a.passes * RPP);
    int r = static_cast<int>(blockIdx.y) * a.passes * RPP + threadIdx.x / GL;
    int pa, pb;
    bool rotates = false;
    if (a.style == AFX_ROPE_HALVES) {
        const int h8 = a.half / 8;
        rotates = l < h8;
        pa = rotates ? l : 2 * l;
        pb = rotates ? l + h8 : 2 * l + 1;
    } else {
        rotates = l < a.half / 8;
        pa = 2 * l;
        pb = 2 * l + 1;
    }
    auto row_of = [&](int rr) {
        return rr < nq ? a.q + (t * a.ldq + static_cast<int64_t>(rr) * D) * XB
             : rr < nq + kv ? a.k + (t * a.ldk + static_cast<int64_t>(rr - nq) * D) * XB
                            : a.v + (t * a.ldv + static_cast<int64_t>(rr - nq - kv) * D) * XB;
    };
    // The first rows are on their way while the token's sequence is looked up; not those that no sequence has: they may not be there.
    const int n0 = a.w.start != nullptr ? a.w.start[0] : 0, n1 = a.w.start != nullptr ? a.w.start[a.w.n_seqs] : a.w.n_seqs;
    const bool early = t >= n0 && t < n1;
    Piece<XT> na, nb;
    auto first_rows = [&]() {
        if (r < r_end) {
            load_piece<XT>(na, row_of(r), pa);
            load_piece<XT>(nb, row_of(r), pb);
        }
    };
    if (early) first_rows();
    int b = t, row0 = t;
    if (a.w.start != nullptr) {  // the sequence in front of the first one that starts behind t
        const int n = a.w.n_seqs;
        int i = 0, upto = 0, lower = 0;  // of 256 starts: how many are at or before t, is one below the one before it
        for (; i <= n; i += kAppendThreads) {
            const int x = i + static_cast<int>(threadIdx.x), at = x <= n ? a.w.start[x] : 0x7FFFFFFF;
            const int before = x > 0 && x <= n ? a.w.start[x - 1] : at;
            const uint32_t in = __ballot_sync(0xFFFFFFFFu, x <= n && at <= t), down = __ballot_sync(0xFFFFFFFFu, at < before);
            int* mine = found[(i / kAppendThreads) & 1];
            if (lane_id() == 0) mine[warp_id()] = __popc(in) + (down != 0 ? 1 << 16 : 0);
            __syncthreads();
            upto = 0;
#pragma unroll
            for (int w = 0; w < kAppendThreads / 32; ++w) upto += mine[w];
            lower = upto >> 16;
            upto &= 0xFFFF;
            if (lower != 0 || upto < kAppendThreads) break;
        }
        if (i > n) return;  // behind the last sequence's rows
        if (lower == 0) {
            b = i + upto - 1;
            row0 = paged_first_row(a.w, max(b, 0));
        } else {
            row0 = 0;
            for (b = -1; b < n; ++b) {
                const int s = a.w.start[b + 1];
                if (s > t) break;
                row0 = max(row0, s);
            }
        }
    }
    if (b < 0 || b >= a.w.n_seqs) return;  // in front of the first sequence's rows or behind the last one's
    if (!early) first_rows();  // (starts that decrease)
    const bool lead = threadIdx.x == 0 && blockIdx.y == 0;
    const SeqSpan s = paged_span(a.w, b, row0, lead);
    const int i = t - s.row0;
    if (i >= s.n) return;  // (reported above)
    const int pos = s.first + i;
    if (pos < 0) return;  // (reported above)
    if (a.half > 0 && pos >= a.rope_len) {
        if (lead) report_status(a.w.status, AFX_ERR_CAPACITY);
        return;
    }
    int in_page;
    const int page = paged_page(a.w, b, pos, in_page);
    if (page < 0 && lead) report_status(a.w.status, AFX_ERR_INVALID_ARG);
    const int64_t cell = page * a.w.page_stride + in_page * a.w.pos_stride;
    // (in shared memory: 16 registers more would leave room for three blocks per SM instead of four)
    if (threadIdx.x < static_cast<unsigned>(a.half) / 2) {
        const int part = threadIdx.x & 1, at = threadIdx.x >> 1;  // cosines and sines, four at a time
        rot[part][at] = reinterpret_cast<const float4*>((part == 0 ? a.cos : a.sin) + static_cast<int64_t>(pos) * a.half)[at];
    }
    __syncthreads();
    for (; r - static_cast<int>(threadIdx.x) / GL < r_end; r += RPP) {  // (all lanes of a warp leave together)
        const bool live = r < r_end;
        const Piece<XT> ca = na, cb = nb;
        if (r + RPP < r_end) {
            load_piece<XT>(na, row_of(r + RPP), pa);
            load_piece<XT>(nb, row_of(r + RPP), pb);
        }
        const bool is_q = r < nq, is_v = r >= nq + kv;
        float x[8], y[8];
        if (live) {
            piece_values<XT>(ca, x);
            piece_values<XT>(cb, y);
        }
        const float* gain = is_q ? a.g_q : a.g_k;
        if (a.g_q != nullptr || a.g_k != nullptr) {
            float ss = 0.0f;
            if (live) {
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(x[j], x[j], fmaf(y[j], y[j], ss));
            }
#pragma unroll
            for (int o = GL / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            if (live && !is_v && gain != nullptr) {
                const float f = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 ga = reinterpret_cast<const float4*>(gain)[2 * pa + j];
                    const float4 gb = reinterpret_cast<const float4*>(gain)[2 * pb + j];
                    x[4 * j] *= f * ga.x; x[4 * j + 1] *= f * ga.y; x[4 * j + 2] *= f * ga.z; x[4 * j + 3] *= f * ga.w;
                    y[4 * j] *= f * gb.x; y[4 * j + 1] *= f * gb.y; y[4 * j + 2] *= f * gb.z; y[4 * j + 3] *= f * gb.w;
                }
            }
        }
        if (!live) continue;
        if (is_v) {
            if (page < 0) continue;
            uint16_t* row = a.w.v + cell + static_cast<int64_t>(r - nq - kv) * a.w.head_stride;
            if (XT == a.cache_type) {
                reinterpret_cast<uint4*>(row)[pa] = ca.raw[0];
                reinterpret_cast<uint4*>(row)[pb] = cb.raw[0];
            } else {
                store_piece(reinterpret_cast<char*>(row), a.cache_type, pa, x);
                store_piece(reinterpret_cast<char*>(row), a.cache_type, pb, y);
            }
            continue;
        }
        if (rotates) {
            float cs[8], sn[8];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 c = rot[0][2 * l + j], n = rot[1][2 * l + j];
                cs[4 * j] = c.x; cs[4 * j + 1] = c.y; cs[4 * j + 2] = c.z; cs[4 * j + 3] = c.w;
                sn[4 * j] = n.x; sn[4 * j + 1] = n.y; sn[4 * j + 2] = n.z; sn[4 * j + 3] = n.w;
            }
            if (a.style == AFX_ROPE_HALVES) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float u = x[j], v = y[j];
                    x[j] = u * cs[j] - v * sn[j];
                    y[j] = u * sn[j] + v * cs[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float u = x[2 * j], v = x[2 * j + 1];
                    x[2 * j] = u * cs[j] - v * sn[j];
                    x[2 * j + 1] = u * sn[j] + v * cs[j];
                    u = y[2 * j], v = y[2 * j + 1];
                    y[2 * j] = u * cs[4 + j] - v * sn[4 + j];
                    y[2 * j + 1] = u * sn[4 + j] + v * cs[4 + j];
                }
            }
        }
        if (is_q) {
            char* row = a.q_out + (static_cast<int64_t>(t) * a.heads + r) * D * (a.q_type == AFX_F32 ? 4 : 2);
            store_piece(row, a.q_type, pa, x);
            store_piece(row, a.q_type, pb, y);
        } else if (page >= 0) {
            char* row = reinterpret_cast<char*>(a.w.k + cell + static_cast<int64_t>(r - nq) * a.w.head_stride);
            store_piece(row, a.cache_type, pa, x);
            store_piece(row, a.cache_type, pb, y);
        }
    }
}

template <int D, int XT>
static afx_status launch_append(AppendArgs& a, cudaStream_t st) {
    constexpr int RPP = kAppendThreads / (D / 16);
    const int rows = (a.q != nullptr ? a.heads : 0) + 2 * a.w.n_kv, all = (rows + RPP - 1) / RPP;
    // a few tokens: as many blocks as there are passes; many: a block per token, which looks its sequence up once
    const int64_t per = static_cast<int64_t>(a.w.n_tokens) * all / (4 * (sm_count() > 0 ? sm_count() : 148));
    a.passes = per < 1 ? 1 : per > all ? all : static_cast<int>(per);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.w.n_tokens, (all + a.passes - 1) / a.passes);
    cfg.blockDim = dim3(kAppendThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, append_kernel<D, XT>, a) != cudaSuccess) {
        cudaGetLastError();
        return AFX_ERR_CUDA;
    }
    return AFX_OK;
}

}  // namespace afx

extern "C" afx_status afx_paged_append(const afx_paged_kv* kv, const afx_head_prep* prep, const void* q, int64_t ldq,
                                       const void* k, int64_t ldk, const void* v, int64_t ldv, void* q_out,
                                       int q_out_dtype, int32_t* dev_status, void* stream) {
    using namespace afx;
    AppendArgs a = {};
    const afx_status rc = paged_view(kv, dev_status, &a.w);
    if (rc != AFX_OK) return rc;
    if (prep == nullptr || k == nullptr || v == nullptr || (q == nullptr) != (q_out == nullptr)) return AFX_ERR_INVALID_ARG;
    const afx_head_prep& p = *prep;
    if (p.x_dtype != AFX_F16 && p.x_dtype != AFX_BF16 && p.x_dtype != AFX_F32) return AFX_ERR_UNSUPPORTED;
    if (q != nullptr && q_out_dtype != AFX_F16 && q_out_dtype != AFX_BF16 && q_out_dtype != AFX_F32) return AFX_ERR_UNSUPPORTED;
    if (p.rope_style != AFX_ROPE_NONE && p.rope_style != AFX_ROPE_PAIRS && p.rope_style != AFX_ROPE_HALVES) return AFX_ERR_UNSUPPORTED;
    const int D = kv->head_dim;
    if (!(p.eps >= 0.0f)) return AFX_ERR_INVALID_ARG;
    if (q != nullptr && (p.n_heads < 1 || p.n_heads % kv->n_kv_heads != 0)) return AFX_ERR_INVALID_ARG;
    if (q != nullptr && p.n_heads > 8192) return AFX_ERR_CAPACITY;
    if (ldk < static_cast<int64_t>(kv->n_kv_heads) * D || ldv < static_cast<int64_t>(kv->n_kv_heads) * D ||
        (q != nullptr && ldq < static_cast<int64_t>(p.n_heads) * D))
        return AFX_ERR_INVALID_ARG;
    if (p.rope_style != AFX_ROPE_NONE) {
        if (p.rotary_dim < 0 || p.rotary_dim > D ||
            (p.rotary_dim > 0 && (p.rope_len < 1 || p.rope_cos == nullptr || p.rope_sin == nullptr)))
            return AFX_ERR_INVALID_ARG;
        if ((p.rotary_dim & 15) != 0 || !aligned16(p.rope_cos) || !aligned16(p.rope_sin)) return AFX_ERR_ALIGNMENT;
    }
    if ((ldk & 7) != 0 || (ldv & 7) != 0 || (q != nullptr && (ldq & 7) != 0) || !aligned16(q) || !aligned16(k) || !aligned16(v) ||
        !aligned16(q_out) || !aligned16(p.g_q) || !aligned16(p.g_k))
        return AFX_ERR_ALIGNMENT;
    // a row of q_out written by one block must not be read by another: in place only row upon row
    if (q != nullptr && q == q_out && (p.x_dtype != q_out_dtype || ldq != static_cast<int64_t>(p.n_heads) * D)) return AFX_ERR_INVALID_ARG;
    if (a.w.n_seqs == 0 || a.w.n_tokens == 0) return AFX_OK;
    a.q = static_cast<const char*>(q);
    a.k = static_cast<const char*>(k);
    a.v = static_cast<const char*>(v);
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.q_out = static_cast<char*>(q_out);
    a.q_type = q_out_dtype;
    a.cache_type = kv->dtype;
    a.heads = p.n_heads;
    a.eps = p.eps;
    a.style = p.rope_style;
    a.half = p.rope_style == AFX_ROPE_NONE ? 0 : p.rotary_dim / 2;
    a.rope_len = p.rope_len;
    a.g_q = p.g_q;
    a.g_k = p.g_k;
    a.cos = p.rope_cos;
    a.sin = p.rope_sin;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (D == 128)
        return p.x_dtype == AFX_F32 ? launch_append<128, AFX_F32>(a, st)
             : p.x_dtype == AFX_F16 ? launch_append<128, AFX_F16>(a, st)
                                    : launch_append<128, AFX_BF16>(a, st);
    return p.x_dtype == AFX_F32 ? launch_append<64, AFX_F32>(a, st)
         : p.x_dtype == AFX_F16 ? launch_append<64, AFX_F16>(a, st)
                                : launch_append<64, AFX_BF16>(a, st);
}
