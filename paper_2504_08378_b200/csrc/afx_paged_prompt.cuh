// Attention of many new tokens per sequence (prompts, chunks of them) over the paged cache, on the 5th-generation
// tensor cores.
//
// A block takes two tiles of 128 rows of one (sequence, kv head) -- rows are (token, query head of the kv head), so that heads which share
// keys share their loads -- and walks the positions that their tokens see in tiles of 128.  Per tile of positions
// and of rows:
//   S = Q K^T    128 x 128 x D, both operands in shared memory, S in tensor memory
//   P = 2^(S scale - m)   a thread per row: S out of tensor memory, P (16 bits) back into S's place
//   O += P V     128 x D x 128, P from tensor memory, V from shared memory as it lies in the cache, O in tensor memory
// One thread issues the products, of the two row tiles in turn: while one tile's P is computed the tensor cores
// work for the other.  O is rescaled only when a row's maximum has grown by 2^8 since the last time (P stays
// below 2^8; fp16 P is carried times 2^7, so that what is lost below its range is 2^-32 of the largest weight).
// P is rounded to the cache's type (half a step of 2^-9 / 2^-12 relative per weight, averaged over the weights; the sums
// of weights are taken before that rounding): 16-bit operands are what the tensor cores multiply at full rate.
// A block stays: while the rows of a work leave, the loads and the first scores of the next one are under way.  It takes works over from
// blocks of the grid that have not begun (cluster launch control), longest first.
// Three warps fetch queries, keys and values.  Pages of a multiple of 16 positions are read in boxes of 16 to 128 positions (the
// largest power of two that divides the page size) with tensor copies; other pages, and the tile in which the sequence
// ends (what lies behind it in its page may be anything, and has to become zero), row by row with cp.async.  (Everything with
// cp.async: the tensor cores waited 1300 of 4000 cycles per step for the copies.)
//
// A step of both row tiles takes 3600 cycles at D = 128 (8192 new tokens of 64 / 8 heads: 1.07 ms, 1030 TFLOP/s, 74 % of cuBLAS in a
// loop under the power limit), where its 2 x 128 x 128 exponentials are 2048 cycles of the special-function units and
// its products 2048 cycles of the tensor cores: a row tile's chain (scores, weights, products) is what is long, and the
// two chains fill each other's gaps only in part.  Exponentials by polynomials on the fp32 pipe for an eighth or a quarter of
// the weights made every size slower (3 to 24 %), as did maxima in front of all weights (7 %).
#pragma once

#include "afx_paged_attn.cuh"
#include "afx_tcgen05.cuh"

namespace afx {

constexpr int kPrThreads = 384;  // warps 0-3: rows of tile 0, 4-7: tile 1, 8: products, 9-11: loads
constexpr int kPrRows = 128, kPrTiles = 2, kPrPos = 128;
constexpr int kPrLoaders = 3;
// Registers of a thread of the loading and issuing warps, and of the rows' warps: 128 and 256 threads share the 384 x 168 of the launch.
constexpr int kPrLoadRegs = 104, kPrRowRegs = 200;
static_assert(128 * kPrLoadRegs + 256 * kPrRowRegs <= kPrThreads * 168, "more than the launch has");
// Positions after which a warp that takes a row again says so (0.3 ms; a build for tests may say otherwise).
#ifndef AFX_TELL_EVERY
#define AFX_TELL_EVERY 1024
#endif
constexpr float kPrGrow = 8.0f;  // powers of two that a row's maximum may grow by before O is rescaled

struct PagedPromptArgs {
    PagedAttnArgs a;
    int box;   // positions of a tensor copy; 1: none are made
    int skip;  // sequences of up to that many new tokens are somebody else's
    int rows;  // of a work: both row tiles' 256, or 128 (the second tile has none)
};

afx_status launch_paged_prompt(int dtype, int D, const PagedAttnArgs& a, int skip, cudaStream_t st);  // afx_paged_prompt.cu

template <int D>
struct PrCfg {
    static constexpr int kRing = D == 128 ? 5 : 8;     // tiles of K and V on their way or in use, in the order of their use: K0, V0, K1, V1, ..
    static constexpr int kBlock = kPrPos * 128;        // bytes of 128 rows of 64 values
    static constexpr int kTile = kBlock * (D / 64);    // bytes of 128 rows of D values
    static constexpr int kQ = 0, kKV = kPrTiles * kTile;
    static constexpr int kDyn = kKV + kRing * kTile + 1024;  // (base rounded up to 1024)
};

struct PrBarriers {
    uint64_t q_full, q_empty, full[8], empty[8], s_full[2], p_half[2], p_full[2], o_full[2], work_full[2], work_empty[2], answered, drain;
};

// A work: what a block does at a time.
struct PrWork {
    int row0, first, end;      // the sequence's first token row and its position; the position behind its last one
    int b, kv_head;
    int row_base, rows;        // its rows of (token, query head of the kv head): row_base .. rows - 1
    int few, low;              // positions: [0, few), then low ..
    int tiles[2];              // tiles of positions that each row tile sees
    int boxed;                 // tiles of positions that are read in boxes: those in front of the one with the sequence's end
};

// Works of a sequence and kv head.
__device__ __forceinline__ int pr_works(const PagedPromptArgs& g, const SeqSpan& s) {
    return s.n > g.skip ? static_cast<int>((static_cast<int64_t>(s.n) * g.a.rep + g.rows - 1) / g.rows) : 0;
}
// A work is as long as what its last row sees; work i of a sequence: min(window and first positions, first + 1 +
// (rows (i + 1) - 1) / rep).  The largest of a sequence, and how many of its n works have at least `least`.
__device__ __forceinline__ int pr_seen_at_most(const PagedAttnArgs& a) {
    return a.mask.window > 0 ? min(a.mask.window, 1 << 29) + min(a.mask.sinks, 1 << 29) : 0x7FFFFFFF;
}
__device__ __forceinline__ int pr_most(const PagedPromptArgs& g, const SeqSpan& s, int n) {
    return n > 0 ? min(pr_seen_at_most(g.a), max(s.first + 1 + static_cast<int>((static_cast<int64_t>(n) * g.rows - 1) / g.a.rep), 1)) : 0;
}
__device__ __forceinline__ int pr_count(const PagedPromptArgs& g, const SeqSpan& s, int n, int least) {
    if (pr_seen_at_most(g.a) < least) return 0;
    const int64_t need = static_cast<int64_t>(least) - 1 - s.first;  // (rows (i + 1) - 1) / rep >= need
    const int64_t from = need <= 0 ? 0 : max((need * g.a.rep + g.rows) / g.rows - 1, int64_t{0});
    return static_cast<int>(max(n - from, int64_t{0}));
}
constexpr int kPrClasses = 4;  // works with more than 1/2, 1/4, 1/8 of the longest one's positions, and the others

// Bits 0 .. n - 1 of a word (n <= 0: none, n >= 32: all).
__device__ __forceinline__ uint32_t pr_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Two weights 2^(s scale + ref), added to the sums, rounded and packed.
template <int CT>
__device__ __forceinline__ uint32_t pr_weights(float s0, float s1, f32x2 scale, f32x2 ref, f32x2& sum) {
    float p0, p1;
    f32x2 t = ref;
    fma_f32x2(t, pack_f32x2(s0, s1), scale);
    unpack_f32x2(t, p0, p1);
    p0 = fast_exp2(p0);
    p1 = fast_exp2(p1);
    fma_f32x2(sum, pack_f32x2(p0, p1), pack_f32x2(1.0f, 1.0f));
    return pack2_bits<CT>(p0, p1);
}

// What a block's first search leaves for the others: the length of the longest work, the works of a kv head, and per lane which of
// its sequences have works (from .. to - 1, and perhaps some that have none between them) with the first token row of the first.
struct PrFound {
    int longest, total;
    int from[32], to[32], row0[32];
};
// Work `place` of the grid: (rows, kv head), kv heads side by side; the works in classes of falling length (a long one
// that begins last is what everybody waits for), in a class sequence by sequence.  One warp; what it finds goes to
// *out; false when there are not so many.  first_call: of the block's.
__device__ __forceinline__ bool pr_find(const PagedPromptArgs& args, int place, bool first_call, PrFound* found, PrWork* out) {
    const PagedAttnArgs& a = args.a;
    const int pair = place / a.w.n_kv, lane = lane_id();
    auto take = [&](const SeqSpan& s, int b, int i) {  // work i of sequence b
        PrWork w;
        w.row0 = s.row0;
        w.first = s.first;
        w.end = min(s.len, s.first + s.n);
        w.b = b;
        w.kv_head = place - pair * a.w.n_kv;
        w.row_base = i * args.rows;
        const int rows = w.rows = min(s.n * a.rep, w.row_base + args.rows);
        const int first = max(s.first + w.row_base / a.rep, 0);
        // (both on a box's border; places that no row sees are masked)
        w.low = paged_low(a.mask, first) & ~(args.box - 1);
        w.few = min((paged_few(a.mask, w.low) + args.box - 1) & ~(args.box - 1), w.low);
        for (int x = 0; x < kPrTiles; ++x) {
            const int r0 = w.row_base + x * kPrRows, r1 = min(r0 + kPrRows, rows) - 1;
            const int last = r0 < rows ? s.first + r1 / a.rep : -1;  // position of the tile's last row
            // (rows in front of the sequence see nothing of their one tile)
            w.tiles[x] = r0 >= rows ? 0 : last >= w.low ? (w.few + last + 1 - w.low + kPrPos - 1) / kPrPos : 1;
        }
        w.boxed = args.box == 1 || w.few + w.end < w.low ? 0 : (w.few + w.end - w.low) / kPrPos;
        *out = w;
    };
    const bool report = first_call && blockIdx.x == 0;
    if (a.w.n_seqs == 1) {
        const SeqSpan s = paged_span(a.w, 0, paged_first_row(a.w, 0), report && lane == 0);
        const int t = pr_works(args, s);
        if (lane == 0 && pair < t) take(s, 0, t - 1 - pair);
        return pair < t;
    }
    // (No loop over the sequences is unrolled: the whole kernel is 4 % faster with less code in it.)
    if (first_call) {
        const int n = a.w.n_seqs, per = (n + 31) / 32, i0 = lane * per, i1 = min(n, i0 + per);
        int top = 0;  // the largest start of the lane's sequences, then of the lanes' in front too
#pragma unroll 1
        for (int i = i0; i < i1; ++i) top = max(top, paged_first_row(a.w, i));
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, top, o);
            if (lane >= o) top = max(top, t);
        }
        top = __shfl_up_sync(0xFFFFFFFFu, top, 1);
        int at = i0 >= n ? 0 : lane > 0 ? max(top, paged_first_row(a.w, i0)) : paged_first_row(a.w, 0);
        int longest = 0, total = 0, from = i0, to = i0, row0 = 0;
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            const SeqSpan s = paged_span(a.w, i, at, report);
            const int t = pr_works(args, s);
            if (t > 0) {
                if (total == 0) {
                    from = i;
                    row0 = at;
                }
                to = i + 1;
                longest = max(longest, pr_most(args, s, t));
            }
            total += t;
            at = s.next;
        }
        found->from[lane] = from;
        found->to[lane] = to;
        found->row0[lane] = row0;
        longest = __reduce_max_sync(0xFFFFFFFFu, longest);
        total = __reduce_add_sync(0xFFFFFFFFu, total);
        if (lane == 0) {
            found->longest = longest;
            found->total = total;
        }
        __syncwarp();
    }
    if (pair >= found->total) return false;
    const int longest = found->longest, i0 = found->from[lane], i1 = found->to[lane], row0 = found->row0[lane];
    int before = 0;  // works of the classes in front
    for (int c = 0; c < kPrClasses; ++c) {
        const int most = (longest >> c) + 1, least = (longest >> (c + 1)) + 1;
        auto in_class = [&](const SeqSpan& s, int t, int& up) {
            up = c > 0 ? pr_count(args, s, t, most) : 0;
            return (c + 1 < kPrClasses ? pr_count(args, s, t, least) : t) - up;
        };
        int mine = 0, up;
#pragma unroll 1
        for (int i = i0, at = row0; i < i1; ++i) {
            const SeqSpan s = paged_span(a.w, i, at, false);
            at = s.next;
            mine += in_class(s, pr_works(args, s), up);
        }
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += t;
        }
        const int all = __shfl_sync(0xFFFFFFFFu, incl, 31);
        int nth = before + incl - mine;
        if (pair >= nth && pair < nth + mine) {
#pragma unroll 1
            for (int i = i0, at = row0; i < i1; ++i) {
                const SeqSpan s = paged_span(a.w, i, at, false);
                at = s.next;
                const int t = pr_works(args, s), k = in_class(s, t, up);
                if (pair - nth < k) {
                    take(s, i, t - 1 - (up + pair - nth));
                    break;
                }
                nth += k;
            }
        }
        before += all;
        if (pair < before) break;
    }
    return true;
}

// Rows 16 half .. + 15 of a warp, those of `left` among them, over what each sees alone: its lanes hold the rows' tokens, heads and
// positions.  Sixteen positions at a time, products of 16 x 8 x 16 straight from the cache; values that are not finite are added to the rows that see
// them and are zeros for the product.  (A warp's 32 rows over 40000 positions, D = 64: 8 ms; a row at a time they took 500.)  That may take long, and the
// block's other warps wait for it with the next work: they are told that it goes on.
template <int D, int CT>
__device__ __forceinline__ void pr_again(const PagedAttnArgs& a, const PrWork& w, int half, uint32_t left, int token, int head, int pos,
                                         Patience* patience) {
    constexpr int NK = D / 16, NT = D / 8;
    constexpr float kUpLog = CT == AFX_F16 ? 7.0f : 0.0f;
    const int lane = lane_id(), gid = lane >> 2, tig = lane & 3;
    uint32_t q[NK][4];
    float o[NT][4], m[2], l[2];
    int64_t at[2];  // the rows' places in out
    int p_row[2];
    bool mine[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = 16 * half + gid + 8 * e;
        const int t = w.row0 + __shfl_sync(0xFFFFFFFFu, token, r), hd = __shfl_sync(0xFFFFFFFFu, head, r);
        const int p = __shfl_sync(0xFFFFFFFFu, pos, r);
        mine[e] = (left >> r) & 1u;
        p_row[e] = mine[e] ? p : -1;
        at[e] = (static_cast<int64_t>(t) * a.heads + hd) * D;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint16_t*>(a.q) + t * a.ldq + static_cast<int64_t>(hd) * D);
#pragma unroll
        for (int i = 0; i < 2 * NK; ++i) q[i >> 1][2 * (i & 1) + e] = mine[e] ? src[4 * i + tig] : 0u;
        m[e] = -INFINITY;
        l[e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[i][x] = 0.0f;
    const int last = __reduce_max_sync(0xFFFFFFFFu, max(p_row[0], p_row[1]));
    const int first = __reduce_min_sync(0xFFFFFFFFu, min(p_row[0] < 0 ? last : p_row[0], p_row[1] < 0 ? last : p_row[1]));
    const int low = paged_low(a.mask, max(first, 0)), few = paged_few(a.mask, low), nv = last < 0 ? 0 : few + last + 1 - low;
#pragma unroll 1
    for (int v0 = 0; v0 < nv; v0 += 16) {
        if (v0 % AFX_TELL_EVERY == 0 && lane == 0) *const_cast<volatile uint32_t*>(&patience->told) = nanoseconds();
        if (v0 % 64 == 0) {  // once every sum is infinite or NaN nothing more is added: none becomes finite again
            bool some = false;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < NT; ++i) some |= mine[e] && (fabsf(o[i][2 * e]) <= 3.402823466e38f || fabsf(o[i][2 * e + 1]) <= 3.402823466e38f);
            if (!__any_sync(0xFFFFFFFFu, some)) break;
        }
        const int v = v0 + (lane & 15);
        const int64_t row = v < nv ? paged_row(a.w, w.b, v < few ? v : v - few + low, w.kv_head) : -1;
        const uint32_t there = __ballot_sync(0xFFFFFFFFu, row >= 0);
        uint32_t raw[2][NT];  // values of position 8 t + gid
        float c[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t from = __shfl_sync(0xFFFFFFFFu, row, 8 * t + gid);
            const uint32_t* k = reinterpret_cast<const uint32_t*>(a.w.k + (from < 0 ? 0 : from)) + tig;
            const uint32_t* vv = reinterpret_cast<const uint32_t*>(a.w.v + (from < 0 ? 0 : from)) + tig;
            uint32_t kb[2 * NK];
#pragma unroll
            for (int i = 0; i < 2 * NK; ++i) kb[i] = from < 0 ? 0u : k[4 * i];
#pragma unroll
            for (int i = 0; i < NT; ++i) raw[t][i] = from < 0 ? 0u : vv[4 * i];
#pragma unroll
            for (int x = 0; x < 4; ++x) c[t][x] = 0.0f;
#pragma unroll
            for (int j = 0; j < NK; ++j) mma_16816<CT>(c[t], q[j], kb[2 * j], kb[2 * j + 1]);
        }
        uint32_t pa[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float s[4], top = -INFINITY;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int j = 8 * (x >> 1) + 2 * tig + (x & 1), vj = v0 + j, p = vj < few ? vj : vj - few + low;
                const bool sees = ((there >> j) & 1u) && p <= p_row[e] && (a.mask.window == 0 || p > p_row[e] - a.mask.window || p < a.mask.sinks);
                s[x] = sees ? c[x >> 1][2 * e + (x & 1)] * a.scale : -INFINITY;
                top = fmaxf(top, s[x]);
            }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2)), m[e]);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float f = fast_exp2(m[e] - ref);  // 0 where nothing was seen before
            m[e] = top;
            l[e] *= f;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                o[i][2 * e] *= f;
                o[i][2 * e + 1] *= f;
            }
            float wt[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                wt[x] = fast_exp2(s[x] - ref + kUpLog);
                l[e] += wt[x];
            }
            pa[e] = pack2_bits<CT>(wt[0], wt[1]);
            pa[2 + e] = pack2_bits<CT>(wt[2], wt[3]);
        }
        uint32_t found = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < NT; ++i) found |= not_finite<CT>(raw[t][i]);
        if (__any_sync(0xFFFFFFFFu, found != 0u)) {
#pragma unroll 1
            for (int j = 0; j < 16; ++j) {
                const int vj = v0 + j, p = vj < few ? vj : vj - few + low;
                bool sees[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    sees[e] = ((there >> j) & 1u) && p <= p_row[e] && (a.mask.window == 0 || p > p_row[e] - a.mask.window || p < a.mask.sinks);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const float2 x = pair_values<CT>(__shfl_sync(0xFFFFFFFFu, j < 8 ? raw[0][i] : raw[1][i], 4 * (j & 7) + tig));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (sees[e] && !(fabsf(x.x) <= 3.402823466e38f)) o[i][2 * e] += x.x;
                        if (sees[e] && !(fabsf(x.y) <= 3.402823466e38f)) o[i][2 * e + 1] += x.y;
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < NT; ++i) raw[t][i] &= ~((not_finite<CT>(raw[t][i]) >> 15) * 0xFFFFu);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) mma_16816<CT>(o[i], pa, transposed_8x8(raw[0][i]), transposed_8x8(raw[1][i]));
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 1);
        l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 2);
        if (!mine[e]) continue;
        const float inv = l[e] == 0.0f ? 0.0f : 1.0f / l[e];
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + at[e]) + tig;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float x = l[e] == 0.0f ? 0.0f : o[i][2 * e] * inv, y = l[e] == 0.0f ? 0.0f : o[i][2 * e + 1] * inv;
            dst[4 * i] = a.out_type == AFX_F16 ? pack2_bits<AFX_F16>(x, y) : pack2_bits<AFX_BF16>(x, y);
        }
    }
}

template <int D, int CT>
__global__ void __launch_bounds__(kPrThreads, 1)
paged_prompt_kernel(const PagedPromptArgs args, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    const PagedAttnArgs& a = args.a;
    using Cfg = PrCfg<D>;
    constexpr int NB = Cfg::kRing;
    constexpr float kUpLog = CT == AFX_F16 ? 7.0f : 0.0f;
    extern __shared__ unsigned char dyn_raw[];
    __shared__ PrBarriers bar;
    __shared__ __align__(16) uint4 answer;  // of the request for the next block
    __shared__ uint32_t tmem_at;
    __shared__ Patience patience;
    __shared__ int steps[kPrLoaders];  // of the ring, that each of the loading warps has made in the end
    __shared__ PrWork work[2];
    __shared__ PrFound found;
    __shared__ __align__(16) uint16_t page_ok[8][8];  // per tile of positions (mod 8) and 16 of them: the cache has them
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* dyn = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t base = smem_u32(dyn);

    if (tid == 0) {
        patience.gave_up = 0;
        patience.told = nanoseconds();
        mbar_init(&bar.q_full, kPrLoaders * 32);
        mbar_init(&bar.q_empty, 1);
        for (int i = 0; i < NB; ++i) {
            mbar_init(&bar.full[i], kPrLoaders * 32);
            mbar_init(&bar.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.s_full[i], 1);
            mbar_init(&bar.p_half[i], 4);
            mbar_init(&bar.p_full[i], 4);
            mbar_init(&bar.o_full[i], 1);
            mbar_init(&bar.work_full[i], 1);
            mbar_init(&bar.work_empty[i], kPrThreads / 32);
        }
        mbar_init(&bar.answered, 1);
        mbar_init(&bar.drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(&tmem_at, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // A warp's next work (in its registers), the same for the whole warp; b < 0: there is none.  it counts the block's works.
    auto next_work = [&](int it, PrWork& w) {
        const bool in = __all_sync(0xFFFFFFFFu, mbar_wait(&bar.work_full[it & 1], (it >> 1) & 1, &patience));
        if (in) {
            w = work[it & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.work_empty[it & 1]);
        }
        return in;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPrLoadRegs));
        if (warp == 8) {
            // ---- products: the warp goes through the waits together and one lane issues, so that the operands'
            // places stay in uniform registers (all of it in a lane's branch: 64 products took 3800 cycles of the thread's time)
            constexpr uint32_t s_desc = mma_desc(CT == AFX_BF16, 128, kPrPos, false);
            constexpr uint32_t o_desc = mma_desc(CT == AFX_BF16, 128, D, true);
            const bool lead = elect_one();
            const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
            auto wait = [&](uint64_t* b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(b, parity, &patience)) != 0; };
            // The ring's tiles in the order of their use (K0, V0, K1, V1, ..).  The loaders' copies of rows are writes like any thread's,
            // the products read shared memory by another path: the fence stands between what the barrier says and them.
            int slot = 0;
            uint32_t turn = 0, q_turn = 0, p_turn[2] = {0, 0};
            auto arrived = [&](bool boxed) {
                const bool in = wait(&bar.full[slot], turn);
                if (!boxed) fence_proxy_async();
                return in;
            };
            auto step = [&]() {
                if (++slot == NB) {
                    slot = 0;
                    turn ^= 1u;
                }
            };
            auto scores = [&](int x, uint32_t k) {
                if (lead) {
                    const uint32_t qd = smem_desc(base + Cfg::kQ + x * Cfg::kTile, 16), kd = smem_desc(base + Cfg::kKV + k * Cfg::kTile, 16);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t off = ((i / 4) * Cfg::kBlock + (i % 4) * 32) >> 4;
                        tc_mma_ss(tm + x * kPrPos, qd + off, kd + off, s_desc, i > 0);
                    }
                    tc_commit(&bar.s_full[x]);
                }
                __syncwarp();
            };
            bool ok = true;
            for (int it = 0; ok; ++it) {
                PrWork w;
                ok = next_work(it, w);
                if (!ok || w.b < 0) break;
                const int tiles[2] = {__shfl_sync(0xFFFFFFFFu, w.tiles[0], 0), __shfl_sync(0xFFFFFFFFu, w.tiles[1], 0)};
                const int nt = max(tiles[0], tiles[1]);
                const int boxed = __shfl_sync(0xFFFFFFFFu, w.boxed, 0);
                ok = wait(&bar.q_full, q_turn) && arrived(false);
                q_turn ^= 1u;
                if (ok) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (tiles[x] > 0) scores(x, slot);
                    if (lead) {
                        tc_commit(&bar.empty[slot]);
                        if (nt == 1) tc_commit(&bar.q_empty);
                    }
                    __syncwarp();
                    step();
                }
                for (int j = 0; ok && j < nt; ++j) {
                    ok = arrived(j < boxed);
                    if (!ok) break;
                    const int vs = slot, last_x = j < tiles[1] ? 1 : 0;
                    step();
                    const int ks = slot;
                    // (Waited for here, while products are still being made: in front of the scores the wait is exposed, 930 -> 946 us;
                    // in front of the last scores of the step before, the copies are not there yet, 1010 us.)
                    if (j + 1 < nt) {
                        ok = arrived(j + 1 < boxed);
                        step();
                        if (!ok) break;
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!ok || j >= tiles[x]) continue;
                        const uint32_t vd = smem_desc(base + Cfg::kKV + vs * Cfg::kTile, Cfg::kBlock);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            ok = ok && wait(half == 0 ? &bar.p_half[x] : &bar.p_full[x], p_turn[x]);
                            tc_fence_after();
                            if (ok && lead) {
#pragma unroll
                                for (int i = half * (kPrPos / 32); i < (half + 1) * (kPrPos / 32); ++i)
                                    tc_mma_ts(tm + 256 + x * D, tm + x * kPrPos + i * 8, vd + i * (2048 >> 4), o_desc, j > 0 || i > 0);
                            }
                            __syncwarp();
                        }
                        p_turn[x] ^= 1u;
                        if (!ok) continue;
                        if (x == last_x && lead) tc_commit(&bar.empty[vs]);
                        if (j + 1 < tiles[x]) {
                            scores(x, ks);
                        } else {
                            if (lead) tc_commit(&bar.o_full[x]);
                            __syncwarp();
                        }
                    }
                    if (ok && lead) {
                        if (j + 1 < nt) tc_commit(&bar.empty[ks]);
                        if (j + 2 == nt) tc_commit(&bar.q_empty);  // the last scores of this work are issued
                    }
                    __syncwarp();
                }
            }
            if (!ok && lead) {  // what has been issued ends before tensor memory is given back
                report_status(a.w.status, AFX_ERR_TIMEOUT);
                tc_commit(&bar.drain);
                mbar_drain(&bar.drain, 0);
            }
            __syncwarp();
        } else {
            // ---- loads: blocks of 16 rows; a lane of the first 16 looks one row up, 16 (or 8) lanes copy a row
            constexpr int PIECES = D / 8, RPI = 32 / PIECES;
            const int lw = warp - 9;
            auto put = [&](uint32_t tile, int row, int piece, const void* src, int bytes) {
                const uint32_t at = tile + (piece >> 3) * Cfg::kBlock + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(src), "r"(bytes) : "memory");
            };
            auto when_landed = [&](uint64_t* full) {  // an arrival of this thread's as soon as its copies so far have landed
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(full)) : "memory");
            };
            auto wait = [&](uint64_t* b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(b, parity, &patience)) != 0; };
            const int boxes = kPrPos / args.box;
            // the ring's next slot: its tile before has been used (after the first turn)
            int slot = 0, ok_slot = 0;
            uint32_t turn = 0, q_turn = 0;
            bool q_used = false, ok = true;
            uint32_t asks = 0;  // for a place in the grid whose block has not begun
            bool open = false;  // the last one has no answer yet
            auto ask = [&]() {
                if (lane == 0) {
                    mbar_expect(&bar.answered, 16);
                    clc_ask(&answer, &bar.answered);
                }
                ++asks;
                open = true;
                __syncwarp();
            };
            auto answered = [&]() {  // the place; -1: none
                ok = wait(&bar.answered, (asks - 1) & 1);
                open = !ok;
                const int place = ok ? clc_place(&answer) : -1;
                fence_proxy_async();
                __syncwarp();
                return place;
            };
            auto room = [&]() { return turn == 0 || wait(&bar.empty[slot], (turn & 1u) ^ 1u); };
            auto step = [&]() {
                if (++slot == NB) {
                    slot = 0;
                    ++turn;
                }
            };
            // The third warp finds the block's works: the first by its place in the grid (turn -1, without loads), the others by taking over
            // places whose blocks have not begun (where that is refused they begin as blocks of their own).
            for (int it = lw == 2 ? -1 : 0; ok; ++it) {
                PrWork w = {};
                if (it >= 0) {
                    ok = next_work(it, w);
                    if (!ok || w.b < 0) break;
                    if (lw == 2) ask();
                }
                const int n_tiles = max(w.tiles[0], w.tiles[1]), rows = w.rows;
                const int end = w.end;
                int64_t off[3], next[3];
                auto look_up = [&](int j) {
#pragma unroll
                    for (int x = 0; x < 3; ++x) {
                        const int v = j * kPrPos + (lw + x * kPrLoaders) * 16 + (lane & 15);
                        const int p = v < w.few ? v : v - w.few + w.low;
                        next[x] = -1;
                        if (lw + x * kPrLoaders < 8 && p < end) {
                            next[x] = paged_row(a.w, w.b, p, w.kv_head);
                            if (next[x] < 0) report_status(a.w.status, AFX_ERR_INVALID_ARG);
                        }
                    }
                };
                auto fill = [&](const uint16_t* pages) {
                    const uint32_t tile = base + Cfg::kKV + slot * Cfg::kTile;
#pragma unroll
                    for (int x = 0; x < 3; ++x) {
                        const int blk = lw + x * kPrLoaders;
                        if (blk >= 8) continue;
#pragma unroll
                        for (int i = 0; i < 16 / RPI; ++i) {
                            const int row = i * RPI + lane / PIECES, piece = lane % PIECES;
                            const int64_t o = __shfl_sync(0xFFFFFFFFu, off[x], row);
                            put(tile, blk * 16 + row, piece, pages + (o < 0 ? 0 : o) + piece * 8, o < 0 ? 0 : 16);
                        }
                    }
                    // (the copies' arrival, and the thread's own, which hands on what it has stored beside them)
                    asm volatile("cp.async.mbarrier.arrive.shared::cta.b64 [%0];" ::"r"(smem_u32(&bar.full[slot])) : "memory");
                    mbar_arrive(&bar.full[slot]);
                };
                // Tiles that are read in boxes: warp j % 3 reads tile j, a box per lane (and half of the dims).
                const int n_boxed = w.boxed;
                int page = -1, in_page = 0;
                auto look_up_box = [&](int j) {
                    const int v = j * kPrPos + (lane % boxes) * args.box, p = v < w.few ? v : v - w.few + w.low;
                    page = paged_page(a.w, w.b, p, in_page);
                    if (page < 0) report_status(a.w.status, AFX_ERR_INVALID_ARG);
                };
                auto fill_boxes = [&](const CUtensorMap* map) {
                    const uint32_t tile = base + Cfg::kKV + slot * Cfg::kTile;
                    if (lane == 0) mbar_expect(&bar.full[slot], Cfg::kTile);
                    __syncwarp();
                    if (lane < boxes * (D / 64)) {
                        const int half = lane / boxes, i = lane % boxes;
                        // a page that is none: out of the tensor, zeros
                        tma_load_4d(tile + half * Cfg::kBlock + i * args.box * 128, map, half * 64, in_page, w.kv_head, page < 0 ? a.w.n_pages : page,
                                    &bar.full[slot]);
                    }
                    if (lane != 0) mbar_arrive(&bar.full[slot]);
                };
                if (lw < n_boxed) look_up_box(lw);
                if (n_boxed == 0 && it >= 0) look_up(0);
                for (int j = it < 0 ? -1 : 0; j < n_tiles; ++j) {
                    if (j >= 0) {
                        const bool boxed = j < n_boxed, mine = boxed && j % kPrLoaders == lw;
                        if (!boxed) {
#pragma unroll
                            for (int x = 0; x < 3; ++x) off[x] = next[x];
                        }
                        if (j + 1 < n_tiles && j + 1 >= n_boxed) look_up(j + 1);
                        ok = room();
                        if (!ok) break;
                        if (!boxed) {
#pragma unroll
                            for (int x = 0; x < 3; ++x) {
                                const uint32_t m = __ballot_sync(0xFFFFFFFFu, off[x] >= 0);
                                if (lane == 0 && lw + x * kPrLoaders < 8) page_ok[ok_slot][lw + x * kPrLoaders] = static_cast<uint16_t>(m);
                            }
                            fill(a.w.k);
                        } else if (mine) {
                            const uint32_t m = __ballot_sync(0xFFFFFFFFu, page >= 0);
                            if (lane < 8) page_ok[ok_slot][lane] = (m >> (lane * 16 / args.box)) & 1u ? 0xFFFFu : 0u;
                            fill_boxes(&k_map);
                        } else {
                            mbar_arrive(&bar.full[slot]);
                        }
                        ok_slot = (ok_slot + 1) & 7;
                        step();
                        if (j == 0) {
                            // the 256 query rows, 32 to a turn of the warp; the work before has made its last scores
                            if (q_used) {
                                ok = wait(&bar.q_empty, q_turn);
                                q_turn ^= 1u;
                                if (!ok) break;
                            }
                            q_used = true;
                            for (int blk = lw; blk < kPrTiles * kPrRows / 32; blk += kPrLoaders) {
                                const int rr = w.row_base + blk * 32 + lane, i = rr / a.rep;
                                const int64_t from = rr < rows ? (w.row0 + i) * a.ldq + static_cast<int64_t>(w.kv_head * a.rep + rr - i * a.rep) * D : -1;
#pragma unroll
                                for (int k = 0; k < 32 / RPI; ++k) {
                                    const int row = k * RPI + lane / PIECES, piece = lane % PIECES;
                                    const int64_t o = __shfl_sync(0xFFFFFFFFu, from, row);
                                    put(base + Cfg::kQ + (blk / 4) * Cfg::kTile, (blk % 4) * 32 + row, piece,
                                        reinterpret_cast<const uint16_t*>(a.q) + (o < 0 ? 0 : o) + piece * 8, o < 0 ? 0 : 16);
                                }
                            }
                            when_landed(&bar.q_full);
                        }
                        ok = room();
                        if (!ok) break;
                        if (!boxed) {
                            fill(a.w.v);
                        } else if (mine) {
                            fill_boxes(&v_map);
                            if (j + kPrLoaders < n_boxed) look_up_box(j + kPrLoaders);
                        } else {
                            mbar_arrive(&bar.full[slot]);
                        }
                        step();
                    }
                    if (lw == 2 && j == min(2, n_tiles - 1)) {
                        // the next work, as soon as this one's first tiles are on their way
                        int place = it < 0 ? static_cast<int>(blockIdx.x) : answered();
                        if (ok && it >= 1) ok = wait(&bar.work_empty[(it + 1) & 1], (((it + 1) >> 1) & 1) ^ 1);
                        if (!ok) break;
                        if (lane == 0) work[(it + 1) & 1].b = -1;
                        __syncwarp();
                        // places behind the last work (the grid is as large as the call could need) are taken over and left: less than a block each
                        for (bool first = it < 0; place >= 0 && !pr_find(args, place, first, &found, &work[(it + 1) & 1]); first = false) {
                            if (lane == 0) *const_cast<volatile uint32_t*>(&patience.told) = nanoseconds();
                            ask();
                            place = answered();
                        }
                        if (!ok) break;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bar.work_full[(it + 1) & 1]);
                        __syncwarp();
                    }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (lane == 0 && !ok) report_status(a.w.status, AFX_ERR_TIMEOUT);
            if (open) mbar_drain(&bar.answered, (asks - 1) & 1);  // the answer is written before the block ends
            if (lane == 0) steps[lw] = static_cast<int>(turn) * NB + slot;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPrRowRegs));
        // ---- softmax: a thread per row
        const int x = warp >> 2;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + x * kPrPos, o_at = tmem + lanes + 256 + x * D;
        const float scale = fabsf(a.scale);
        uint32_t s_turn = 0, o_turn = 0;
        int ok_slot = 0;
        bool ok = true;
        for (int it = 0; ok; ++it) {
            PrWork w;
            ok = next_work(it, w);
            if (!ok || w.b < 0) break;
            const int rows = w.rows;
            const int rr = w.row_base + x * kPrRows + (warp & 3) * 32 + lane;
            const int i = rr / a.rep, h = w.kv_head * a.rep + rr - i * a.rep;
            const bool live = rr < rows;
            const int pos = live ? w.first + i : -1;
            const int shift = w.few - w.low;  // place in the list of visible positions = position + shift, behind the first ones
            const int v_hi = pos + shift;     // the row sees places <= v_hi that are >= v_lo or < v_few
            const int v_lo = a.mask.window > 0 ? pos - a.mask.window + 1 + shift : 0;
            const int v_few = a.mask.window > 0 ? a.mask.sinks : 0;  // (first positions are their own places: few covers them, or few = low)
            // places that every row of the tile sees: below v_few and [lo_all, hi_all]
            const int rr0 = w.row_base + x * kPrRows, rr1 = min(rr0 + kPrRows, rows) - 1;
            const int hi_all = w.first + rr0 / a.rep + shift;
            const int lo_all = a.mask.window > 0 ? w.first + max(rr1, 0) / a.rep - a.mask.window + 1 + shift : 0;
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; ok && j < w.tiles[x]; ++j) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bar.s_full[x], s_turn, &patience));
                s_turn ^= 1u;
                if (!ok) break;
                tc_fence_after();
                float s[kPrPos];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(s + 32 * c, s_at + 32 * c);
                tmem_wait_ld();
                if (a.scale < 0.0f) {  // the largest of s times a negative scale is that of the smallest s
#pragma unroll
                    for (int c = 0; c < kPrPos; ++c) s[c] = -s[c];
                }
                const int v0 = j * kPrPos;
                const uint4 okw = *reinterpret_cast<const uint4*>(page_ok[(ok_slot + j) & 7]);
                const bool pages = (okw.x & okw.y & okw.z & okw.w) == 0xFFFFFFFFu;
                const bool all = pages && v0 + kPrPos - 1 <= hi_all && (v0 >= lo_all || v0 + kPrPos <= v_few);
                if (!all) {  // 32 places as bits: those up to v_hi that are from v_lo on or below v_few, and have a page
                    const uint32_t word[4] = {okw.x, okw.y, okw.z, okw.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int v = v0 + 32 * c;
                        const uint32_t see = pr_below(v_hi + 1 - v) & (~pr_below(v_lo - v) | pr_below(v_few - v)) & word[c];
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[32 * c + e] = (see & (1u << e)) != 0u ? s[32 * c + e] : -INFINITY;
                    }
                }
                if (j == 0) {  // the first maximum is the reference; afterwards it stays while it is not exceeded by far
                    float top = fmaxf(s[0], s[1]);
#pragma unroll
                    for (int c = 2; c < kPrPos; c += 2) top = max3(top, s[c], s[c + 1]);
                    m = top * scale;
                }
                const f32x2 scale2 = pack_f32x2(scale, scale);
                uint32_t p[kPrPos / 4];
                f32x2 sum[2];
                // The first half of the weights and, beside them, the maximum of all scores; when a row's has grown by too much
                // (seldom), the rows' sums so far are rescaled and the weights taken again.
                for (int pass = 0; pass < 2; ++pass) {
                    const float ref = m == -INFINITY ? 0.0f : m - kUpLog;
                    const f32x2 ref2 = pack_f32x2(-ref, -ref);
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    sum[0] = sum[1] = 0;
#pragma unroll
                    for (int e = 0; e < kPrPos / 4; ++e) {
                        p[e] = pr_weights<CT>(s[2 * e], s[2 * e + 1], scale2, ref2, sum[e & 1]);
                        mx[(2 * e) & 3] = max3(mx[(2 * e) & 3], s[4 * e], s[4 * e + 1]);
                        mx[(2 * e + 1) & 3] = max3(mx[(2 * e + 1) & 3], s[4 * e + 2], s[4 * e + 3]);
                    }
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                    const bool grow = top > m + kPrGrow || (m == -INFINITY && top > m);
                    if (pass == 1 || !__any_sync(0xFFFFFFFFu, grow)) break;
                    const float f = grow ? fast_exp2(m - top) : 1.0f;  // 0 where nothing was seen before
                    if (grow) m = top;
                    l *= f;
                    if (j > 0) {  // (the scores are there: what was issued before them, O's last addition too, is done)
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            float o[16];
                            tmem_ld16(o, o_at + 16 * c);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= f;
                            tmem_st16(o_at + 16 * c, reinterpret_cast<const uint32_t*>(o));
                        }
                    }
                }
                tmem_st16(s_at, p);
                tmem_st16(s_at + 16, p + 16);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.p_half[x]);  // half of the positions may be multiplied
                {
                    const float ref = m == -INFINITY ? 0.0f : m - kUpLog;
                    const f32x2 ref2 = pack_f32x2(-ref, -ref);
#pragma unroll
                    for (int e = 0; e < kPrPos / 4; ++e)
                        p[e] = pr_weights<CT>(s[kPrPos / 2 + 2 * e], s[kPrPos / 2 + 2 * e + 1], scale2, ref2, sum[e & 1]);
                }
                tmem_st16(s_at + 32, p);
                tmem_st16(s_at + 48, p + 16);
                float sums[4];
                unpack_f32x2(sum[0], sums[0], sums[1]);
                unpack_f32x2(sum[1], sums[2], sums[3]);
                l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.p_full[x]);
            }
            if (!ok) break;
            ok_slot = (ok_slot + max(w.tiles[0], w.tiles[1])) & 7;
            if (w.tiles[x] > 0) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bar.o_full[x], o_turn, &patience));
                o_turn ^= 1u;
                if (!ok) break;
                tc_fence_after();
            }
            // ---- the rows leave.  (Straight from the threads: staged in shared memory they would leave in whole lines, but the
            // next work's queries are on their way into the room for that.)
            const int64_t at = static_cast<int64_t>(w.row0 + i) * a.heads + h;
            float o[D];
            if (w.tiles[x] > 0) {
#pragma unroll
                for (int c = 0; c < D / 32; ++c) tmem_ld32(o + 32 * c, o_at + 32 * c);
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int c = 0; c < D; ++c) o[c] = 0.0f;
            }
            const bool none = l == 0.0f;
            const float inv = 1.0f / l;
            bool fin = true;
#pragma unroll
            for (int c = 0; c < D; ++c) {
                fin &= fabsf(o[c]) <= 3.402823466e38f;
                o[c] = none ? 0.0f : o[c] * inv;
            }
            // Rows whose sums are not finite.  Where they see what is not finite, that is what they are; but a weight of zero times a NaN or
            // an infinity that a row does not see has to be nothing.  Only the tiles at the ends of what the rows see hold places that
            // are masked: if a value there is not finite, the rows are taken again, over what they see alone.
            bool again = false;
            if (__any_sync(0xFFFFFFFFu, live && !fin)) {
                const uint32_t there = __ballot_sync(0xFFFFFFFFu, live);  // (the warp's rows in front)
                const int lo = max(__shfl_sync(0xFFFFFFFFu, pos, 0), -1), hi = __shfl_sync(0xFFFFFFFFu, pos, there != 0 ? 31 - __clz(there) : 0);
                const int back = min(w.end, w.tiles[x] * kPrPos - shift);  // behind the last tile's places
#pragma unroll 1
                for (int part = 0; part < (a.mask.window > 0 ? 3 : 1) && !again; ++part) {
                    const int from = part == 0 ? max(lo + 1, 0) : part == 1 ? w.low : min(a.mask.sinks, w.few);
                    const int to = part == 0 ? back : part == 1 ? min(max(hi - a.mask.window + 1, w.low), w.end) : w.few;
                    again = any_value_not_finite<D, CT>(a.w, w.b, w.kv_head, from, to);
                }
            }
            if (live && (fin || !again)) {
                uint16_t* dst = a.out + at * D;
                uint32_t y[D / 2];
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const float* t = o + 8 * c;
                    *reinterpret_cast<uint4*>(y + 4 * c) = a.out_type == AFX_F16 ? make_uint4(pack2_bits<AFX_F16>(t[0], t[1]), pack2_bits<AFX_F16>(t[2], t[3]),
                                                                pack2_bits<AFX_F16>(t[4], t[5]), pack2_bits<AFX_F16>(t[6], t[7]))
                                                   : make_uint4(pack2_bits<AFX_BF16>(t[0], t[1]), pack2_bits<AFX_BF16>(t[2], t[3]),
                                                                pack2_bits<AFX_BF16>(t[4], t[5]), pack2_bits<AFX_BF16>(t[6], t[7]));
                }
                if ((reinterpret_cast<uintptr_t>(a.out) & 31u) == 0) {  // whole sectors
#pragma unroll
                    for (int c = 0; c < D / 16; ++c)
                        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + 16 * c), "r"(y[8 * c]), "r"(y[8 * c + 1]),
                                     "r"(y[8 * c + 2]), "r"(y[8 * c + 3]), "r"(y[8 * c + 4]), "r"(y[8 * c + 5]), "r"(y[8 * c + 6]), "r"(y[8 * c + 7])
                                     : "memory");
                } else {
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) reinterpret_cast<uint4*>(dst)[c] = *reinterpret_cast<const uint4*>(y + 4 * c);
                }
            }
            if (live && a.lse != nullptr) a.lse[at] = none ? -INFINITY : (m + log2f(l) - kUpLog) * kLn2;  // (the values have no part in it)
            const uint32_t left = __ballot_sync(0xFFFFFFFFu, live && !fin && again);
#pragma unroll 1
            for (int half = 0; half < 2; ++half)
                if (((left >> (16 * half)) & 0xFFFFu) != 0u) {
                    const int rr2 = w.row_base + x * kPrRows + (warp & 3) * 32 + lane, i2 = rr2 / a.rep;
                    pr_again<D, CT>(a, w, half, left, i2, w.kv_head * a.rep + rr2 - i2 * a.rep, rr2 < w.rows ? w.first + i2 : -1, &patience);
                }
        }
        if (!ok && lane == 0) report_status(a.w.status, AFX_ERR_TIMEOUT);
    }
    // ---- nothing is in flight any more: all products were waited for by the rows' threads, all copies by the loaders or them
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (patience.gave_up != 0 && warp > 8) {
        // Boxes may be under way yet.  A slot's phase ends when its boxes are there and all three warps have arrived; one that gave
        // up owes arrivals for the steps that another has made (fewer than the ring has slots: a slot is filled again after all have
        // arrived for its step before), and makes them now.
        const int all = max(max(steps[0], steps[1]), steps[2]);
        for (int i = steps[warp - 9]; i < all; ++i) mbar_arrive(&bar.full[i % NB]);
        for (int i = max(all - NB, 0); i < all; ++i) mbar_drain(&bar.full[i % NB], (i / NB) & 1);
    }
    if (warp == 8) tmem_free(tmem, 512);
}

}  // namespace afx
