// Attention of few new tokens per sequence over the paged cache: the cached positions of all sequences are one list of
// tiles, cut into equal ranges, one per block; what a range leaves unfinished is joined by a second kernel.
//
// An item is (sequence, kv head, group of up to 16 rows); its rows are the sequence's new tokens times the query heads of
// the kv head.  Its positions are those that any of its tokens sees: the first `few` ones and the window from `low` on,
// counted through without the gap between them.  A tile is 64 of them; a block walks its range of the list, the
// positions of a tile 16 to a warp (a chunk), every warp with a ring of chunks of its own that cp.async fills across the borders of
// items: nobody waits for another warp before an item's end.  A chunk is two matrix products on the tensor cores
// (16 rows x 16 positions x D and 16 rows x D x 16 positions); softmax is online and in base 2, the weights are split
// into two 16-bit halves, fp32 queries likewise, which keep 22 of their bits in fp16 and 16 in bf16.  Where there are at most 8 rows (one new token
// and up to 8 heads per kv head), the two halves are the 16 rows of a product.
//
// Bound by HBM: 16 positions are 8 KB of K and V at D = 128 and about 250 instructions of a warp, an SM's share of the
// bandwidth is 8 KB every 190 ns = 1400 issue slots.  Two blocks of 4 warps per SM with rings of 96 KB each keep
// up to 128 KB of an SM on their way.  64 windows of 4096 positions, 32 / 8 heads: 167 us, 93 % of the copy rate; 61 sequences of 1 to
// 8192 positions, 64 / 8 heads: 65 us, 81 %; what is missing is latency (list 1.8 us, first look-ups and rows 2.5, join 3).
#pragma once

#include "afx_attn_mma.cuh"
#include "afx_paged_attn.cuh"

namespace afx {

constexpr int kFewWarps = 4;
constexpr int kFewThreads = kFewWarps * 32;
constexpr int kFewChunk = 16;
constexpr int kFewTile = kFewChunk * kFewWarps;
constexpr int kFewMaxBlocks = 296;  // ranges at most (two blocks on each of 148 SMs); sizes the workspace
constexpr int kFewRows = 16;
constexpr int kOneWarps = 8, kOneCluster = 16;  // one sequence: warps of a block, blocks of a cluster at most

template <int D>
struct FewCfg {
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kChunkBytes = 2 * kFewChunk * D * 2;  // K rows, V rows
    static constexpr int kWarpRing = kStages * kChunkBytes;
    static constexpr int kRing = kFewWarps * kWarpRing;
    static constexpr int kMerge = kFewWarps * 1024 * 4;        // [warp][1024 values of the partial outputs]
    static constexpr int kDyn = kRing + kMerge;
    // one sequence: the rings (where the warps' sums meet too, in the end), and the cluster's sums
    static constexpr int kOneRing = kOneWarps * kWarpRing;
    static constexpr int kOneRecv = (16 * D / 4 + kOneCluster) * 16;
    static constexpr int kOneDyn = kOneRing + kOneRecv + 2 * kOneCluster * 16 * 4;
};

// What an item costs beside its tiles (queries, the warps' sums), in tiles: the ranges are cut with it counted in.  (61 sequences
// of 1 to 8192 positions with a cold L2: 103, 83, 81 and 83 us with 1, 2, 3 and 5.)
constexpr int kFewItemCost = 3;

// The workspace: a descriptor per range, then slots of an unfinished item's sums (m[16], l[16], acc[16][D]).  Slot 2 i is
// the piece that range i begins with where the item began in an earlier range, 2 i + 1 the piece of the item that begins in
// range i and ends in a later one (the descriptor of range i tells which).
struct FewJoin {
    int32_t last;             // range in which the item ends; < 0: none
    int32_t row0, h0;         // the sequence's first token row, the kv head's first query head
    int32_t first, rows;      // rows first .. first + rows - 1 of (token, query head of the kv head)
    int32_t pad[3];
};
__host__ __device__ constexpr int few_slot_floats(int D) { return kFewRows * (D + 2); }
__host__ __device__ constexpr size_t few_slots_at() { return kFewMaxBlocks * sizeof(FewJoin); }
__host__ __device__ constexpr size_t few_workspace_bytes(int D) {
    return few_slots_at() + static_cast<size_t>(2) * kFewMaxBlocks * few_slot_floats(D) * sizeof(float);
}

struct PagedFewArgs {
    PagedAttnArgs a;
    int rows_per_group;  // 8 (packed) or 16
    int most;            // sequences of more new tokens are somebody else's
    uint32_t rep_mul;    // r / rep = (r * rep_mul) >> 32 for 0 <= r < 2^16 (rep > 1)
    FewJoin* joins;
    float* slots;
    int limit;           // tokens at positions from there on take no part
    bool past_final;     // what lies before the new tokens is final since two kernels ago
};

// Most new tokens of a sequence that these kernels take: AFX_MAX_T, or what makes `groups` groups of 16 rows.  More groups than
// AFX_MAX_T tokens have cost more products than a tile of 128 rows, but use the whole machine where the tiles are few: with up
// to as many groups as SMs in a call this is the faster way (a sequence of 4000 positions, 32 / 8 heads: 16 new tokens 16 us, by
// tiles 60, 32 new tokens 25 and 61; 32000 positions and 32 new tokens 144 and 417; 32 / 32 heads, 48 new tokens 43 and 61); beyond,
// the slower (32 / 32 heads, 128 new tokens at 1000 positions 30 and 23; 64 sequences of 16 new tokens at 2000 positions 329 and 154).
constexpr int kFewMostGroups = 16;
inline int few_most_tokens(int rep, int groups) {
    const int by_groups = groups * 16 / rep;
    return by_groups > AFX_MAX_T ? by_groups : AFX_MAX_T;
}
afx_status launch_paged_few(int dtype, int D, PagedFewArgs& f, cudaStream_t st);  // afx_paged_few.cu
inline bool few_packed(int max_new, int rep) { return static_cast<int64_t>(max_new) * rep <= 8; }

// A sequence in the list of tiles.
struct FewSeq {
    SeqSpan s;
    int few, low, nv;  // visible positions: [0, few) and low ..; nv of them
    int tiles;         // per item
    int items;         // kv heads times row groups
    int groups;        // row groups
};

__device__ __forceinline__ FewSeq few_seq(const PagedFewArgs& f, int b, int row0, bool report) {
    FewSeq q;
    q.s = paged_span(f.a.w, b, row0, report);
    if (q.s.n > f.most) q.s.n = 0;
    q.s.n = min(q.s.n, max(f.limit - q.s.first, 0));
    const int first = max(q.s.first, 0), end = min(q.s.len, q.s.first + q.s.n);
    q.low = paged_low(f.a.mask, first);
    q.few = paged_few(f.a.mask, q.low);
    q.nv = max(end - q.low, 0) + (end > q.low ? q.few : 0);
    q.groups = (q.s.n * f.a.rep + f.rows_per_group - 1) >> (f.rows_per_group == 8 ? 3 : 4);
    q.items = f.a.w.n_kv * q.groups;
    q.tiles = (q.nv + kFewTile - 1) / kFewTile;
    return q;
}

// a / b of non-negative numbers that usually have 32 bits (the 64-bit quotient is a hundred instructions)
__device__ __forceinline__ int64_t few_quotient(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Where a range begins in the list (units: tiles, and kFewItemCost in front of an item's).
struct FewStart {
    int64_t before;  // units in front of the sequence
    FewSeq q;
    int b;
};
struct FewScratch {
    int64_t warp_units[kFewWarps];
    FewStart start;
};
// The list's length.  All threads of the block call it.
// (row0: first token row of this thread's first sequence; last: the last of its sequences)
__device__ __forceinline__ int64_t few_list(const PagedFewArgs& f, FewScratch* sc, bool report, int& row0, int64_t& mine_before, int64_t& mine,
                                            FewSeq& last) {
    const int n = f.a.w.n_seqs, per = (n + kFewThreads - 1) / kFewThreads, tid = threadIdx.x;
    const int i0 = min(tid * per, n), i1 = min(n, i0 + per);
    row0 = paged_first_row(f.a.w, i0);
    int64_t incl;
    for (bool again = false;; again = true) {
        int at = row0;
        bool down = false;  // a start is below the one before it
        mine = 0;
        for (int i = i0; i < i1; ++i) {
            const FewSeq q = few_seq(f, i, at, report);
            last = q;
            mine += static_cast<int64_t>(q.tiles + kFewItemCost) * q.items;
            at = q.s.next;
            down |= f.a.w.start != nullptr && f.a.w.start[i + 1] < f.a.w.start[i];
        }
        incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane_id() >= o) incl += up;
        }
        if (lane_id() == 31) sc->warp_units[warp_id()] = incl;
        if (!__syncthreads_or(down) || again) break;
        for (int i = 0; i <= i0; ++i) row0 = max(row0, paged_first_row(f.a.w, i));
    }
    int64_t total = 0;
    mine_before = incl - mine;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
        if (w < warp_id()) mine_before += sc->warp_units[w];
        total += sc->warp_units[w];
    }
    return total;
}
// The thread among whose sequences unit `at` lies writes down which.
__device__ __forceinline__ void few_find(const PagedFewArgs& f, FewScratch* sc, int64_t at, int row0, int64_t mine_before, int64_t mine,
                                         const FewSeq& last) {
    if (at < mine_before || at >= mine_before + mine) return;
    const int n = f.a.w.n_seqs, per = (n + kFewThreads - 1) / kFewThreads;
    if (per == 1) {
        sc->start = {mine_before, last, static_cast<int>(threadIdx.x)};
        return;
    }
    for (int b = threadIdx.x * per; b < min(n, static_cast<int>(threadIdx.x + 1) * per); ++b) {
        const FewSeq q = few_seq(f, b, row0, false);
        const int64_t t = static_cast<int64_t>(q.tiles + kFewItemCost) * q.items;
        row0 = q.s.next;
        if (mine_before + t > at) {
            sc->start = {mine_before, q, b};
            break;
        }
        mine_before += t;
    }
}
// Range i holds units [i per + min(i, rest), ..): the first `rest` ranges one more.
struct FewRanges {
    int64_t per;
    int rest, n;
    __device__ __forceinline__ FewRanges(int64_t total, int blocks) {
        n = static_cast<int>(min(static_cast<int64_t>(blocks), total));
        per = n > 0 ? few_quotient(total, n) : 0;
        rest = n > 0 ? static_cast<int>(total - per * n) : 0;
    }
    __device__ __forceinline__ int64_t begin(int i) const { return per * i + min(i, rest); }
    __device__ __forceinline__ int of(int64_t unit) const {
        const int64_t wide = (per + 1) * rest;
        return static_cast<int>(unit < wide ? few_quotient(unit, per + 1) : rest + few_quotient(unit - wide, per));
    }
};

// A block's walk over its range: the pieces of items in it, one after the other.
struct FewWalk {
    FewSeq q;
    int b, item;
    int kv_head, group;  // of the item
    int t0, t1;         // this piece's tiles of the item
    int64_t left;       // units of the range behind this piece
    bool more;          // there is a piece

    __device__ __forceinline__ void place() {
        kv_head = item;
        if (q.groups > 1) kv_head = static_cast<int>(static_cast<uint32_t>(item) / static_cast<uint32_t>(q.groups));
        group = item - kv_head * q.groups;
    }
    // The piece from unit u0 of the item on; false where the range ends in front of its tiles.
    __device__ __forceinline__ bool cut(int u0) {
        const int u1 = static_cast<int>(min(static_cast<int64_t>(q.tiles + kFewItemCost), u0 + left));
        left -= u1 - u0;
        t0 = max(u0 - kFewItemCost, 0);
        t1 = max(u1 - kFewItemCost, 0);
        place();
        return t1 > t0 || q.tiles == 0;
    }
    __device__ __forceinline__ void next(const PagedFewArgs& f) {
        do {
            if (left <= 0) {
                more = false;
                return;
            }
            if (++item >= q.items) {
                item = 0;
                do {
                    if (++b >= f.a.w.n_seqs) {  // (lengths that changed under the call)
                        more = false;
                        return;
                    }
                    q = few_seq(f, b, q.s.next, false);
                } while (q.items == 0);
            }
        } while (!cut(0));
    }
    // chunks of this piece that warp w of W takes: w, w + W, ..
    template <int W>
    __device__ __forceinline__ int chunks(int w) const {
        const int n = (min(q.nv, t1 * (W * kFewChunk)) - t0 * (W * kFewChunk) + kFewChunk - 1) / kFewChunk;
        return n > w ? (n - w + W - 1) / W : 0;
    }
};

__device__ __forceinline__ void few_copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at));
}
// (a, b) rounded to the cache's type, and what that left out
template <int CT>
__device__ __forceinline__ void few_split(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack2_bits<CT>(a, b);
    const float2 f = pair_values<CT>(hi);
    lo = pack2_bits<CT>(a - f.x, b - f.y);
}

// Token of row rr of the sequence's rows.  rep_mul = floor(2^32 / rep) + 1 exceeds 2^32 / rep by at most 1: rr times that is below 1 / rep.
__device__ __forceinline__ int few_token(const PagedFewArgs& f, int rr) {
    return f.a.rep == 1 ? rr : static_cast<int>(__umulhi(static_cast<uint32_t>(rr), f.rep_mul));
}

// Row r (0 .. 15) of row group g of a piece: token row and position, query head.  live: it exists.
struct FewRow {
    int t, pos, h;
    bool live;
};
__device__ __forceinline__ FewRow few_row(const PagedFewArgs& f, const FewSeq& q, int kv_head, int group, int r) {
    const int rr = group * f.rows_per_group + r, i = few_token(f, rr);
    FewRow o;
    o.live = r < f.rows_per_group && i < q.s.n;
    o.t = q.s.row0 + i;
    o.pos = q.s.first + i;
    o.h = kv_head * f.a.rep + rr - i * f.a.rep;
    return o;
}
__device__ __forceinline__ int few_pos(const FewSeq& q, int v) { return v < q.few ? v : v - q.few + q.low; }
__device__ __forceinline__ bool few_sees(const PagedMask& m, int pos, int p) {
    return p <= pos && (m.window == 0 || p > pos - m.window || p < m.sinks);
}

// Where value d of row r lies among the sums that meet: blocks of 8 values change places by the row (all rows of a product
// at the same banks otherwise).
template <int DW>
__device__ __forceinline__ int few_place(int r, int d) {
    return r * DW + (d ^ ((r & 7) << 3));
}

// Sums that are NaN (of rows `bad`, 64 dims, a lane's two at a time) where the values that are not finite and that the row sees add up
// to something else: these are the sum.  One pass over the piece's values for all rows; it ends when what is left is NaN.
template <int D, int CT, int W>
__device__ __forceinline__ void few_infinite(const PagedFewArgs& f, const FewWalk& c, int warp, uint32_t bad, int part, float* sums) {
    const int lane = lane_id(), n_chunks = c.chunks<W>(warp);
    uint32_t open[2] = {0, 0}, hit[2] = {0, 0};  // rows with a NaN in the lane's first and second dim, and those where a value was found
    for (uint32_t left = bad; left != 0; left &= left - 1) {
        const int r = __ffs(left) - 1;
        float* s = sums + few_place<64>(r, 2 * lane);
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (s[x] != s[x]) {
                open[x] |= 1u << r;
                s[x] = 0.0f;
            }
    }
    for (int k = 0; k < n_chunks && __any_sync(0xFFFFFFFFu, (open[0] | open[1]) != 0u); ++k) {
        const int v0 = ((c.t0 + k) * W + warp) * kFewChunk, n = min(kFewChunk, c.q.nv - v0);
        const int64_t mine = lane < n ? paged_row(f.a.w, c.b, few_pos(c.q, v0 + lane), c.kv_head) : -1;
        uint32_t raw[kFewChunk];
#pragma unroll
        for (int j = 0; j < kFewChunk; ++j) {
            const int64_t at = __shfl_sync(0xFFFFFFFFu, mine, j);
            raw[j] = at >= 0 ? reinterpret_cast<const uint32_t*>(f.a.w.v + at + part * 64)[lane] : 0u;
        }
#pragma unroll
        for (int j = 0; j < kFewChunk; ++j) {
            if (not_finite<CT>(raw[j]) == 0u) continue;
            const float2 v = pair_values<CT>(raw[j]);
            const int p = few_pos(c.q, v0 + j);
            for (uint32_t left = open[0] | open[1]; left != 0; left &= left - 1) {
                const int r = __ffs(left) - 1;
                const FewRow fr = few_row(f, c.q, c.kv_head, c.group, r);
                if (!fr.live || !few_sees(f.a.mask, fr.pos, p)) continue;
                float* s = sums + few_place<64>(r, 2 * lane);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float value = x == 0 ? v.x : v.y;
                    if (!((open[x] >> r) & 1u) || fabsf(value) <= 3.402823466e38f) continue;
                    s[x] += value;
                    hit[x] |= 1u << r;
                    if (s[x] != s[x]) open[x] &= ~(1u << r);
                }
            }
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
        for (uint32_t left = open[x] & ~hit[x]; left != 0; left &= left - 1) sums[few_place<64>(__ffs(left) - 1, 2 * lane) + x] = NAN;
}

// Four dims of a finished row; nothing seen: zeros.
template <int D>
__device__ __forceinline__ void few_store(const PagedFewArgs& f, int t, int h, int d, const float4& s, float M, float L) {
    const bool none = L == 0.0f;
    const float inv = 1.0f / L;
    const float4 v = none ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv);
    const int64_t at = static_cast<int64_t>(t) * f.a.heads + h;
    uint2 y;
    if (f.a.out_type == AFX_F16)
        y = make_uint2(pack2_bits<AFX_F16>(v.x, v.y), pack2_bits<AFX_F16>(v.z, v.w));
    else
        y = make_uint2(pack2_bits<AFX_BF16>(v.x, v.y), pack2_bits<AFX_BF16>(v.z, v.w));
    *reinterpret_cast<uint2*>(f.a.out + at * D + d) = y;
    if (f.a.lse != nullptr && d == 0) f.a.lse[at] = none ? -INFINITY : (M + log2f(L)) * kLn2;
}

// ONE: the cache of one sequence.  All its items have the same length, so that a cluster of blocks takes an item, a block an
// equal share of its tiles (8 warps and the whole SM), and the sums meet through distributed shared memory: one kernel, no
// list, no workspace.  grid (blocks of a cluster, items).
template <int D, int CT, bool PACK, bool QF32, bool ONE>
__global__ void __launch_bounds__(ONE ? kOneWarps * 32 : kFewThreads, ONE ? 1 : 2) paged_few_kernel(PagedFewArgs f) {
    using Cfg = FewCfg<D>;
    constexpr int W = ONE ? kOneWarps : kFewWarps, THREADS = W * 32;
    constexpr int ST = Cfg::kStages, NK = D / 16, NT = D / 8, PIECES = D / 8;
    constexpr int NR = PACK ? 1 : 2;                       // rows of a lane: gid (and gid + 8)
    constexpr float kUp = CT == AFX_F16 ? 1024.0f : 1.0f;  // weights are carried times this: the low halves of small ones stay normal
    extern __shared__ __align__(128) unsigned char dyn[];
    __shared__ uint32_t stage_mask[W][ST];
    __shared__ float sm_m[W][kFewRows], sm_l[W][kFewRows];
    __shared__ FewScratch scratch;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    // where warp w's sums meet the others': behind the rings, or in its ring, which is empty by then
    auto merge = [&](int w) { return reinterpret_cast<float*>(dyn + (ONE ? w * Cfg::kWarpRing : Cfg::kRing + w * 4096)); };
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(dyn)) + warp * Cfg::kWarpRing;

    if constexpr (ONE) cluster_arrive();
    bool waited = false;  // (the same for a warp)
    auto depend = [&]() {
        if (waited) return;
        waited = true;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        // A block of ONE fills its SM.  Were the next kernel let in now, its blocks would all wait on the few SMs without one,
        // and share them afterwards: a layer step of 4096 x 11008 with 2049 positions took 97 us like that, 75 without.
        if constexpr (!ONE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    };
    // Inside a layer step the previous kernel is the one that stores the new tokens' rows.  Lengths, table and what lies
    // before the first new position were there earlier: the first chunks are requested while it runs.  Not for several
    // sequences: one's past may be another's new token, where they share pages.
    if (!ONE || !f.past_final) depend();

    const int my = blockIdx.x;  // range, or rank in the cluster
    FewWalk con;
    FewRanges ranges(0, 1);
    int64_t hi = 0;
    if constexpr (ONE) {
        con.b = 0;
        con.q = few_seq(f, 0, paged_first_row(f.a.w, 0), blockIdx.x == 0 && blockIdx.y == 0);
        con.item = blockIdx.y;
        if (con.item >= con.q.items) {  // (the same for the cluster)
            depend();
            cluster_wait();
            return;
        }
        con.q.tiles = (con.q.nv + W * kFewChunk - 1) / (W * kFewChunk);
        const int64_t S = gridDim.x;
        con.place();
        con.t0 = static_cast<int>(static_cast<uint32_t>(my * con.q.tiles) / static_cast<uint32_t>(S));
        con.t1 = static_cast<int>(static_cast<uint32_t>((my + 1) * con.q.tiles) / static_cast<uint32_t>(S));
        con.left = 0;
        con.more = true;
    } else {
        int row0;
        int64_t mine_before, mine;
        FewSeq last;
        const int64_t total = few_list(f, &scratch, blockIdx.x == 0, row0, mine_before, mine, last);
        ranges = FewRanges(total, gridDim.x);
        if (tid == 0) f.joins[my].last = -1;  // (a later piece may say otherwise)
        if (my >= ranges.n) return;
        const int64_t lo = ranges.begin(my);
        hi = ranges.begin(my + 1);
        few_find(f, &scratch, lo, row0, mine_before, mine, last);
        __syncthreads();
        con.b = scratch.start.b;
        con.q = scratch.start.q;
        const int64_t u = lo - scratch.start.before;
        const int per_item = con.q.tiles + kFewItemCost;
        con.item = static_cast<int>(few_quotient(u, per_item));
        con.left = hi - lo;
        con.more = true;
        if (!con.cut(static_cast<int>(u - static_cast<int64_t>(con.item) * per_item))) con.next(f);
    }

    // ---- the ring's filling side: chunk after chunk of this warp, across pieces
    FewWalk pro = con;
    int pk = 0, pn = pro.more ? pro.chunks<W>(warp) : 0, p_stage = 0;
    // the item's query rows into L1, a line of 128 bytes per lane: they are wanted as soon as its first chunk is there
    auto warm_queries = [&](const FewWalk& w) {
        constexpr int LINES = D * (QF32 ? 4 : 2) / 128;
        for (int x = lane; x < (PACK ? 8 : 16) * LINES; x += 32) {
            const FewRow r = few_row(f, w.q, w.kv_head, w.group, x / LINES);
            if (r.live) {
                const char* at = f.a.q + (r.t * f.a.ldq + static_cast<int64_t>(r.h) * D) * (QF32 ? 4 : 2) + x % LINES * 128;
                asm volatile("prefetch.global.L1 [%0];" ::"l"(at));
            }
        }
    };
    // Lane j < 16: where position j of the next chunk lies.  The table's entry is not looked at here, but when the chunk is
    // requested: nobody waits for it meanwhile.  Moves on.
    struct Ahead {
        int64_t rest;  // what comes to the page's offset
        int page;
        int kind;      // 0: a position, -1: behind the last one, -2: there is no chunk (the same for all lanes)
        bool fresh;    // a new token's position
    };
    auto look_up = [&]() -> Ahead {
        while (pro.more && pk >= pn) {
            pro.next(f);
            pk = 0;
            pn = pro.more ? pro.chunks<W>(warp) : 0;
            if (pro.more) warm_queries(pro);  // (never of ONE, whose blocks have a piece each)
        }
        Ahead a = {0, 0, -2, false};
        if (!pro.more) return a;
        const int v = ((pro.t0 + pk) * W + warp) * kFewChunk + (lane & 15);
        ++pk;
        a.kind = v < pro.q.nv ? 0 : -1;
        if (a.kind == 0) {
            int in_page;
            const int p = few_pos(pro.q, v);
            a.fresh = p >= pro.q.s.first;
            a.page = paged_entry(f.a.w, pro.b, p, in_page);
            a.rest = in_page * f.a.w.pos_stride + pro.kv_head * f.a.w.head_stride;
        }
        return a;
    };
    auto issue = [&](const Ahead& a) {
        if (a.kind != -2) {
            const bool good = a.kind == 0 && static_cast<uint32_t>(a.page) < static_cast<uint32_t>(f.a.w.n_pages);
            if (a.kind == 0 && !good) report_status(f.a.w.status, AFX_ERR_INVALID_ARG);
            const int64_t p_off = good ? a.page * f.a.w.page_stride + a.rest : -1;
            const uint32_t at = ring + p_stage * Cfg::kChunkBytes;
            const uint32_t mask = __ballot_sync(0xFFFFFFFFu, good) & 0xFFFFu;
            if (lane == 0) stage_mask[warp][p_stage] = mask;
            constexpr int RPI = 32 / PIECES;  // rows per instruction
#pragma unroll
            for (int i = 0; i < kFewChunk / RPI; ++i) {
                const int row = i * RPI + lane / PIECES, piece = lane % PIECES;
                const int64_t off = __shfl_sync(0xFFFFFFFFu, p_off, row);
                const int64_t e = (off < 0 ? 0 : off) + piece * 8;
                const uint32_t d = at + row * (D * 2) + ((piece ^ (row & 7)) << 4);
                few_copy16(d, f.a.w.k + e, off < 0 ? 0 : 16);
                few_copy16(d + kFewChunk * D * 2, f.a.w.v + e, off < 0 ? 0 : 16);
            }
            p_stage = p_stage + 1 == ST ? 0 : p_stage + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (waited && con.more) warm_queries(con);
    Ahead ahead;  // the chunk behind those on their way: looked up a chunk's time before it is wanted
    {
        Ahead off[ST - 1];
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) off[i] = look_up();
        ahead = look_up();
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) {
            if (!waited && __any_sync(0xFFFFFFFFu, off[i].fresh)) depend();
            issue(off[i]);
        }
    }
    depend();

    int stage = 0;
    for (; con.more; con.next(f)) {
        const FewSeq& q = con.q;
        const int kv_head = con.kv_head, group = con.group;
        // ---- queries of the lane's rows as fragments of the first product
        uint32_t qa[NK][4], ql[QF32 && !PACK ? NK : 1][4];
        float unit[NR];
        int pos[NR];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const FewRow r = few_row(f, q, kv_head, group, gid + 8 * e);
            if (e < NR) {
                unit[e < NR ? e : 0] = f.a.scale;
                pos[e < NR ? e : 0] = r.live ? r.pos : -1;
            }
            const bool row = r.live && e < NR;
            const int64_t at = row ? r.t * f.a.ldq + static_cast<int64_t>(r.h) * D : 0;
            if constexpr (QF32) {
                const float* src = reinterpret_cast<const float*>(f.a.q) + at;
                float2 x[2 * NK];
                float big = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * NK; ++i) {
                    x[i] = row ? *reinterpret_cast<const float2*>(src + 8 * i + 2 * tig) : make_float2(0.0f, 0.0f);
                    big = fmaxf(big, fmaxf(fabsf(x[i].x), fabsf(x[i].y)));
                }
                float up = 1.0f;
                if constexpr (CT == AFX_F16) {  // the row's largest value lands in [2^9, 2^10): fp16's range holds both halves
                    big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
                    const int ex = min(max(static_cast<int>((__float_as_uint(big) >> 23) & 0xFFu) - 127, -100), 110);
                    up = __uint_as_float(static_cast<uint32_t>(127 + 9 - ex) << 23);
                    if (e < NR) unit[e < NR ? e : 0] = f.a.scale * __uint_as_float(static_cast<uint32_t>(127 - 9 + ex) << 23);
                }
                if (e < NR) {
#pragma unroll
                    for (int i = 0; i < 2 * NK; ++i) {
                        uint32_t h16, l16;
                        few_split<CT>(x[i].x * up, x[i].y * up, h16, l16);
                        qa[i >> 1][2 * (i & 1) + e] = h16;
                        if constexpr (PACK) qa[i >> 1][2 * (i & 1) + 1] = l16;
                        else ql[i >> 1][2 * (i & 1) + e] = l16;
                    }
                }
            } else {
                const uint16_t* src = reinterpret_cast<const uint16_t*>(f.a.q) + at;
#pragma unroll
                for (int i = 0; i < 2 * NK; ++i)
                    qa[i >> 1][2 * (i & 1) + e] = row ? *reinterpret_cast<const uint32_t*>(src + 8 * i + 2 * tig) : 0u;
            }
        }
        float m[NR], l[NR], o[NT][4];
#pragma unroll
        for (int e = 0; e < NR; ++e) {
            m[e] = -INFINITY;
            l[e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i][x] = 0.0f;
        const int last = q.s.first + q.s.n - 1;
        const int n_chunks = con.chunks<W>(warp);
        for (int k = 0; k < n_chunks; ++k) {
            const int v0 = ((con.t0 + k) * W + warp) * kFewChunk;
            asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
            __syncwarp();
            const uint32_t kat = ring + stage * Cfg::kChunkBytes, vat = kat + kFewChunk * D * 2;
            const uint32_t vm = stage_mask[warp][stage];
            float c[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            float cl[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            {
                const int row = (lane & 7) + ((lane & 16) >> 1), half = (lane >> 3) & 1;
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    uint32_t kb[4];
                    ldmatrix_x4(kb, kat + row * (D * 2) + (((2 * j + half) ^ (row & 7)) << 4));
                    mma_16816<CT>(c[0], qa[j], kb[0], kb[1]);
                    mma_16816<CT>(c[1], qa[j], kb[2], kb[3]);
                    if constexpr (QF32 && !PACK) {
                        mma_16816<CT>(cl[0], ql[j], kb[0], kb[1]);
                        mma_16816<CT>(cl[1], ql[j], kb[2], kb[3]);
                    }
                }
            }
            float s[NR][4];  // positions 2 tig, 2 tig + 1, 8 + 2 tig, 9 + 2 tig
#pragma unroll
            for (int e = 0; e < NR; ++e)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float hi32 = c[x >> 1][2 * e + (x & 1)];
                    float t = hi32;
                    if constexpr (PACK) { if constexpr (QF32) t = whole(hi32, c[x >> 1][2 + (x & 1)]); }
                    else if constexpr (QF32) t = whole(hi32, cl[x >> 1][2 * e + (x & 1)]);
                    s[e][x] = t * unit[e];
                }
            // every row sees the whole chunk, in the usual case
            bool all = vm == 0xFFFFu;
            if (q.s.n > 1 && all) {
                const int p0 = few_pos(q, v0), p1 = few_pos(q, v0 + kFewChunk - 1);
                all = p1 <= q.s.first && (f.a.mask.window == 0 || p0 > last - f.a.mask.window || p1 < f.a.mask.sinks);
            }
            if (!all) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int j = 8 * (x >> 1) + 2 * tig + (x & 1), p = few_pos(q, v0 + j);
#pragma unroll
                    for (int e = 0; e < NR; ++e)
                        if (!((vm >> j) & 1u) || !few_sees(f.a.mask, pos[e], p)) s[e][x] = -INFINITY;
                }
            }
            uint32_t pa[4], pl[4];
            float grow[NR], ref[NR];
            bool moved = false;
#pragma unroll
            for (int e = 0; e < NR; ++e) {
                float mn = fmaxf(fmaxf(s[e][0], s[e][1]), fmaxf(s[e][2], s[e][3]));
                mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, 1));
                mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, 2));
                mn = fmaxf(mn, m[e]);
                ref[e] = mn == -INFINITY ? 0.0f : mn;
                grow[e] = fast_exp2(m[e] - ref[e]);  // 0 where nothing was seen before
                moved |= mn > m[e];
                m[e] = mn;
            }
            if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
                for (int e = 0; e < NR; ++e) l[e] *= grow[e];
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[i][x] *= grow[PACK ? 0 : x >> 1];
            }
#pragma unroll
            for (int e = 0; e < NR; ++e) {
                float p[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) p[x] = fast_exp2(s[e][x] - ref[e]) * kUp;
                l[e] += (p[0] + p[1]) + (p[2] + p[3]);
                if constexpr (PACK) {
                    few_split<CT>(p[0], p[1], pa[0], pa[1]);
                    few_split<CT>(p[2], p[3], pa[2], pa[3]);
                } else {
                    few_split<CT>(p[0], p[1], pa[e], pl[e]);
                    few_split<CT>(p[2], p[3], pa[2 + e], pl[2 + e]);
                }
            }
            // A weight of zero times an infinity or a NaN that its row does not see has to be nothing: in a chunk that not every row sees
            // such values are added to the rows that see them and are zeros for the product.  (One token sees all that is read.)
            if (!all && q.s.n > 1) {
                uint4* vs = reinterpret_cast<uint4*>(dyn + warp * Cfg::kWarpRing + stage * Cfg::kChunkBytes + kFewChunk * D * 2);
                uint32_t found = 0;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) found |= not_finite<CT>(vs[i * 32 + lane]);
                if (__any_sync(0xFFFFFFFFu, found != 0u)) {
#pragma unroll 1
                    for (int j = 0; j < kFewChunk; ++j) {
                        const int p = few_pos(q, v0 + j);
                        const uint32_t* at = reinterpret_cast<const uint32_t*>(vs + j * PIECES) + tig;
#pragma unroll
                        for (int e = 0; e < NR; ++e) {
                            if (!((vm >> j) & 1u) || !few_sees(f.a.mask, pos[e], p)) continue;
#pragma unroll
                            for (int i = 0; i < NT; ++i) {
                                const float2 v = pair_values<CT>(at[(i ^ (j & 7)) * 4]);
                                if (!(fabsf(v.x) <= 3.402823466e38f)) o[i][2 * e] += v.x;
                                if (!(fabsf(v.y) <= 3.402823466e38f)) o[i][2 * e + 1] += v.y;
                            }
                        }
                    }
                    __syncwarp();
#pragma unroll 1
                    for (int i = 0; i < D / 16; ++i) {
                        uint4 x = vs[i * 32 + lane];
                        uint32_t* w = &x.x;
#pragma unroll
                        for (int c = 0; c < 4; ++c) w[c] &= ~((not_finite<CT>(w[c]) >> 15) * 0xFFFFu);
                        vs[i * 32 + lane] = x;
                    }
                    __syncwarp();
                }
            }
            {
                const int row = (lane & 7) + (lane & 8), half = lane >> 4;
#pragma unroll
                for (int i = 0; i < NT; i += 2) {
                    uint32_t vb[4];
                    ldmatrix_x4_trans(vb, vat + row * (D * 2) + (((i + half) ^ (row & 7)) << 4));
                    mma_16816<CT>(o[i], pa, vb[0], vb[1]);
                    mma_16816<CT>(o[i + 1], pa, vb[2], vb[3]);
                    if constexpr (!PACK) {
                        mma_16816<CT>(o[i], pl, vb[0], vb[1]);
                        mma_16816<CT>(o[i + 1], pl, vb[2], vb[3]);
                    }
                }
            }
            __syncwarp();
            stage = stage + 1 == ST ? 0 : stage + 1;
            issue(ahead);
            ahead = look_up();
        }

        // ---- the warps' sums meet
        uint32_t bad = 0;  // rows with sums that are NaN: in 16 rows the signs of a weight's two halves may make an infinity that they see one
#pragma unroll
        for (int e = 0; e < NR; ++e) {
            l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 1);
            l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 2);
            bool nan = false;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float& t = o[i][2 * e + x];
                    if constexpr (PACK) t = whole(t, o[i][2 + x]);
                    t *= 1.0f / kUp;
                    nan |= t != t;
                }
            if constexpr (!PACK) {
                const uint32_t lanes = __ballot_sync(0xFFFFFFFFu, nan);
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if ((lanes >> (4 * r)) & 0xFu) bad |= 1u << (r + 8 * e);
            }
        }
        if (tig == 0) {
#pragma unroll
            for (int e = 0; e < NR; ++e) {
                sm_m[warp][gid + 8 * e] = m[e];
                sm_l[warp][gid + 8 * e] = l[e] * (1.0f / kUp);
            }
        }
        const bool whole_item = !ONE && con.t0 == 0 && con.t1 == q.tiles;
        float* slot = ONE ? nullptr : f.slots + static_cast<int64_t>(2 * my + (con.t0 > 0 ? 0 : 1)) * few_slot_floats(D);
        if (!ONE && !whole_item && con.t0 == 0 && tid == 0) {  // this range has the item joined
            const int64_t end = hi + (q.tiles - con.t1);   // (its piece ends the range)
            const int first = group * f.rows_per_group;
            FewJoin j = {};
            j.last = ranges.of(end - 1);
            j.row0 = q.s.row0;
            j.h0 = kv_head * f.a.rep;
            j.first = first;
            j.rows = min(f.rows_per_group, q.s.n * f.a.rep - first);
            f.joins[my] = j;
        }
        // 1024 values of a warp at a time: 8 rows x 128 dims, 16 rows x 64 dims (twice), 8 rows x 64 dims
        constexpr int RW = PACK ? 8 : 16, DW = PACK ? D : 64;
#pragma unroll
        for (int part = 0; part < D / DW; ++part) {
            float* mine = merge(warp);
#pragma unroll
            for (int i = 0; i < DW / 8; ++i)
#pragma unroll
                for (int e = 0; e < NR; ++e) {
                    const float* t = &o[part * (DW / 8) + i][2 * e];
                    *reinterpret_cast<float2*>(mine + few_place<DW>(gid + 8 * e, 8 * i + 2 * tig)) = make_float2(t[0], t[1]);
                }
            __syncwarp();
            if constexpr (!PACK) {
                if (bad != 0) few_infinite<D, CT, W>(f, con, warp, bad, part, mine);
                __syncwarp();
            }
            if (ONE && part == 0) cluster_wait();  // the peers are running
            __syncthreads();
            // four neighbouring dims of a row per thread and turn
            for (int x = tid * 4; x < RW * DW; x += THREADS * 4) {
                const int r = x / DW, d = part * DW + x % DW;
                const FewRow fr = few_row(f, q, kv_head, group, r);
                if (!fr.live) continue;
                float M = -INFINITY;
#pragma unroll
                for (int w = 0; w < W; ++w) M = fmaxf(M, sm_m[w][r]);
                float L = 0.0f;
                float4 s4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float4 t = *reinterpret_cast<const float4*>(merge(w) + few_place<DW>(r, x % DW));
                    const float wt = sm_m[w][r] == -INFINITY ? 0.0f : fast_exp2(sm_m[w][r] - M);
                    if (wt == 0.0f && sm_l[w][r] == 0.0f) continue;
                    L = fmaf(wt, sm_l[w][r], L);
                    s4.x = fmaf(wt, t.x, s4.x);
                    s4.y = fmaf(wt, t.y, s4.y);
                    s4.z = fmaf(wt, t.z, s4.z);
                    s4.w = fmaf(wt, t.w, s4.w);
                }
                if constexpr (ONE) {  // block e % S of the cluster finishes the e-th four values
                    cg::cluster_group cluster = cg::this_cluster();
                    const int S = gridDim.x, e = (r * D + d) / 4, per = (RW * D / 4 + S - 1) / S;
                    float4* recv = reinterpret_cast<float4*>(dyn + Cfg::kOneRing);
                    cluster.map_shared_rank(recv, e % S)[my * per + e / S] = s4;
                    if (d / 4 < S) {
                        float* ml = cluster.map_shared_rank(reinterpret_cast<float*>(dyn + Cfg::kOneRing + Cfg::kOneRecv), d / 4);
                        ml[my * kFewRows + r] = M;
                        ml[(kOneCluster + my) * kFewRows + r] = L;
                    }
                } else if (whole_item) {
                    few_store<D>(f, fr.t, fr.h, d, s4, M, L);
                } else {
                    *reinterpret_cast<float4*>(slot + 2 * kFewRows + r * D + d) = s4;
                    if (d == 0) {
                        slot[r] = M;
                        slot[kFewRows + r] = L;
                    }
                }
            }
            __syncthreads();
        }
    }
    if constexpr (ONE) {
        cluster_arrive();
        cluster_wait();
        const FewSeq& q = con.q;
        constexpr int RW = PACK ? 8 : 16;
        const int S = gridDim.x, per = (RW * D / 4 + S - 1) / S;
        const float4* recv = reinterpret_cast<const float4*>(dyn + Cfg::kOneRing);
        const float* ml = reinterpret_cast<const float*>(dyn + Cfg::kOneRing + Cfg::kOneRecv);
        for (int i = tid; my + S * i < RW * D / 4; i += THREADS) {
            const int e = (my + S * i) * 4, r = e / D, d = e % D;
            const FewRow fr = few_row(f, q, con.kv_head, con.group, r);
            if (!fr.live) continue;
            float M = -INFINITY, L = 0.0f;
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int k = 0; k < S; ++k) M = fmaxf(M, ml[k * kFewRows + r]);
            for (int k = 0; k < S; ++k) {
                const float m = ml[k * kFewRows + r], l = ml[(kOneCluster + k) * kFewRows + r];
                if (m == -INFINITY && l == 0.0f) continue;  // (nothing seen there)
                const float wt = fast_exp2(m - M);
                const float4 t = recv[k * per + i];
                L = fmaf(wt, l, L);
                s.x = fmaf(wt, t.x, s.x);
                s.y = fmaf(wt, t.y, s.y);
                s.z = fmaf(wt, t.z, s.z);
                s.w = fmaf(wt, t.w, s.w);
            }
            few_store<D>(f, fr.t, fr.h, d, s, M, L);
        }
    }
}

// Joins what the ranges left unfinished, in the ranges' order: grid (ranges, pieces of 512 values of an item).
template <int D>
__global__ void __launch_bounds__(kFewThreads) paged_join_kernel(PagedFewArgs f) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const FewJoin j = f.joins[blockIdx.x];
    const int x = (static_cast<int>(blockIdx.y) * kFewThreads + static_cast<int>(threadIdx.x)) * 4, r = x / D, d = x % D;
    if (j.last < 0 || r >= j.rows) return;
    float M = -INFINITY, L = 0.0f;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    constexpr int U = 8;  // pieces on their way at once
    for (int i0 = blockIdx.x; i0 <= j.last; i0 += U) {
        float m[U], l[U];
        float4 t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u, j.last);
            const float* slot = f.slots + static_cast<int64_t>(2 * i + (i == static_cast<int>(blockIdx.x) ? 1 : 0)) * few_slot_floats(D);
            m[u] = slot[r];
            l[u] = slot[kFewRows + r];
            t[u] = *reinterpret_cast<const float4*>(slot + 2 * kFewRows + r * D + d);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u > j.last || (m[u] == -INFINITY && l[u] == 0.0f)) continue;  // (nothing seen there)
            const float mn = fmaxf(M, m[u]), wa = M == -INFINITY ? 0.0f : fast_exp2(M - mn), wb = fast_exp2(m[u] - mn);
            M = mn;
            L = fmaf(L, wa, l[u] * wb);
            s.x = fmaf(s.x, wa, t[u].x * wb);
            s.y = fmaf(s.y, wa, t[u].y * wb);
            s.z = fmaf(s.z, wa, t[u].z * wb);
            s.w = fmaf(s.w, wa, t[u].w * wb);
        }
    }
    const int rr = j.first + r, i = few_token(f, rr);
    few_store<D>(f, j.row0 + i, j.h0 + rr - i * f.a.rep, d, s, M, L);
}

}  // namespace afx
