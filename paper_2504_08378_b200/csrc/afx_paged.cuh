// Paged key-value cache: what the kernels of afx_paged_append and afx_paged_attn share -- the device view of the
// caller's descriptor, the bounds checks of device data, and which positions a token sees.
#pragma once

#include "afx_common.cuh"

namespace afx {

struct PagedView {
    uint16_t* k;
    uint16_t* v;
    const int32_t* table;
    const int32_t* len;
    const int32_t* start;  // or NULL: sequence b has the one row b
    int32_t* status;
    int64_t page_stride, pos_stride, head_stride, table_stride;
    int n_kv, n_pages, n_seqs, n_tokens, max_new, page_size;
    int cap;       // positions that a row of the table can hold
    uint32_t mul;  // p / page_size = (p * mul) >> (31 + shift) for 0 <= p < 2^31
    int shift;
};

// The rows that visible positions come from: token at position p sees [0, min(sinks, lo)) and [lo, p].
struct PagedMask {
    int window, sinks;  // window 0: none
};

struct SeqSpan {
    int row0;   // first token row
    int n;      // rows taken part in (at most max_new)
    int first;  // position of row0 (negative: more new tokens than positions)
    int len;    // positions of the cache
    int next;   // first token row of the next sequence
};

// Host: checks the descriptor and fills the view.  AFX_OK with n_seqs = 0 or n_tokens = 0: nothing to do.
afx_status paged_view(const afx_paged_kv* kv, int32_t* dev_status, PagedView* out);  // afx_paged.cu

// A sequence's rows begin at the largest start so far (starts that decrease are clamped to it): at start[b] where none
// decreases, and where the sequence before it ends (next) in any case.
__device__ __forceinline__ int paged_first_row(const PagedView& w, int b) {
    return w.start != nullptr ? min(max(w.start[b], 0), w.n_tokens) : b;
}
__device__ __forceinline__ SeqSpan paged_span(const PagedView& w, int b, int row0, bool report) {
    SeqSpan s;
    const int len = w.len[b], hi = w.start != nullptr ? w.start[b + 1] : b + 1;
    const int row1 = min(max(hi, row0), w.n_tokens);
    s.len = min(max(len, 0), w.cap);
    s.row0 = row0;
    s.next = row1;
    s.first = s.len - (row1 - row0);
    s.n = min(row1 - row0, w.max_new);
    if (report) {
        if (s.len != len) report_status(w.status, AFX_ERR_CAPACITY);
        if ((w.start != nullptr && w.start[b] != row0) || row1 != hi || s.first < 0) report_status(w.status, AFX_ERR_INVALID_ARG);
        if (s.n != row1 - row0) report_status(w.status, AFX_ERR_CAPACITY);
    }
    return s;
}

// The table's entry for position p (0 <= p < cap) of sequence b as it stands there, and the place in the page.
__device__ __forceinline__ int paged_entry(const PagedView& w, int b, int p, int& in_page) {
    const int i = static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(p)) * w.mul) >> (31 + w.shift));
    in_page = p - i * w.page_size;
    return w.table[static_cast<int64_t>(b) * w.table_stride + i];
}

// The page of that position; -1 where the entry is none.
__device__ __forceinline__ int paged_page(const PagedView& w, int b, int p, int& in_page) {
    const int page = paged_entry(w, b, p, in_page);
    return static_cast<uint32_t>(page) < static_cast<uint32_t>(w.n_pages) ? page : -1;
}

// Element offset of position p's row of kv head g; -1 where it has no page.
__device__ __forceinline__ int64_t paged_row(const PagedView& w, int b, int p, int g) {
    int in_page;
    const int page = paged_page(w, b, p, in_page);
    if (page < 0) return -1;
    return page * w.page_stride + in_page * w.pos_stride + g * w.head_stride;
}

// First position of the window of a token at position p, and how many first positions stay visible before it.
__device__ __forceinline__ int paged_low(const PagedMask& m, int p) { return m.window > 0 ? max(0, p - m.window + 1) : 0; }
__device__ __forceinline__ int paged_few(const PagedMask& m, int low) { return min(m.sinks, low); }

}  // namespace afx
