// The prompts' attention built with a limit of its waits that a test sets (test_gpu_paged_waits.py).
// Rows that are taken again say so after tell_every positions: never, unless the test says otherwise.
static __device__ unsigned long long limit_ns;
static __device__ int tell_every = 0x7FFFFFFF;
#define AFX_WAIT_NS limit_ns
#define AFX_TELL_EVERY tell_every
#include "afx_paged_prompt.cu"
#include "afx_paged.cu"

int afx::sm_count() {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

extern "C" int waits_limit(unsigned long long ns) { return static_cast<int>(cudaMemcpyToSymbol(limit_ns, &ns, sizeof ns)); }

extern "C" int waits_tell_every(int positions) { return static_cast<int>(cudaMemcpyToSymbol(tell_every, &positions, sizeof positions)); }

// afx_paged_attn of every sequence by tiles, out in the cache's type
extern "C" int waits_prompt(const afx_paged_kv* kv, const void* q, int64_t ldq, int n_heads, void* out, float* lse, int32_t* dev_status) {
    afx::PagedAttnArgs a = {};
    const afx_status rc = afx::paged_view(kv, dev_status, &a.w);
    if (rc != AFX_OK) return rc;
    a.heads = n_heads;
    a.rep = n_heads / kv->n_kv_heads;
    a.q = static_cast<const char*>(q);
    a.ldq = ldq;
    a.q_type = a.out_type = kv->dtype;
    a.scale = 1.4426950408889634f / sqrtf(static_cast<float>(kv->head_dim));
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    return afx::launch_paged_prompt(kv->dtype, kv->head_dim, a, 0, nullptr);
}
