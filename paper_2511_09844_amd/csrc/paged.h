// Paged K/V caches: what the kernels of paged_attn.hip and pages.hip take, for the C entry points and
// for handles created by sd2_create_paged.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sd2.h"

namespace sd2 {

// Where the rows of a paged cache lie: page p's row of KV head h and slot s starts at element
// p * page_stride + (h * page_size + s) * head_dim of k and of v.
struct PagedView {
    void *k, *v;
    int64_t page_stride;
    int32_t n_pages, shift, Hkv, hd;  // page_size = 1 << shift
    const int32_t* table;             // [nseq][max_pages]; an entry outside 0 .. n_pages - 1: no page
    int32_t max_pages;
};

// The rows a call brings: sequence b has rows row_off[b] .. row_off[b + 1] - 1 (at most max_rows of
// them), or max_rows rows each when row_off is null; they are the last ones of lens[b] positions.
struct PagedRows {
    int32_t nseq, max_rows, total_rows;
    const int32_t* row_off;
    const int32_t* lens;     // or null: one more than the position of the sequence's last row
    const int32_t* row_pos;  // (lens null) [total_rows]; paged_append leaves out rows at -1
};

struct PagedAttnArgs {
    PagedView c;
    PagedRows r;
    const void* q;
    void* out;
    int64_t q_stride, out_stride;  // elements between rows
    uint16_t* planes;              // fp32: output as planes of Mp rows (see pgemm.hip), in place of out; or null
    int32_t Mp;
    int32_t H;
    float scale;
};

// Workspace of a call (0: more than can be launched), and the call.  max_len: the largest length expected.  bf16: of
// q, the cache and out (else fp32).
size_t paged_attn_bytes(const PagedView& c, const PagedRows& r, int H, bool bf16, int64_t max_len);
// With less than that the keys are split less.
hipError_t paged_attn(hipStream_t s, const PagedAttnArgs& a, bool bf16, int64_t max_len, void* ws, size_t ws_bytes);

// k, v rows [total_rows][Hkv][hd] (row strides in elements) into their pages; size: bytes of an element.
hipError_t paged_append(hipStream_t s, const PagedView& c, const PagedRows& r, const void* k, int64_t k_stride,
                        const void* v, int64_t v_stride, int size);

bool pages_ok(const sd2_pages* p);
size_t pages_bytes(const sd2_pages& p);
// whole: a sequence that the pool cannot give every page it asks for gets none of them, and those behind it are
// served all the same.
hipError_t pages_reserve(hipStream_t s, const sd2_pages& p, int nseq, const int32_t* first, const int32_t* last,
                         const int32_t* keep, int32_t* granted, void* ws, bool whole = false);
hipError_t pages_fork(hipStream_t s, const sd2_pages& p, int n, const int32_t* src, const int32_t* dst);
hipError_t pages_trim(hipStream_t s, const sd2_pages& p, int nseq, const int32_t* lens);
hipError_t pages_compact(hipStream_t s, const sd2_pages& p, int32_t* live, void* ws);

// A kernel launch whose error is returned and not left behind.
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s, A... args) {
    void* ptrs[] = {(void*)&args...};
    static_assert(sizeof...(P) == sizeof...(A) && (std::is_same_v<P, A> && ...), "the kernel's own argument types");
    return hipLaunchKernel((const void*)kernel, grid, block, ptrs, 0, s);
}

#ifdef __HIPCC__
// First row and number of rows of sequence b, within 0 .. total_rows whatever row_off holds.
__device__ __forceinline__ int paged_rows(const PagedRows& r, int b, int& n) {
    if (!r.row_off) {
        n = r.max_rows;
        return b * r.max_rows;
    }
    const int r0 = min(max(r.row_off[b], 0), r.total_rows), r1 = min(max(r.row_off[b + 1], r0), r.total_rows);
    n = min(r1 - r0, r.max_rows);
    return r0;
}
// Positions of sequence b whose rows are r0 .. r0 + n - 1.
__device__ __forceinline__ int paged_len(const PagedRows& r, int b, int r0, int n) {
    return max(r.lens ? r.lens[b] : n > 0 ? r.row_pos[r0 + n - 1] + 1 : 0, 0);
}
// Both, loaded at once.
struct SeqRows {
    int r0, n, len;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedRows& r, int b) {
    SeqRows s;
    const int len = r.lens ? r.lens[b] : 0;
    s.r0 = paged_rows(r, b, s.n);
    s.len = r.lens ? max(len, 0) : paged_len(r, b, s.r0, s.n);
    return s;
}
// Those that lane l holds, for all lanes.
__device__ __forceinline__ SeqRows lane_rows(const SeqRows& s, int l) {
    return SeqRows{__builtin_amdgcn_readlane(s.r0, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.len, l)};
}
// The sequence that row `row` belongs to, or -1 (rows behind the last one's).
__device__ __forceinline__ int paged_seq(const PagedRows& r, int row) {
    if (!r.row_off) return row / r.max_rows;
    int lo = 0, hi = r.nseq;  // the last b with row_off[b] <= row, if row_off ascends as it has to
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (r.row_off[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}
// Page of entry j of sequence b, or -1.
__device__ __forceinline__ int paged_page(const PagedView& c, int b, int j) {
    if (j < 0 || j >= c.max_pages) return -1;
    const int p = c.table[(int64_t)b * c.max_pages + j];
    return (uint32_t)p < (uint32_t)c.n_pages ? p : -1;
}
#endif

}  // namespace sd2
