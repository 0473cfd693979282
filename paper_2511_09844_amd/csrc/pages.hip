// Pages of a K/V cache: rows appended to them, pages given, shared, taken back and moved together, and
// the C entry points of everything paged that belongs to no handle.
#include <string.h>

#include <algorithm>
#include <atomic>

#include "device_common.h"
#include "paged.h"

namespace sd2 {

namespace {

// ---------------------------------------------------------------------------------------------
// Rows into pages.  A wave per row: its position and page are the same for all lanes, and the
// Hkv * hd elements of k and of v are copied 16 bytes a lane.  Bound by the bytes: a prompt batch's 301 MB in 58 us,
// 5.2 TB/s; a row of each of 16 sequences 3.9 us, a launch and two round trips.
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
    PagedView c;
    PagedRows r;
    const char *k, *v;
    int64_t k_stride, v_stride;  // bytes
    int lc;                      // 16-byte units of a head's row: a power of two, 1 << lc
};
constexpr int kAppendBlocks = 1 << 22;  // (of 256 threads: a launch may have fewer than 2^32)

__global__ __launch_bounds__(256) void k_paged_append(AppendArgs a) {
    const int lane = threadIdx.x & 63;
    // (a wave has one row, but where there are more than kAppendBlocks workgroups of them)
    for (int64_t at_row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); at_row < a.r.total_rows;
         at_row += (int64_t)gridDim.x * 4) {
        const int row = (int)at_row;
        const int b = paged_seq(a.r, row);
        int n;
        const int r0 = paged_rows(a.r, b, n);
        if (row < r0 || row >= r0 + n) continue;
        const int pos = a.r.row_pos ? a.r.row_pos[row] : paged_len(a.r, b, r0, n) - n + (row - r0);
        if (pos < 0) continue;
        const int page = paged_page(a.c, b, pos >> a.c.shift);
        if (page < 0) continue;
        const int slot = pos & ((1 << a.c.shift) - 1), unit = 16 << a.lc;
        const int64_t base = (int64_t)page * a.c.page_stride * (unit / a.c.hd);
        for (int i = lane; i < a.c.Hkv << a.lc; i += 64) {
            const int h = i >> a.lc, u = i & ((1 << a.lc) - 1);
            const int64_t at = base + (((int64_t)h << a.c.shift) + slot) * unit + 16 * u;
            const uint4 x = *(const uint4*)(a.k + row * a.k_stride + 16 * i), y = *(const uint4*)(a.v + row * a.v_stride + 16 * i);
            *(uint4*)((char*)a.c.k + at) = x;
            *(uint4*)((char*)a.c.v + at) = y;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The book-keeping.  One workgroup decides for all sequences, so that pages are given in one order
// whatever runs first; what it decides is a list that the copying kernel walks.  Latency: 5 to 9 us a call for pools
// of 64 to 240 pages, a scan of the references per 4096 pages.
// ---------------------------------------------------------------------------------------------
constexpr int kBookThreads = 1024, kBookWaves = kBookThreads / 64;

// Workspace: head: entries of the list, pages in use; src (-1: nothing to copy), dst and rows of every
// entry; need: entries that each sequence asks for, then those of the sequences before it; name: what
// each page from the number in use on is called when they have moved.
struct PageList {
    int32_t *head, *src, *dst, *rows, *need, *name;
};
size_t list_carve(const sd2_pages& p, char* base, PageList* l) {
    size_t off = 0;
    auto take = [&](size_t n) {
        int32_t* q = base ? (int32_t*)(base + off) : nullptr;
        off += (n * sizeof(int32_t) + 255) / 256 * 256;
        return q;
    };
    PageList w;
    w.head = take(2);
    w.src = take(p.n_pages);
    w.dst = take(p.n_pages);
    w.rows = take(p.n_pages);
    w.need = take(std::max(p.max_seqs, 1));
    w.name = take(p.n_pages);
    if (l) *l = w;
    return off;
}

struct BookArgs {
    int32_t *table, *refs;
    int32_t n_pages, max_pages, shift, nseq, max_seqs;
    const int32_t *first, *last, *keep;
    int32_t *granted, *live;
    bool whole;  // reserve: a sequence gets all it asks for, or nothing
    PageList l;
};

// Sum of x over the threads before this one; total: over all.
template <typename T>
__device__ T block_before(T x, T* red, T& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T inc = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T y = __shfl_up(inc, d, 64);
        if (lane >= d) inc += y;
    }
    __syncthreads();
    if (lane == 63) red[wave] = inc;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kBookWaves; ++w) {
        before += w < wave ? red[w] : 0;
        total += red[w];
    }
    return before + inc - x;
}

// What sequence b asks for at entry j of its window.
struct Want {
    int lo, hi, from, upto;  // entries [lo, hi) of the table's row; positions
};
__device__ __forceinline__ Want window(const BookArgs& a, int b) {
    Want w;
    w.from = max(a.first[b], 0);
    w.upto = max(a.last[b], 0);
    w.lo = w.from >> a.shift;
    w.hi = w.from < w.upto ? min(((w.upto - 1) >> a.shift) + 1, a.max_pages) : w.lo;
    return w;
}
__device__ __forceinline__ bool asks(const BookArgs& a, int b, int j, int& page) {
    page = a.table[(int64_t)b * a.max_pages + j];
    if ((uint32_t)page >= (uint32_t)a.n_pages) page = -1;
    return page < 0 || a.refs[page] > 1;
}

// From the entries that each sequence asks for to those of the sequences before it; returns those of all.  Pages are at
// most 2^24, so a sequence that has more than kBehind entries before it gets none, however many they are.
constexpr int kBehind = 1 << 30;
template <typename T>
__device__ int64_t entries_before(const BookArgs& a, T* red) {
    T asked = 0;
    for (int b0 = 0; b0 < a.nseq; b0 += kBookThreads) {
        const int b = b0 + threadIdx.x;
        T n;
        const T before = asked + block_before<T>(b < a.nseq ? a.l.need[b] : 0, red, n);
        if (b < a.nseq) a.l.need[b] = min(before, (T)kBehind);
        asked += n;
    }
    return asked;
}
__global__ __launch_bounds__(kBookThreads) void k_pages_reserve(BookArgs a) {
    __shared__ int red[kBookWaves];
    __shared__ int64_t sums[kBookWaves];
    __shared__ int taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int b = wave; b < a.nseq; b += kBookWaves) {
        const Want w = window(a, b);
        int n = 0;
        for (int j = w.lo + lane; j < w.hi; j += 64) {
            int page;
            n += asks(a, b, j, page);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
        if (lane == 0) a.l.need[b] = n;
    }
    __syncthreads();
    // in 64 bits where 32 may not hold them, up to 4096 times 2^26 (always in 64, it took 0.6 us more of 6)
    const int64_t asked = (int64_t)a.nseq * a.max_pages > INT32_MAX ? entries_before<int64_t>(a, sums) : entries_before<int>(a, red);
    const int want = min(asked, (int64_t)a.n_pages);
    // the first `want` free pages, ascending
    int found = 0;
    for (int p0 = 0; p0 < a.n_pages && found < want; p0 += 4 * kBookThreads) {
        const int p = p0 + 4 * tid;
        int4 f;
        int c = 0;
        int* fr = (int*)&f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fr[i] = p + i < a.n_pages && a.refs[p + i] == 0;
            c += fr[i];
        }
        int n, at = found + block_before(c, red, n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (fr[i] && at < want) a.l.dst[at++] = p + i;
        found += n;
    }
    found = min(found, want);
    __syncthreads();
    if (a.whole && found < asked) {
        // in the sequences' order, those that fit into what is left, the others passed over
        if (wave == 0) {
            int given = 0;
            for (int b0 = 0; b0 < a.nseq; b0 += 64) {
                const int b = b0 + lane;
                const int64_t behind = b + 1 < a.nseq ? a.l.need[b + 1] : min(asked, (int64_t)kBehind);
                const int mine = b < a.nseq ? (int)behind - a.l.need[b] : 0;
                int at = kBehind;
                for (int l = 0; l < 64; ++l) {
                    const int n = __builtin_amdgcn_readlane(mine, l);
                    if (n > found - given) continue;
                    if (lane == l) at = given;
                    given += n;
                }
                if (b < a.nseq) a.l.need[b] = at;
            }
            if (lane == 0) taken = given;
        }
        __syncthreads();
        found = taken;
    }
    for (int b = wave; b < a.nseq; b += kBookWaves) {
        const Want w = window(a, b);
        const int keep = a.keep ? max(a.keep[b], 0) : w.from;
        int at = a.l.need[b], bad = a.max_pages;
        for (int j0 = w.lo; j0 < w.hi; j0 += 64) {
            const int j = j0 + lane;
            int page = -1;
            const bool ask = j < w.hi && asks(a, b, j, page);
            const uint64_t m = __ballot(ask);
            const int rank = at + __popcll(m & ((1ull << lane) - 1));
            if (ask && rank < found) {
                a.l.src[rank] = page;
                a.l.rows[rank] = min(max(keep - (j << a.shift), 0), 1 << a.shift);
                a.table[(int64_t)b * a.max_pages + j] = a.l.dst[rank];
            }
            const uint64_t no = __ballot(ask && rank >= found);
            if (no) bad = min(bad, j0 + (int)__builtin_ctzll(no));
            at += __popcll(m);
        }
        if (lane == 0 && a.granted) a.granted[b] = min((int64_t)w.upto, (int64_t)bad << a.shift);
    }
    __syncthreads();  // (every reference has been read)
    for (int i = tid; i < found; i += kBookThreads) {
        a.refs[a.l.dst[i]] = 1;
        if (a.l.src[i] >= 0) atomicSub(a.refs + a.l.src[i], 1);
    }
    if (tid == 0) a.l.head[0] = found;
}

__global__ __launch_bounds__(kBookThreads) void k_pages_compact(BookArgs a) {
    __shared__ int red[kBookWaves];
    const int tid = threadIdx.x;
    int n = 0;
    for (int p = tid; p < a.n_pages; p += kBookThreads) n += a.refs[p] > 0;
    int live;
    block_before(n, red, live);
    int ns = 0, nd = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += kBookThreads) {
        const int p = p0 + tid;
        const bool used = p < a.n_pages && a.refs[p] > 0;
        const bool s = used && p >= live, d = !used && p < live;
        int ts, td;
        const int is = ns + block_before<int>(s, red, ts), id = nd + block_before<int>(d, red, td);
        if (s) a.l.src[is] = p;
        else if (p >= live && p < a.n_pages) a.l.name[p] = p;  // (an entry that names a free page keeps it)
        if (d) a.l.dst[id] = p;
        ns += ts;
        nd += td;
    }
    __syncthreads();
    for (int i = tid; i < ns; i += kBookThreads) {
        const int s = a.l.src[i], d = a.l.dst[i];
        a.l.rows[i] = 1 << a.shift;
        a.l.name[s] = d;
        a.refs[d] = a.refs[s];
        a.refs[s] = 0;
    }
    if (tid == 0) {
        a.l.head[0] = ns;
        a.l.head[1] = live;
        if (a.live) *a.live = live;
    }
}

// Bytes: 2.6 GB read and written in two calls of a long sequence take 460 us, 5.6 TB/s; 32 forked sequences' last pages
// 25 us.
// A wave per block of a listed page and array: the first rows[i] rows of the block, or a record whole.  With a table its
// entries that name a moved page are renamed as well.
struct CopyArgs {
    PageList l;
    int32_t n_arrays, shift;
    char* data[SD2_PAGE_ARRAYS];
    int32_t blocks[SD2_PAGE_ARRAYS], row_bytes[SD2_PAGE_ARRAYS];
    int32_t total_blocks;
    int32_t* table;    // null: nothing is renamed
    int64_t entries;
    int32_t n_pages;
};

__global__ __launch_bounds__(256) void k_pages_copy(CopyArgs a) {
    const int lane = threadIdx.x & 63;
    const int n = a.l.head[0];
    if (a.table && n) {
        const int live = a.l.head[1];
        const int64_t step = (int64_t)gridDim.x * 256;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.entries; i += step) {
            const int p = a.table[i];
            if (p >= live && p < a.n_pages) a.table[i] = a.l.name[p];
        }
    }
    const int64_t units = (int64_t)n * a.total_blocks, step = (int64_t)gridDim.x * 4;
    for (int64_t u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); u < units; u += step) {
        const int i = u / a.total_blocks;
        int blk = u - (int64_t)i * a.total_blocks, arr = 0;
        while (blk >= a.blocks[arr]) blk -= a.blocks[arr++];
        const int src = a.l.src[i];
        if (src < 0) continue;
        if (a.row_bytes[arr] < 0) {  // a record: whole, where anything of the page is kept
            const int bytes = a.l.rows[i] ? -a.row_bytes[arr] : 0;
            const char* s = a.data[arr] + ((int64_t)src * a.blocks[arr] + blk) * -a.row_bytes[arr];
            char* d = a.data[arr] + ((int64_t)a.l.dst[i] * a.blocks[arr] + blk) * -a.row_bytes[arr];
            if (a.row_bytes[arr] % 16 == 0)
                for (int x = 16 * lane; x < bytes; x += 1024) *(uint4*)(d + x) = *(const uint4*)(s + x);
            else
                for (int x = 2 * lane; x < bytes; x += 128) *(uint16_t*)(d + x) = *(const uint16_t*)(s + x);
            continue;
        }
        const int64_t page = (int64_t)a.row_bytes[arr] << a.shift;
        const uint4* s = (const uint4*)(a.data[arr] + ((int64_t)src * a.blocks[arr] + blk) * page);
        uint4* d = (uint4*)(a.data[arr] + ((int64_t)a.l.dst[i] * a.blocks[arr] + blk) * page);
        const int m = a.l.rows[i] * (a.row_bytes[arr] / 16);
        for (int x = lane; x < m; x += 64) d[x] = s[x];
    }
}

constexpr int kForkPairs = 64;
struct ForkArgs {
    int32_t *table, *refs;
    int32_t n_pages, max_pages;
    int32_t src[kForkPairs], dst[kForkPairs];
};
__global__ __launch_bounds__(256) void k_pages_fork(ForkArgs a) {
    const int32_t* src = a.table + (int64_t)a.src[blockIdx.x] * a.max_pages;
    int32_t* dst = a.table + (int64_t)a.dst[blockIdx.x] * a.max_pages;
    for (int j = threadIdx.x; j < a.max_pages; j += 256) {
        const int o = dst[j], p = src[j];
        if (o == p) continue;
        if ((uint32_t)o < (uint32_t)a.n_pages) atomicSub(a.refs + o, 1);
        if ((uint32_t)p < (uint32_t)a.n_pages) atomicAdd(a.refs + p, 1);
        dst[j] = p;
    }
}

__global__ __launch_bounds__(256) void k_pages_trim(int32_t* table, int32_t* refs, int n_pages, int max_pages, int shift,
                                                    const int32_t* lens) {
    const int len = lens[blockIdx.x];
    if (len < 0) return;
    int32_t* row = table + (int64_t)blockIdx.x * max_pages;
    for (int j = (len >> shift) + ((len & ((1 << shift) - 1)) != 0) + threadIdx.x; j < max_pages; j += 256) {
        const int p = row[j];
        if ((uint32_t)p < (uint32_t)n_pages) atomicSub(refs + p, 1);
        row[j] = -1;
    }
}

// Entries lo .. hi - 1 of every sequence whose positions no row at lens[b] or behind reads, and no sink is among: a
// workgroup per kSlideEntries of them, as long tables hold many that were given up before.  Latency: 4 us for 64 sequences
// of up to 1024 entries.
constexpr int kSlideEntries = 2048, kSlideGroups = 64;
__global__ __launch_bounds__(256) void k_pages_slide(int32_t* table, int32_t* refs, int n_pages, int max_pages, int shift,
                                                     const int32_t* lens, int window, int sinks, int groups) {
    const int b = blockIdx.x / groups, len = lens[b];
    if (len < 0) return;
    int32_t* row = table + (int64_t)b * max_pages;
    const int lo = (sinks + (1 << shift) - 1) >> shift, hi = min((int)max((int64_t)len - window + 1, (int64_t)0) >> shift, max_pages);
    for (int j = lo + blockIdx.x % groups * 256 + threadIdx.x; j < hi; j += groups * 256) {
        const int p = row[j];
        if ((uint32_t)p < (uint32_t)n_pages) atomicSub(refs + p, 1);
        row[j] = -1;
    }
}

int shift_of(int page_size) {
    for (int s = 4; s <= 10; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}

// Bytes of a record (an array without rows) at most.
constexpr int32_t kRecordBytes = 1 << 20;

bool aligned(const void* p, size_t n) { return p && (uintptr_t)p % n == 0; }

BookArgs book(const sd2_pages& p, void* ws) {
    BookArgs a{};
    a.table = p.table; a.refs = p.refs; a.n_pages = p.n_pages; a.max_pages = p.max_pages;
    a.shift = shift_of(p.page_size); a.max_seqs = p.max_seqs;
    list_carve(p, (char*)ws, &a.l);
    return a;
}

hipError_t copy_listed(hipStream_t s, const sd2_pages& p, const PageList& l, bool rename) {
    CopyArgs c{};
    c.l = l;
    c.n_arrays = p.n_arrays;
    c.shift = shift_of(p.page_size);
    for (int i = 0; i < p.n_arrays; ++i) {
        c.data[i] = (char*)p.arrays[i].data;
        c.blocks[i] = p.arrays[i].blocks;
        c.row_bytes[i] = p.arrays[i].row_bytes;
        c.total_blocks += p.arrays[i].blocks;
    }
    c.table = rename ? p.table : nullptr;
    c.entries = (int64_t)p.max_seqs * p.max_pages;
    c.n_pages = p.n_pages;
    return launch(k_pages_copy, dim3(1024), dim3(256), s, c);
}

}  // namespace

bool pages_ok(const sd2_pages* p) {
    if (!p || shift_of(p->page_size) < 0 || p->n_pages < 1 || p->n_pages > 1 << 24 || p->max_seqs < 1 ||
        p->max_seqs > SD2_PAGED_MAX_SEQS || p->max_pages < 1 || (int64_t)p->max_pages * p->page_size > 1 << 30 ||
        !aligned(p->table, 4) || !aligned(p->refs, 4) || p->n_arrays < 1 || p->n_arrays > SD2_PAGE_ARRAYS)
        return false;
    for (int i = 0; i < p->n_arrays; ++i) {
        const sd2_page_array& a = p->arrays[i];
        if (!aligned(a.data, 16) || a.blocks < 1 || a.blocks > 65536) return false;
        if (a.row_bytes < 0 ? a.row_bytes < -kRecordBytes || a.row_bytes % 2 : a.row_bytes < 16 || a.row_bytes > 65536 || a.row_bytes % 16)
            return false;
    }
    return true;
}

size_t pages_bytes(const sd2_pages& p) { return list_carve(p, nullptr, nullptr); }

hipError_t pages_reserve(hipStream_t s, const sd2_pages& p, int nseq, const int32_t* first, const int32_t* last,
                         const int32_t* keep, int32_t* granted, void* ws, bool whole) {
    BookArgs a = book(p, ws);
    a.nseq = nseq; a.first = first; a.last = last; a.keep = keep; a.granted = granted; a.whole = whole;
    const hipError_t err = launch(k_pages_reserve, dim3(1), dim3(kBookThreads), s, a);
    return err != hipSuccess ? err : copy_listed(s, p, a.l, false);
}

hipError_t pages_fork(hipStream_t s, const sd2_pages& p, int n, const int32_t* src, const int32_t* dst) {
    ForkArgs a{};
    a.table = p.table; a.refs = p.refs; a.n_pages = p.n_pages; a.max_pages = p.max_pages;
    for (int i = 0; i < n; i += kForkPairs) {
        const int m = std::min(kForkPairs, n - i);
        memcpy(a.src, src + i, sizeof(int32_t) * m);
        memcpy(a.dst, dst + i, sizeof(int32_t) * m);
        const hipError_t err = launch(k_pages_fork, dim3(m), dim3(256), s, a);
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t pages_trim(hipStream_t s, const sd2_pages& p, int nseq, const int32_t* lens) {
    return launch(k_pages_trim, dim3(nseq), dim3(256), s, p.table, p.refs, (int)p.n_pages, (int)p.max_pages,
                  shift_of(p.page_size), lens);
}

hipError_t pages_slide(hipStream_t s, const sd2_pages& p, int nseq, const int32_t* lens, int window, int sinks) {
    const int groups = std::min((p.max_pages + kSlideEntries - 1) / kSlideEntries, kSlideGroups);
    return launch(k_pages_slide, dim3(nseq * groups), dim3(256), s, p.table, p.refs, (int)p.n_pages, (int)p.max_pages,
                  shift_of(p.page_size), lens, window, sinks, groups);
}

hipError_t pages_compact(hipStream_t s, const sd2_pages& p, int32_t* live, void* ws) {
    BookArgs a = book(p, ws);
    a.live = live;
    const hipError_t err = launch(k_pages_compact, dim3(1), dim3(kBookThreads), s, a);
    return err != hipSuccess ? err : copy_listed(s, p, a.l, true);
}

hipError_t paged_append(hipStream_t s, const PagedView& c, const PagedRows& r, const void* k, int64_t k_stride,
                        const void* v, int64_t v_stride, int size) {
    if (!r.total_rows || !r.nseq) return hipSuccess;
    AppendArgs a{c, r, (const char*)k, (const char*)v, k_stride * size, v_stride * size, 0};
    while (16 << a.lc < c.hd * size) ++a.lc;
    return launch(k_paged_append, dim3((unsigned)std::min<int64_t>(((int64_t)r.total_rows + 3) / 4, kAppendBlocks)), dim3(256), s, a);
}

namespace {

// The kernels are built for gfx950 with XNACK off (see sd2_create); asked once per device.
sd2_status device_ok() {
    static std::atomic<int8_t> known[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return SD2_ERR_HIP;
    if (dev >= 0 && dev < 64 && known[dev].load(std::memory_order_relaxed)) return SD2_OK;
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return SD2_ERR_HIP;
    if (strncmp(prop.gcnArchName, "gfx950", 6) != 0 || strstr(prop.gcnArchName, "xnack+") != nullptr)
        return SD2_ERR_UNSUPPORTED;
    if (dev >= 0 && dev < 64) known[dev].store(1, std::memory_order_relaxed);
    return SD2_OK;
}

sd2_status status_of(hipError_t err) { return err == hipSuccess ? SD2_OK : SD2_ERR_HIP; }

// held: bytes of an element of the cache, where they are not the rows' (0)
bool view_of(const sd2_paged_kv* kv, PagedView* c, int* size, int held = 0) {
    if (!kv || (kv->dtype != SD2_F32 && kv->dtype != SD2_BF16)) return false;
    *size = kv->dtype == SD2_BF16 ? 2 : 4;
    if (!held) held = *size;
    const int shift = shift_of(kv->page_size);
    if (shift < 0 || kv->n_pages < 1 || kv->n_pages > 1 << 24 || kv->n_kv_heads < 1 || kv->n_kv_heads > 1024 ||
        (kv->head_dim != 32 && kv->head_dim != 64 && kv->head_dim != 128) || kv->max_pages < 1 ||
        (int64_t)kv->max_pages * kv->page_size > 1 << 30 || !aligned(kv->k, 16) || !aligned(kv->v, 16) ||
        !aligned(kv->table, 4))
        return false;
    if (kv->page_stride < (int64_t)kv->n_kv_heads * kv->page_size * kv->head_dim || kv->page_stride % (16 / held) ||
        kv->page_stride > (int64_t)1 << 40)
        return false;
    *c = PagedView{kv->k, kv->v, kv->page_stride, kv->n_pages, shift, kv->n_kv_heads, kv->head_dim, kv->table, kv->max_pages, nullptr, 0};
    return true;
}
bool view_of(const sd2_paged_scaled* kv, PagedView* c, int* size) {
    if (!kv || !view_of(&kv->kv, c, size, 1) || !aligned(kv->scales, 2) || kv->scale_stride % 2 ||
        kv->scale_stride < (int64_t)c->Hkv << (c->shift - 3) || kv->scale_stride > (int64_t)1 << 40)
        return false;
    c->scales = (uint8_t*)kv->scales;
    c->scale_stride = kv->scale_stride;
    return true;
}

bool rows_of(const sd2_paged_rows* rows, PagedRows* r) {
    if (!rows || rows->nseq < 0 || rows->nseq > SD2_PAGED_MAX_SEQS || rows->max_rows < 1 || rows->total_rows < 0)
        return false;
    if (rows->nseq && !aligned(rows->lens, 4)) return false;
    if (rows->row_off ? !aligned(rows->row_off, 4) : (int64_t)rows->nseq * rows->max_rows != rows->total_rows) return false;
    const int32_t most = std::min(rows->max_rows, std::max(rows->total_rows, 1));
    *r = PagedRows{rows->nseq, most, rows->total_rows, rows->row_off, rows->lens, nullptr};
    return true;
}

// A row-major operand of rows of `width` elements.
bool strided(const void* p, int64_t stride, int64_t width, int size) {
    return aligned(p, 16) && stride >= width && stride % (16 / size) == 0 && stride <= (int64_t)1 << 40;
}

// Whether two such operands of n rows share an element.  Rows of one stride may lie in one another's gaps; of others
// it is enough that their extents meet.
bool overlap(const void* p, int64_t ps, const void* q, int64_t qs, int64_t n, int64_t width, int size) {
    const __int128 d = ((__int128)(uintptr_t)q - (__int128)(uintptr_t)p) / size;  // (16-byte aligned)
    if (d >= (n - 1) * (__int128)ps + width || -d >= (n - 1) * (__int128)qs + width) return false;
    if (ps != qs || n == 1) return true;
    const int64_t gap = (int64_t)((d % ps + ps) % ps);
    return gap < width || gap > ps - width;
}

constexpr int32_t kMostPositions = 1 << 30;

// The attention calls, of either kind of cache.
template <typename KV>
size_t attn_bytes(const KV* kv, const sd2_paged_rows* rows, int32_t n_heads, int32_t max_len, int32_t window, int32_t sinks) {
    PagedView c;
    PagedRows r;
    int size;
    if (!view_of(kv, &c, &size) || !rows_of(rows, &r) || n_heads < 1 || n_heads > 1024 || n_heads % c.Hkv) return 0;
    if ((int64_t)r.max_rows * (n_heads / c.Hkv) > 1 << 30) return 0;
    if (max_len < 1 || max_len > (int64_t)c.max_pages << c.shift) return 0;
    if (window < 0 || window > kMostPositions || sinks < 0 || sinks > kMostPositions) return 0;
    return paged_attn_bytes(c, r, n_heads, size == 2, max_len, window, sinks);
}
template <typename KV>
sd2_status attn_call(const KV* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                     int32_t n_heads, float scale, int32_t max_len, int32_t window, int32_t sinks, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
    PagedAttnArgs a{};
    int size;
    if (!view_of(kv, &a.c, &size) || !rows_of(rows, &a.r)) return SD2_ERR_INVALID_ARG;
    if (n_heads < 1 || n_heads > 1024 || n_heads % a.c.Hkv || !(scale >= -1e30f && scale <= 1e30f)) return SD2_ERR_INVALID_ARG;
    if (max_len < 1 || max_len > (int64_t)a.c.max_pages << a.c.shift) return SD2_ERR_INVALID_ARG;
    if (window < 0 || window > kMostPositions || sinks < 0 || sinks > kMostPositions) return SD2_ERR_INVALID_ARG;
    if ((int64_t)a.r.max_rows * (n_heads / a.c.Hkv) > 1 << 30) return SD2_ERR_INVALID_ARG;
    if (!a.r.nseq || !a.r.total_rows) return SD2_OK;
    const int64_t width = (int64_t)n_heads * a.c.hd;
    if (!strided(q, q_stride, width, size) || !strided(out, out_stride, width, size) ||
        overlap(q, q_stride, out, out_stride, a.r.total_rows, width, size))
        return SD2_ERR_INVALID_ARG;
    const size_t need = paged_attn_bytes(a.c, a.r, n_heads, size == 2, max_len, window, sinks);
    if (!need || !aligned(workspace, 256) || workspace_bytes < need) return SD2_ERR_INVALID_ARG;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride; a.H = n_heads; a.scale = scale;
    a.window = window; a.sinks = sinks;
    return status_of(paged_attn((hipStream_t)hip_stream, a, size == 2, max_len, workspace, workspace_bytes));
}

}  // namespace

}  // namespace sd2

using namespace sd2;

extern "C" {

size_t sd2_pages_workspace_bytes(const sd2_pages* pages) { return pages_ok(pages) ? pages_bytes(*pages) : 0; }

sd2_status sd2_pages_reserve(const sd2_pages* pages, int32_t nseq, const int32_t* first, const int32_t* last,
                             const int32_t* keep, int32_t* granted, void* workspace, size_t workspace_bytes,
                             void* hip_stream) {
    if (!pages_ok(pages) || nseq < 0 || nseq > pages->max_seqs) return SD2_ERR_INVALID_ARG;
    if (nseq && (!aligned(first, 4) || !aligned(last, 4))) return SD2_ERR_INVALID_ARG;
    if (!aligned(workspace, 256) || workspace_bytes < pages_bytes(*pages)) return SD2_ERR_INVALID_ARG;
    if (!nseq) return SD2_OK;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(pages_reserve((hipStream_t)hip_stream, *pages, nseq, first, last, keep, granted, workspace));
}

sd2_status sd2_pages_fork(const sd2_pages* pages, int32_t n, const int32_t* src, const int32_t* dst, void* hip_stream) {
    if (!pages_ok(pages) || n < 0 || n > pages->max_seqs || (n && (!src || !dst))) return SD2_ERR_INVALID_ARG;
    uint64_t taken[SD2_PAGED_MAX_SEQS / 64] = {};
    for (int i = 0; i < n; ++i) {
        if (src[i] < 0 || src[i] >= pages->max_seqs || dst[i] < 0 || dst[i] >= pages->max_seqs) return SD2_ERR_INVALID_ARG;
        if (taken[dst[i] / 64] >> (dst[i] % 64) & 1) return SD2_ERR_INVALID_ARG;
        taken[dst[i] / 64] |= (uint64_t)1 << (dst[i] % 64);
    }
    for (int i = 0; i < n; ++i)
        if (taken[src[i] / 64] >> (src[i] % 64) & 1) return SD2_ERR_INVALID_ARG;
    if (!n) return SD2_OK;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(pages_fork((hipStream_t)hip_stream, *pages, n, src, dst));
}

sd2_status sd2_pages_trim(const sd2_pages* pages, int32_t nseq, const int32_t* lens, void* hip_stream) {
    if (!pages_ok(pages) || nseq < 0 || nseq > pages->max_seqs || (nseq && !aligned(lens, 4))) return SD2_ERR_INVALID_ARG;
    if (!nseq) return SD2_OK;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(pages_trim((hipStream_t)hip_stream, *pages, nseq, lens));
}

sd2_status sd2_pages_compact(const sd2_pages* pages, int32_t* live, void* workspace, size_t workspace_bytes,
                             void* hip_stream) {
    if (!pages_ok(pages) || !aligned(workspace, 256) || workspace_bytes < pages_bytes(*pages)) return SD2_ERR_INVALID_ARG;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(pages_compact((hipStream_t)hip_stream, *pages, live, workspace));
}

sd2_status sd2_paged_append(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride, void* hip_stream) {
    PagedView c;
    PagedRows r;
    int size;
    if (!view_of(kv, &c, &size) || !rows_of(rows, &r)) return SD2_ERR_INVALID_ARG;
    if (!r.nseq || !r.total_rows) return SD2_OK;
    const int64_t width = (int64_t)c.Hkv * c.hd;
    if (!strided(k, k_stride, width, size) || !strided(v, v_stride, width, size)) return SD2_ERR_INVALID_ARG;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(paged_append((hipStream_t)hip_stream, c, r, k, k_stride, v, v_stride, size));
}

size_t sd2_paged_attn_workspace_bytes(const sd2_paged_kv* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                      int32_t max_len) {
    return attn_bytes(kv, rows, n_heads, max_len, 0, 0);
}
sd2_status sd2_paged_attn(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                          void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attn_call(kv, rows, q, q_stride, out, out_stride, n_heads, scale, max_len, 0, 0, workspace, workspace_bytes, hip_stream);
}

size_t sd2_paged_attn_window_workspace_bytes(const sd2_paged_kv* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                             int32_t max_len, int32_t window, int32_t sinks) {
    return attn_bytes(kv, rows, n_heads, max_len, window, sinks);
}
sd2_status sd2_paged_attn_window(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                                 void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                                 int32_t window, int32_t sinks, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attn_call(kv, rows, q, q_stride, out, out_stride, n_heads, scale, max_len, window, sinks, workspace, workspace_bytes, hip_stream);
}

size_t sd2_paged_attn_scaled_workspace_bytes(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                       int32_t max_len, int32_t window, int32_t sinks) {
    return attn_bytes(kv, rows, n_heads, max_len, window, sinks);
}
sd2_status sd2_paged_attn_scaled(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                           void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                           int32_t window, int32_t sinks, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attn_call(kv, rows, q, q_stride, out, out_stride, n_heads, scale, max_len, window, sinks, workspace, workspace_bytes, hip_stream);
}

sd2_status sd2_paged_append_scaled(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, void* hip_stream) {
    PagedView c;
    PagedRows r;
    int size;
    if (!view_of(kv, &c, &size) || !rows_of(rows, &r)) return SD2_ERR_INVALID_ARG;
    if (!r.nseq || !r.total_rows) return SD2_OK;
    const int64_t width = (int64_t)c.Hkv * c.hd;
    if (!strided(k, k_stride, width, size) || !strided(v, v_stride, width, size)) return SD2_ERR_INVALID_ARG;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(paged_append8((hipStream_t)hip_stream, c, r, k, k_stride, v, v_stride, size == 2));
}

sd2_status sd2_pages_slide(const sd2_pages* pages, int32_t nseq, const int32_t* lens, int32_t window, int32_t sinks,
                           void* hip_stream) {
    if (!pages_ok(pages) || nseq < 0 || nseq > pages->max_seqs || (nseq && !aligned(lens, 4))) return SD2_ERR_INVALID_ARG;
    if (window < 1 || window > kMostPositions || sinks < 0 || sinks > kMostPositions) return SD2_ERR_INVALID_ARG;
    if (!nseq) return SD2_OK;
    const sd2_status st = device_ok();
    if (st != SD2_OK) return st;
    return status_of(pages_slide((hipStream_t)hip_stream, *pages, nseq, lens, window, sinks));
}

}  // extern "C"
