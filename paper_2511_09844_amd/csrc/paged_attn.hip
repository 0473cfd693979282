// Causal grouped-query attention over a paged K/V cache.
//
// For few rows per sequence (decoding, speculative blocks): k_pdecode.  A query vector is a (row, head)
// pair; those of one sequence and KV head read the same keys, so they are the 16 columns of a matrix
// instruction (NT times 16 of them per wave), and both products are computed transposed,
//   S^T = K Q^T   (16 keys x 16 query vectors)
//   O^T += V^T P^T (16 columns of v x 16 query vectors, HD / 16 of them),
// with the contraction index of the second one numbered as the result of the first lies in the
// registers: lane group g holds keys 4 g + r of every 16.  So a lane holds one query vector's scores,
// its running maximum and its part of the sums, the softmax needs one exchange over the four lane groups
// per block of keys, and neither the weights nor K and V go through LDS: a lane loads rows of K and V
// straight from the pages as operands.  bf16 V needs its columns' values of eight keys in one
// register set: a lane loads HD / 16 neighbouring columns of its eight keys and permutes bytes.
//
// A page is looked up once per 16 keys (pages are multiples of 16 positions) and all lanes' loads of
// those keys go through one buffer descriptor, whose size says how many of the 16 rows exist: rows behind
// the last position and pages that are missing read as zeros, whatever lies there, and nothing
// outside a page is ever addressed.
//
// Few rows are bound by the bytes of K and V: on MI355X one token of 16 fp32 sequences (152 MB) takes 37 us with
// its join, one of a bf16 batch of 905 MB 165 (5.5 TB/s), eight rows of 16 fp32 sequences 50 (155 MB, and
// 16 us of fp32 matrix instructions that overlap with the loads in part); one short sequence is
// bound by round trips to memory in a row, 7.1 us.  Prompts are bound by the matrix cores, see k_pprompt_bf16.
#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "paged.h"
#include "pgemm.h"

namespace sd2 {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;

// Maximum and sum over the four 16-lane groups of a wave (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float col_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float col_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sum over a wave.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_total(int v) {
    v = dpp_add<0xB1, 0xf>(v);   // quad_perm [1,0,3,2]
    v = dpp_add<0x4E, 0xf>(v);   // quad_perm [2,3,0,1]
    v = dpp_add<0x141, 0xf>(v);  // row_half_mirror
    v = dpp_add<0x140, 0xf>(v);  // row_mirror
    v = dpp_add<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
    v = dpp_add<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
    return __builtin_amdgcn_readlane(v, 63);
}
// Maximum over a wave of values that are not negative.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_max(int v) {
    return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int wave_most(int v) {
    v = dpp_max<0x142, 0xa>(dpp_max<0x140, 0xf>(dpp_max<0x141, 0xf>(dpp_max<0x4E, 0xf>(dpp_max<0xB1, 0xf>(v)))));
    return __builtin_amdgcn_readlane(dpp_max<0x143, 0xc>(v), 63);
}

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    const f2 v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}

// A value that is the same in all lanes, in scalar registers (the compiler does not see it of one that
// was loaded through vector memory).
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// n neighbouring output values of a row (n columns from c, a multiple of n).
template <typename T, int N>
__device__ __forceinline__ void put(const PagedAttnArgs& a, int row, int c, const float* v) {
    if constexpr (sizeof(T) == 2) {
        uint16_t* p = (uint16_t*)a.out + row * a.out_stride + c;
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 8)
                *(u4*)(p + i) = u4{pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3]), pack_bf16(v[i + 4], v[i + 5]),
                                   pack_bf16(v[i + 6], v[i + 7])};
        } else {
            static_assert(N == 4);
            *(u2*)p = u2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 x = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            if (a.planes) pg_put4(a.planes, a.Mp, row, c + i, x);
            else *(float4*)((float*)a.out + row * a.out_stride + c + i) = x;
        }
    }
}

// What a row's sums are multiplied by.  A sum of weights of 0 is that of a row that reads nothing, which gives zeros, or
// of one whose every score is -inf, which gives NaN; only such waves look which it is, in the table: at the first
// position that has a page, up to `upto`.  For whole waves, of one sequence.
__device__ __forceinline__ float inverse(const PagedView& c, int b, float sum, int pos, int upto) {
    const float inv = 1.f / sum;
    if (!__any(!(sum > 0.f))) return inv;
    const int lane = threadIdx.x & 63, n = min((upto >> c.shift) + 1, c.max_pages);
    int first = INT32_MAX;
    for (int j = 0; j < n; j += 64) {
        const uint64_t there = __ballot(j + lane < n && paged_page(c, b, j + lane) >= 0);
        if (there) {
            first = (j + (int)__builtin_ctzll(there)) << c.shift;
            break;
        }
    }
    return sum > 0.f ? inv : pos < first ? 0.f : NAN;
}

// The keys a workgroup of k_pdecode takes at a time, 16 or 32 per wave.
template <typename T>
constexpr int kBlockKeys = sizeof(T) == 2 ? 32 : 16;
// Waves of a workgroup: with 8 the one-token calls of 16 fp32 sequences take 42.5 us, not 36.5, and blocks of eight
// rows 57, not 49 (larger units, and one more join of the waves' sums).
constexpr int kDecodeWaves = 4;

struct DecodeArgs {
    PagedAttnArgs a;
    int ncg;       // groups of 16 NT query vectors of a sequence and KV head, at most
    int target;    // units that the sequences are to come to (see units_of); 0: one each
    int min_keys;  // of a unit
    int units;     // units there may be
    float* part;   // partials: [unit][KV head][cg] of [16 NT][HD] sums, then of [16 NT] (maximum, sum)
    int64_t ml;    // floats of the first
};

// How the keys are dealt out.  A unit is up to `keys` positions of one sequence, the same number for all, so
// that workgroups (a unit, KV head and group of query vectors each) get equal work however the
// lengths differ; it follows from the lengths on the device, which a captured call does not know
// when it is recorded.  Sequence b has the units from first[b] on.  keys is at least the total over
// target, so that there are at most target + nseq units.
struct Units {
    int keys, b, first, count;  // of sequence b: its units
    SeqRows rows;
};

// Positions of a sequence that pages may hold, 0 without rows.
__device__ __forceinline__ int seq_end(const PagedAttnArgs& a, const SeqRows& s) {
    return s.n > 0 ? (int)min((int64_t)s.len, (int64_t)a.c.max_pages << a.c.shift) : 0;
}

// The sequence that unit `unit` belongs to (b = -1: none), or sequence `b` itself when unit is negative.
template <typename T>
__device__ __forceinline__ Units units_of(const DecodeArgs& d, int unit, int b) {
    constexpr int step = kDecodeWaves * kBlockKeys<T>;
    const PagedAttnArgs& a = d.a;
    Units u;
    if (!d.target) {
        u.b = unit < 0 ? b : unit < a.r.nseq ? unit : -1;
        u.first = u.b;
        u.count = 1;
        u.rows = u.b >= 0 ? seq_rows(a.r, u.b) : SeqRows{};
        u.keys = INT32_MAX;
        return u;
    }
    const int lane = threadIdx.x & 63, nseq = a.r.nseq;
    SeqRows mine = lane < nseq ? seq_rows(a.r, lane) : SeqRows{};
    float total = (float)seq_end(a, mine);
    for (int b0 = 64; b0 < nseq; b0 += 64) total += b0 + lane < nseq ? (float)seq_end(a, seq_rows(a.r, b0 + lane)) : 0.f;
    total = wave_sum_dpp(total);
    // (rounded up past what the sum may have lost)
    const float want = fmaxf(total / (float)d.target * 1.00001f, (float)d.min_keys);
    u.keys = want < 1.0e9f ? ((int)want + step) / step * step : 1 << 30;
    u.b = -1;
    int at = 0;
    for (int b0 = 0; b0 < nseq; b0 += 64) {
        if (b0) mine = b0 + lane < nseq ? seq_rows(a.r, b0 + lane) : SeqRows{};
        const int cnt = b0 + lane < nseq ? max((seq_end(a, mine) + (u.keys - 1)) / u.keys, 1) : 0;
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int y = __shfl_up(inc, o, 64);
            if (lane >= o) inc += y;
        }
        const uint64_t here = unit < 0 ? (b >= b0 && b < b0 + 64 ? (uint64_t)1 << (b - b0) : 0) : __ballot(unit < at + inc);
        if (here) {
            const int l = __builtin_ctzll(here);
            u.b = b0 + l;
            u.first = at + __builtin_amdgcn_readlane(inc - cnt, l);
            u.count = __builtin_amdgcn_readlane(cnt, l);
            u.rows = lane_rows(mine, l);
            break;
        }
        at += __builtin_amdgcn_readlane(inc, 63);
    }
    return u;
}

// One block of keys in registers, as loaded.
template <typename T, int HD>
struct Block {
    static constexpr bool H = sizeof(T) == 2;
    static constexpr int TK = H ? 2 : 1;              // tiles of 16 keys
    static constexpr int NK = H ? HD / 32 : HD / 16;  // 16-byte loads of a row of K per lane
    static constexpr int VW = H ? HD / 16 : HD / 16 < 4 ? HD / 16 : 4;  // neighbouring columns of V per lane
    static constexpr int VU = HD / 16 / VW;
    static constexpr int VD = VW * sizeof(T) / 4;     // dwords of them
    typedef uint32_t vv __attribute__((ext_vector_type(VD)));
    u4 k[TK][NK];
    vv v[TK * 4][VU];
};

// Which of a block's operands.
enum { kLoadK = 1, kLoadV = 2 };
template <typename T, int HD, int WHAT>
__device__ __forceinline__ void load_block(Block<T, HD>& x, const PagedView& c, int kvh, const int* page, int k0, int end,
                                           int lane) {
    using B = Block<T, HD>;
    constexpr int RB = HD * sizeof(T);
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < B::TK; ++t) {
        const int key = k0 + 16 * t;
        const int rows = uniform(page[t] < 0 ? 0 : max(min(end - key, 16), 0));
        const int64_t at = uniform((int64_t)max(page[t], 0) * c.page_stride +
                                   (((int64_t)kvh << c.shift) + (key & ((1 << c.shift) - 1))) * HD);
        if constexpr (WHAT & kLoadK) {
            const auto rk = __builtin_amdgcn_make_buffer_rsrc((T*)c.k + at, 0, rows * RB, 0x00020000);
#pragma unroll
            for (int i = 0; i < B::NK; ++i)
                x.k[t][i] = __builtin_amdgcn_raw_buffer_load_b128(rk, n * RB + 16 * g + 64 * i, 0, 0);
        }
        if constexpr (WHAT & kLoadV) {
            const auto rv = __builtin_amdgcn_make_buffer_rsrc((T*)c.v + at, 0, rows * RB, 0x00020000);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int u = 0; u < B::VU; ++u) {
                    const int off = (4 * g + r) * RB + (u * 16 + n) * B::VW * (int)sizeof(T);
                    if constexpr (B::VD == 4) x.v[4 * t + r][u] = __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0);
                    else if constexpr (B::VD == 2) x.v[4 * t + r][u] = __builtin_amdgcn_raw_buffer_load_b64(rv, off, 0, 0);
                    else x.v[4 * t + r][u] = __builtin_amdgcn_raw_buffer_load_b32(rv, off, 0, 0);
                }
        }
    }
}

template <typename T, int HD, int NT>
struct Acc {
    f4 o[NT][HD / 16];
    float m[NT], l[NT];
};

// Infinities and NaN of v.  A row that does not read a key multiplies the key's values by a weight of 0, which
// would make NaN of them.  So where rows of a block differ in what they read, such values are looked for; a
// block with any is multiplied once per position that rows end at, with the values behind it as 0, and only the
// rows that end there take the product.
template <typename T>
__device__ __forceinline__ uint32_t odd_bits(uint32_t x) {  // the sign bit of such a value set
    return sizeof(T) == 2 ? (x & 0x7f807f80) + 0x00800080 : (x & 0x7f800000) + 0x00800000;
}
template <typename T>
__device__ __forceinline__ bool any_odd(uint32_t bits) {
    return __any((bits & (sizeof(T) == 2 ? 0x80008000 : 0x80000000)) != 0);
}
// A value that the compiler does not know, so that what follows from it is not kept in registers over a loop.
__device__ __forceinline__ int unknown(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
// Of two bf16 values of neighbouring keys those up to position `upto`.
__device__ __forceinline__ uint32_t cut_mask(int key, int upto) {
    return (key <= upto ? 0xffffu : 0u) | (key < upto ? 0xffff0000u : 0u);
}

// Scores of a block, in units of log2, those that a row does not read at -inf.
template <typename T, int HD, int NT>
__device__ __forceinline__ void block_scores(const Block<T, HD>& x, const u4 (&q)[NT][Block<T, HD>::NK],
                                             f4 (&sc)[NT][Block<T, HD>::TK], const int* page, int k0, const int (&pos)[NT],
                                             bool whole, float scale, int lane) {
    using B = Block<T, HD>;
    const int g = lane >> 4;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int t = 0; t < B::TK; ++t) {
            f4 s = f4{0.f, 0.f, 0.f, 0.f};
            if constexpr (B::H) {
#pragma unroll
                for (int i = 0; i < B::NK; ++i)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, x.k[t][i]), __builtin_bit_cast(b8, q[j][i]),
                                                                s, 0, 0, 0);
            } else {
                f4 s1 = s;  // two chains
#pragma unroll
                for (int i = 0; i < B::NK; ++i) {
                    const f4 kk = __builtin_bit_cast(f4, x.k[t][i]), qq = __builtin_bit_cast(f4, q[j][i]);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        s = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], qq[e], s, 0, 0, 0);
                        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e + 1], qq[e + 1], s1, 0, 0, 0);
                    }
                }
                s += s1;
            }
            s *= scale;
            if (!whole)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = page[t] >= 0 && k0 + 16 * t + 4 * g + r <= pos[j] ? s[r] : -INFINITY;
            sc[j][t] = s;
        }
}

// The block's part of the softmax: its scores become weights.
template <typename T, int HD, int NT>
__device__ __forceinline__ void block_weights(Acc<T, HD, NT>& acc, f4 (&sc)[NT][Block<T, HD>::TK]) {
    using B = Block<T, HD>;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        f4(&s)[B::TK] = sc[j];
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < B::TK; ++t) mx = fmaxf(mx, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
        mx = fmaxf(acc.m[j], col_max(mx));
        // (nothing readable yet: the maximum is -inf, and every weight 0)
        const float base = mx == -INFINITY ? 0.f : mx;
        if (__any(mx != acc.m[j])) {
            const float f = __builtin_amdgcn_exp2f(acc.m[j] - base);
            acc.l[j] *= f;
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) acc.o[j][i] *= f;
            acc.m[j] = mx;
        }
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < B::TK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - base);
                sum += s[t][r];
            }
        acc.l[j] += sum;
    }
}

// The weights in the type of the matrix instruction that v enters as it is, bf16, as the sum of two: the leading
// digits (less than the weight by up to 2^-7 of it), and what they left out rounded (half a step, 2^-8 of that).  Neither
// is 0 or negative unless the weight is 0, so that an infinity of v stays what it is.  The largest error of 64
// sequences of up to 4000 is 1.8e-3, the output's own rounding, and 2.2e-3 with the weights rounded once.  That would save
// 0.2 us of 7.1 for one short sequence, 3 % for blocks of eight rows, 7 % for 64 query vectors of head dim 32, and
// nothing in long batches, whose matrix cores wait for bytes.
struct Split {
    u4 hi, lo;
};
__device__ __forceinline__ Split split_b8(const f4 (&s)[2]) {
    Split w;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const float x = s[d / 2][d % 2 * 2], y = s[d / 2][d % 2 * 2 + 1];
        const uint32_t a = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xffff0000,
                       b = __builtin_elementwise_sub_sat(__float_as_uint(y), 1u) & 0xffff0000;
        w.hi[d] = __builtin_amdgcn_perm(b, a, 0x07060302);
        w.lo[d] = pack_bf16(x - __uint_as_float(a), y - __uint_as_float(b));
    }
    return w;
}
__device__ __forceinline__ f4 mfma_b8(u4 v, u4 w, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, v), __builtin_bit_cast(b8, w), c, 0, 0, 0);
}
// Columns 16 i .. 16 i + 15 of a bf16 block's V as an operand.
template <int HD>
__device__ __forceinline__ u4 values_b8(const Block<uint16_t, HD>& x, int i, int zero = 0) {
    u4 w;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        w[d] = __builtin_amdgcn_perm(x.v[2 * d + 1][0][i / 2], x.v[2 * d][0][i / 2], (i % 2 ? 0x07060302 : 0x05040100) + zero);
    return w;
}

// The block's product with V.
template <typename T, int HD, int NT>
__device__ __forceinline__ void block_sums(const Block<T, HD>& x, const f4 (&sc)[NT][Block<T, HD>::TK], Acc<T, HD, NT>& acc) {
    using B = Block<T, HD>;
    if constexpr (B::H) {
        Split p[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) p[j] = split_b8(sc[j]);
        // (all of the leading digits' products first, where registers hold the operands meanwhile: 7.07 and 7.19 us for
        // one short sequence)
        constexpr int W = NT == 1 || HD < 128 ? HD / 16 : 1;
#pragma unroll
        for (int i0 = 0; i0 < HD / 16; i0 += W) {
            u4 w[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                w[i] = values_b8<HD>(x, i0 + i);
#pragma unroll
                for (int j = 0; j < NT; ++j) acc.o[j][i0 + i] = mfma_b8(w[i], p[j].hi, acc.o[j][i0 + i]);
            }
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc.o[j][i0 + i] = mfma_b8(w[i], p[j].lo, acc.o[j][i0 + i]);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int u = 0; u < B::VU; ++u)
#pragma unroll
                for (int e = 0; e < B::VW; ++e)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        acc.o[j][u * B::VW + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[r][u][e]), sc[j][0][r],
                                                                                     acc.o[j][u * B::VW + e], 0, 0, 0);
    }
}

template <typename T, int HD>
__device__ __forceinline__ bool block_odd(const Block<T, HD>& x) {
    using B = Block<T, HD>;
    uint32_t any = 0;
#pragma unroll
    for (int r = 0; r < 4 * B::TK; ++r)
#pragma unroll
        for (int u = 0; u < B::VU; ++u)
#pragma unroll
            for (int e = 0; e < B::VD; ++e) any |= odd_bits<T>(x.v[r][u][e]);
    return any_odd<T>(any);
}
// block_sums for a block with such values, whose rows end at `from` .. `upto` (or behind).
template <typename T, int HD, int NT>
__device__ __forceinline__ void block_sums_odd(const Block<T, HD>& x, const f4 (&sc)[NT][Block<T, HD>::TK], int k0, int from,
                                               int upto, const int (&pos)[NT], Acc<T, HD, NT>& acc, int lane) {
    using B = Block<T, HD>;
#pragma unroll 1
    for (int at = from; at <= upto; ++at)
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            const int key = unknown(k0 + (lane >> 4) * 4);
            u4 w = {};
            if constexpr (B::H) {
                w = values_b8<HD>(x, i, unknown(0));
#pragma unroll
                for (int d = 0; d < 4; ++d) w[d] &= cut_mask(key + 16 * (d / 2) + d % 2 * 2, at);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                f4 c = {0.f, 0.f, 0.f, 0.f};
                if constexpr (B::H) {
                    const Split p = split_b8(sc[j]);
                    c = mfma_b8(w, p.hi, mfma_b8(w, p.lo, c));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        c = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            key + r <= at ? __uint_as_float(x.v[r][i / B::VW][i % B::VW]) : 0.f, sc[j][0][r], c, 0, 0, 0);
                }
                const bool mine = min(pos[j], upto) == at;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc.o[j][i][r] += mine ? c[r] : 0.f;
            }
        }
}

// Query vector v of a sequence and KV head: row v / G of the sequence, head kvh * G + v % G.
template <typename T, int HD, int NT>
__global__ __launch_bounds__(64 * kDecodeWaves, 2) void k_pdecode(DecodeArgs d) {
    using B = Block<T, HD>;
    constexpr int QV = 16 * NT, BK = kBlockKeys<T>;
    __shared__ __attribute__((aligned(16))) f4 os[kDecodeWaves / 2][NT * (HD / 16)][64];
    __shared__ float ms[kDecodeWaves][QV][2];
    const PagedAttnArgs& a = d.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    // groups of one unit and KV head that read the same keys lie on one XCD (workgroups go round
    // them in turn)
    const int per = (d.units * a.c.Hkv + 7) / 8 * 8;
    const int cg = blockIdx.x / per, unit = blockIdx.x % per / a.c.Hkv, kvh = blockIdx.x % per % a.c.Hkv;
    if (unit >= d.units) return;
    const Units un = units_of<T>(d, unit, 0);
    const int b = un.b;
    if (b < 0) return;
    const int G = a.H / a.c.Hkv;
    // the first two blocks' table entries, which need no length (a sequence that is one unit has been asked
    // for nothing else yet, and one round trip to memory is saved)
    constexpr int step = kDecodeWaves * BK;
    const int kb = (unit - un.first) * un.keys;
    int k0 = kb + wave * BK;
    int entry[2][B::TK];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < B::TK; ++t) {
            const int j = (k0 + i * step + 16 * t) >> a.c.shift;
            entry[i][t] = j < a.c.max_pages ? a.c.table[(int64_t)b * a.c.max_pages + j] : -1;
        }
    const int r0 = uniform(un.rows.r0), nrows = uniform(un.rows.n), len = uniform(un.rows.len);
    const int nqv = nrows * G, v0 = cg * QV;
    if (v0 >= nqv) return;
    // the unit's positions that some row of this group reads
    const int ke = min(min(len - nrows + min(v0 + QV - 1, nqv - 1) / G + 1, seq_end(a, un.rows)), un.count > 1 ? kb + un.keys : INT32_MAX);
    const bool whole_seq = un.count == 1;
    const int64_t slot = ((int64_t)unit * a.c.Hkv + kvh) * d.ncg + cg;
    u4 q[NT][B::NK];
    int pos[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int v = v0 + 16 * j + n, row = min(v, nqv - 1) / G, h = kvh * G + min(v, nqv - 1) % G;
        pos[j] = len - nrows + row;
        const T* p = (const T*)a.q + (r0 + row) * a.q_stride + h * HD + g * (16 / (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < B::NK; ++i) q[j][i] = *(const u4*)(p + i * (64 / (int)sizeof(T)));
    }
    const int first = len - nrows + v0 / G;  // of the group's rows
    const float scale = a.scale * kLog2e;
    Acc<T, HD, NT> acc;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        acc.m[j] = -INFINITY;
        acc.l[j] = 0.f;
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) acc.o[j][i] = f4{0.f, 0.f, 0.f, 0.f};
    }
    auto look = [&](int k0, int (&page)[B::TK]) {
#pragma unroll
        for (int t = 0; t < B::TK; ++t)
            page[t] = k0 + 16 * t < ke ? __builtin_amdgcn_readfirstlane(paged_page(a.c, b, (k0 + 16 * t) >> a.c.shift)) : -1;
    };
    int page[3][B::TK];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < B::TK; ++t) {
            const int p = uniform(entry[i][t]);
            page[i][t] = k0 + i * step + 16 * t < ke && (uint32_t)p < (uint32_t)a.c.n_pages ? p : -1;
        }
    f4 sc[NT][B::TK];
    auto whole = [&](int k) {
        bool w = k + BK - 1 <= min(first, ke - 1);
#pragma unroll
        for (int t = 0; t < B::TK; ++t) w &= page[0][t] >= 0;
        return w;
    };
    auto shift = [&] {
#pragma unroll
        for (int t = 0; t < B::TK; ++t) {
            page[0][t] = page[1][t];
            page[1][t] = page[2][t];
        }
    };
    // whether rows differ in what they read of a block; such blocks come last
    auto mixed = [&](int k) { return min(k + BK, ke) - 1 > first; };
    bool odd = false;
    if constexpr (NT == 1) {
        // the next block is requested before this one is used
        Block<T, HD> x[2];
        load_block<T, HD, kLoadK | kLoadV>(x[0], a.c, kvh, page[0], k0, ke, lane);
        for (; k0 < ke; k0 += 2 * step) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = k0 + i * step;
                if (k >= ke) break;
                look(k + 2 * step, page[2]);
                load_block<T, HD, kLoadK | kLoadV>(x[1 - i], a.c, kvh, page[1], k + step, ke, lane);
                if (mixed(k) && block_odd<T, HD>(x[i])) {
                    odd = true;
                    k0 = k;
                    break;
                }
                block_scores<T, HD, NT>(x[i], q, sc, page[0], k, pos, whole(k), scale, lane);
                block_weights<T, HD, NT>(acc, sc);
                block_sums<T, HD, NT>(x[i], sc, acc);
                shift();
            }
            if (odd) break;
        }
    } else {
        // registers for one block: its K is replaced when the scores are there, its V when the sums are
        Block<T, HD> x;
        load_block<T, HD, kLoadK | kLoadV>(x, a.c, kvh, page[0], k0, ke, lane);
        for (; k0 < ke && !(mixed(k0) && block_odd<T, HD>(x)); k0 += step) {
            look(k0 + 2 * step, page[2]);
            block_scores<T, HD, NT>(x, q, sc, page[0], k0, pos, whole(k0), scale, lane);
            load_block<T, HD, kLoadK>(x, a.c, kvh, page[1], k0 + step, ke, lane);
            block_weights<T, HD, NT>(acc, sc);
            block_sums<T, HD, NT>(x, sc, acc);
            load_block<T, HD, kLoadV>(x, a.c, kvh, page[1], k0 + step, ke, lane);
            shift();
        }
    }
    // from a block with infinities or NaN on one by one, apart so that it costs the others no registers
#pragma unroll 1
    for (; k0 < ke; k0 += step) {
        Block<T, HD> x;
        const int lane = unknown(threadIdx.x) & 63;
        look(k0, page[0]);
        load_block<T, HD, kLoadK>(x, a.c, kvh, page[0], k0, ke, lane);
        block_scores<T, HD, NT>(x, q, sc, page[0], k0, pos, false, scale, lane);
        block_weights<T, HD, NT>(acc, sc);
        load_block<T, HD, kLoadV>(x, a.c, kvh, page[0], k0, ke, lane);
        block_sums_odd<T, HD, NT>(x, sc, k0, max(first, k0), min(k0 + BK, ke) - 1, pos, acc, lane);
    }
    // the waves' parts on one maximum, then added
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        acc.l[j] = col_sum(acc.l[j]);
        if (g == 0) {
            ms[wave][16 * j + n][0] = acc.m[j];
            ms[wave][16 * j + n][1] = acc.l[j];
        }
    }
    __syncthreads();
    float mt[NT], lt[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) m = fmaxf(m, ms[w][16 * j + n][0]);
        mt[j] = m;
        const float base = m == -INFINITY ? 0.f : m;
        lt[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) lt[j] += ms[w][16 * j + n][1] * __builtin_amdgcn_exp2f(ms[w][16 * j + n][0] - base);
        const float f = __builtin_amdgcn_exp2f(acc.m[j] - base);
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) acc.o[j][i] *= f;
    }
#pragma unroll
    for (int half = kDecodeWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) os[wave - half][j * (HD / 16) + i][lane] = acc.o[j][i];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) acc.o[j][i] += os[wave][j * (HD / 16) + i][lane];
        __syncthreads();
    }
    if (wave) return;
    // a lane holds, of query vector n, columns (16 u + 4 g + r) VW + e for r < 4, e < VW
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int v = v0 + 16 * j + n;
        const float inv = !whole_seq ? 1.f : inverse(a.c, b, lt[j], pos[j], len - nrows + min(v0 + QV - 1, nqv - 1) / G);
#pragma unroll
        for (int u = 0; u < B::VU; ++u) {
            float y[4 * B::VW];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < B::VW; ++e) y[r * B::VW + e] = acc.o[j][u * B::VW + e][r] * inv;
            const int c = (16 * u + 4 * g) * B::VW;
            if (!whole_seq) {
                float* p = d.part + (slot * QV + 16 * j + n) * HD + c;
#pragma unroll
                for (int i = 0; i < 4 * B::VW; i += 4) *(f4*)(p + i) = f4{y[i], y[i + 1], y[i + 2], y[i + 3]};
            } else if (v < nqv) {
                put<T, 4 * B::VW>(a, r0 + v / G, (kvh * G + v % G) * HD + c, y);
            }
        }
        if (!whole_seq && g == 0) {
            float* p = d.part + d.ml + (slot * QV + 16 * j + n) * 2;
            *(f2*)p = f2{mt[j], lt[j]};
        }
    }
}

// `live` partials, `next` query vectors apart, joined: 4 columns of one, and its sum of weights.
__device__ __forceinline__ f4 join_parts(const float* po, const float* pm, int live, int64_t next, int hd, float& l) {
    float m = -INFINITY;
    l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < live; s0 += 8) {
        f2 ml[8];
        f4 x[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int64_t k = min(s0 + s, live - 1) * next;
            ml[s] = *(const f2*)(pm + k * 2);
            x[s] = *(const f4*)(po + k * hd);
        }
        float mn = m;
#pragma unroll
        for (int s = 0; s < 8; ++s) mn = fmaxf(mn, ml[s][0]);
        const float base = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(m - base);
        l *= f;
        o *= f;
        m = mn;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const bool on = s0 + s < live;  // (a select: 0 times an infinity is NaN)
            const float w = on ? __builtin_amdgcn_exp2f(ml[s][0] - base) : 0.f;
            l += w * ml[s][1];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += on ? w * x[s][i] : 0.f;
        }
    }
    return o;
}

// The units of a sequence joined: a thread per query vector and 4 columns.
template <typename T, int HD, int NT>
__global__ __launch_bounds__(256) void k_pjoin(DecodeArgs d) {
    constexpr int QV = 16 * NT, PER = 256 / (HD / 4);
    const PagedAttnArgs& a = d.a;
    const int nb = (QV + PER - 1) / PER, group = blockIdx.x / nb;
    const int i = blockIdx.x % nb * PER + threadIdx.x / (HD / 4), c = threadIdx.x % (HD / 4) * 4;
    const int cg = group % d.ncg, kvh = group / d.ncg % a.c.Hkv, b = group / d.ncg / a.c.Hkv, G = a.H / a.c.Hkv;
    const Units un = units_of<T>(d, -1, b);
    const int live = un.count;
    if (live == 1) return;
    const int r0 = un.rows.r0, nqv = un.rows.n * G, v0 = cg * QV, n = min(QV, nqv - v0);
    if (!__any(i < n)) return;
    const int at = min(i, n - 1), v = v0 + at;  // (lanes without a query vector go along with the last one)
    // from one unit's partials to the next
    const int64_t slot = ((int64_t)un.first * a.c.Hkv + kvh) * d.ncg + cg, next = (int64_t)a.c.Hkv * d.ncg * QV;
    const float* po = d.part + (slot * QV + at) * HD + c;
    const float* pm = d.part + d.ml + (slot * QV + at) * 2;
    float sum;
    const f4 parts = join_parts(po, pm, live, next, HD, sum);
    const int at0 = un.rows.len - un.rows.n;
    const f4 o = parts * inverse(a.c, b, sum, at0 + v / G, at0 + (v0 + n - 1) / G);
    const float y[4] = {o[0], o[1], o[2], o[3]};
    if (i < n) put<T, 4>(a, r0 + v / G, (kvh * G + v % G) * HD + c, y);
}

// ---------------------------------------------------------------------------------------------
// Many rows per sequence (prompts): k_pprompt_bf16.  A workgroup takes 256 query vectors of a sequence and
// KV head, 32 to each of its eight waves, and goes through the keys in tiles of KT, whose K and V
// arrive in LDS by themselves (loads with LDS as their destination), one tile ahead.  The products are
// those of k_pdecode on 32 x 32 tiles: in the result of S^T = K Q^T lane group g holds keys 8 (r / 4) + 4 g +
// r % 4, r < 16, of one query vector, which are the contraction slots of the two PV products.  V's
// eight keys of a column come out of LDS by reads that turn 4 x 16 blocks.
//
// The two waves of a SIMD take turns: while one computes weights (vector instructions) the other has the
// matrix cores and LDS (its sums with V, then the next block's scores, the operands of both read
// meanwhile); a barrier after each turn keeps them apart.  Unsynchronised, both tended to want the same unit:
// 8192 positions, 32/8 heads of 128, took 660 us that way, 570 in turns, and 510 to 540 (1.05 PFLOP/s; a large
// matrix product of torch reaches 1.16) since the waves' turns are balanced (about 700 cycles of softmax
// and 660 of matrix work in a slot of 945) and rows are stored whole.  Besides, a workgroup takes 6 to 8 thousand
// cycles until its first scores and 5 for its rows, which short prompts show: 24 of 1 to 2001 positions reach
// 0.7 PFLOP/s.
//
// The running maximum is raised only when a weight exceeds 2^kLazy: until then the sums need no
// rescaling, and a block's scores no maximum, since large weights show in their bits.
//
// With few workgroups the keys of each are split into spans, whose partial sums k_prompt_join joins.
// ---------------------------------------------------------------------------------------------
typedef float f16v __attribute__((ext_vector_type(16)));
constexpr int kLazy = 8;
constexpr int kPromptWaves = 8;
// Keys of a tile in LDS (bf16): 32 KB of K and of V, or 256 of head dim 32.
constexpr int prompt_keys(int hd) { return hd == 128 ? 128 : 256; }

struct PromptArgs {
    PagedAttnArgs a;
    int tiles;    // workgroups of a KV head and span
    int nspan, least;  // spans at most, keys of one at least
    float* part;  // partials: [tile][KV head][span] of [QV][HD] sums, then of [QV] (maximum, sum)
    int64_t ml;   // floats of the first
};

// Maximum and sum over the two halves of a wave.
__device__ __forceinline__ float half_max(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Workgroup w of a KV head: its sequence (-1: none) and first query vector there.  A sequence's tiles of QV
// query vectors are numbered from its first row on, and the last tiles of all sequences go first, since
// they read the most keys.
struct Tile {
    int b, v0;
    SeqRows rows;
};
template <int QV>
__device__ __forceinline__ Tile prompt_tile(const PagedRows& r, int G, int w) {
    const int most = ((int64_t)r.max_rows * G + QV - 1) / QV;  // of a sequence
    Tile t;
    t.b = -1;
    t.v0 = 0;
    if (!r.row_off) {
        if (w >= most * r.nseq) return t;
        t.b = w % r.nseq;
        t.v0 = (most - 1 - w / r.nseq) * QV;
        t.rows = seq_rows(r, t.b);
        return t;
    }
    const int lane = threadIdx.x & 63;
    SeqRows mine = lane < r.nseq ? seq_rows(r, lane) : SeqRows{};
    auto tiles_of = [&](const SeqRows& s) { return (int)(((int64_t)s.n * G + QV - 1) / QV); };
    auto others = [&](int b) { return tiles_of(b < r.nseq ? seq_rows(r, b) : SeqRows{}); };
    const int tiles = tiles_of(mine);
    // tiles numbered j or more
    auto from = [&](int j) {
        int n = max(tiles - j, 0);
        for (int b0 = 64; b0 < r.nseq; b0 += 64) n += max(others(b0 + lane) - j, 0);
        return wave_total(n);
    };
    // the largest j with more than w of them
    if (from(0) <= w) return t;
    int lo = 0, hi = most;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (from(mid) > w) lo = mid;
        else hi = mid;
    }
    t.v0 = lo * QV;
    int rank = w - from(lo + 1);  // among the sequences that have a tile lo
    for (int b0 = 0; b0 < r.nseq; b0 += 64) {
        if (b0) mine = b0 + lane < r.nseq ? seq_rows(r, b0 + lane) : SeqRows{};
        const bool has = tiles_of(mine) > lo;
        const uint64_t m = __ballot(has);
        const int c = __popcll(m);
        if (rank < c) {
            const uint64_t me = __ballot(has && __popcll(m & (((uint64_t)1 << lane) - 1)) == rank);
            const int l = __builtin_ctzll(me);
            t.b = b0 + l;
            t.rows = lane_rows(mine, l);
            break;
        }
        rank -= c;
    }
    return t;
}

// Keys of a span, the same number for all tiles, so that the workgroups' work is alike: the longest sequence's in
// nspan parts, which the lengths on the device say.  What the call expects may be far more: with spans of that
// length 512 bf16 rows (32/8 heads of 128) of 20000 positions, of 150000 that the table holds, took 459 us, not 186, and 64 fp32
// rows of four sequences of 2000 527, not 109; with the length known, parts from the device cost up to 1.5 us.
// For whole waves; mine: the tile's sequence.
__device__ __forceinline__ int span_keys(const PromptArgs& d, int kt, const SeqRows& mine) {
    if (d.nspan == 1) return 1 << 30;
    int longest = seq_end(d.a, mine);
    if (d.a.r.nseq > 1) {
        for (int b0 = 0; b0 < d.a.r.nseq; b0 += 64) {
            const int b = b0 + (threadIdx.x & 63);
            if (b < d.a.r.nseq) longest = max(longest, seq_end(d.a, seq_rows(d.a.r, b)));
        }
        longest = wave_most(longest);
    }
    return max(((longest + d.nspan - 1) / d.nspan + kt - 1) / kt * kt, d.least);
}
// The keys of a tile that workgroup `span` of it reads: of `end` in all, `keys` to each; the last span takes
// what is left.
struct Span {
    int from, upto, live;  // spans that have keys
};
__device__ __forceinline__ Span prompt_span(int end, int nspan, int keys, int span) {
    Span s;
    s.live = min(max((int)(((int64_t)end + keys - 1) / keys), 1), nspan);
    s.from = span < s.live ? span * keys : 0;
    s.upto = span + 1 < s.live ? s.from + keys : end;
    return s;
}

template <int HD>
__global__ __launch_bounds__(64 * kPromptWaves, HD == 32 ? 4 : 2) void k_pprompt_bf16(PromptArgs d) {
    constexpr int NW = kPromptWaves, KT = prompt_keys(HD), NB = KT / 32, NS = HD / 16, NC = HD / 32, CH = HD / 8;
    constexpr int QV = 32 * NW, RB = HD * 2;
    __shared__ __attribute__((aligned(1024))) char ks[2][KT * RB], vs[2][KT * RB];
    const PagedAttnArgs& a = d.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;
    const int G = a.H / a.c.Hkv;
    // (KV heads lie on XCDs in turn)
    const int kvh = blockIdx.x % a.c.Hkv, span = blockIdx.x / a.c.Hkv % d.nspan, tile = blockIdx.x / a.c.Hkv / d.nspan;
    const Tile tl = prompt_tile<QV>(a.r, G, tile);
    const int b = uniform(tl.b), v0 = uniform(tl.v0), r0 = uniform(tl.rows.r0), nrows = uniform(tl.rows.n);
    if (b < 0) return;
    const int nqv = nrows * G;
    if (v0 >= nqv) return;
    // table entries of the KT / 16 groups of keys of a tile, a lane each, and the pages they name (apart: the
    // first test of an entry waits for it, and for all loads before).  Those of the first two tiles, and q, are
    // requested before the length is there.
    auto ask = [&](int key) {
        int e = -1;
        if (lane < KT / 16 && key >> a.c.shift < a.c.max_pages) e = a.c.table[(int64_t)b * a.c.max_pages + (key >> a.c.shift)];
        return e;
    };
    // (Where keys are split, the first one's position follows from the lengths.)
    int entry = -1, entry1 = -1;
    if (d.nspan == 1) {
        entry = ask(16 * lane);
        entry1 = ask(KT + 16 * lane);
    }
    const int wv = v0 + 32 * wave;  // the wave's first query vector
    u4 q[NS];
    const int v = wv + n, vc = min(v, nqv - 1);
    {
        const uint16_t* p = (const uint16_t*)a.q + (r0 + vc / G) * a.q_stride + (kvh * G + vc % G) * HD + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = *(const u4*)(p + 16 * s);
    }
    const int at0 = uniform(tl.rows.len) - nrows, pos = at0 + vc / G;
    const Span sp = prompt_span(max(min(at0 + min(v0 + QV - 1, nqv - 1) / G + 1, (int64_t)a.c.max_pages << a.c.shift), 0), d.nspan, span_keys(d, KT, tl.rows), span);
    if (span >= sp.live) return;
    const int end = sp.upto;
    const int wfirst = at0 + wv / G, wend = wv < nqv ? min(end, at0 + min(wv + 31, nqv - 1) / G + 1) : 0;
    auto look = [&](int k0) {
        const int key = k0 + 16 * lane;
        return key < end ? ask(key) : -1;
    };
    auto named = [&](int e) { return (uint32_t)e < (uint32_t)a.c.n_pages ? e : -1; };
    const int t0 = sp.from / KT, nt = (end + KT - 1) / KT;
    if (d.nspan > 1) {
        entry = look(t0 * KT);
        entry1 = look((t0 + 1) * KT);
    } else {
        if (16 * lane >= end) entry = -1;
        if (KT + 16 * lane >= end) entry1 = -1;
    }
    const float c = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;
    f16v o[NC];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    const int mask = (1 << a.c.shift) - 1;
    // This wave's groups of 16 keys of a tile, straight into LDS, 1 KB an instruction: 16-byte unit u of a
    // row at u ^ (row % 8) (K) and u ^ 2 (row % 4) (V).  Rows that do not exist arrive as zeros.
    constexpr int RL = 16 / CH, RI = 64 / CH, NI = 16 / RI;  // rows of 256 bytes; rows of an instruction, instructions of a group
    const int lrow = lane / CH, lch = lane % CH;
    auto load = [&](int k0, int pg, int buf) {
#pragma unroll
        for (int w = 0; w < KT / 8 / NW; ++w) {
            const int task = wave + w * NW, grp = task % (KT / 16), key = k0 + 16 * grp, page = __builtin_amdgcn_readlane(pg, grp);
            const int rows = uniform(page < 0 ? 0 : max(min(end - key, 16), 0));
            const int64_t at = max(page, 0) * a.c.page_stride + (((int64_t)kvh << a.c.shift) + (key & mask)) * HD;
            const bool isv = task >= KT / 16;
            const int64_t base = uniform((int64_t)((uint16_t*)(isv ? a.c.v : a.c.k) + at));
            const u4 rs = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffff, (uint32_t)(rows * RB), 0x00020000};
            typedef __attribute__((address_space(3))) char* lds;
            const uint32_t to = uniform((int)(uint32_t)(uintptr_t)(lds)((isv ? vs[buf] : ks[buf]) + grp * 16 * RB));
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int row = i * RI + lrow;
                const int off = row * RB + ((lch ^ ((isv ? 4 * ((row & 3) / RL) : row / RL) & (CH - 1))) * 16);
                // (no builtin: with it every read of LDS waits for what is still on its way to the other buffers;
                // `meet` below says who waits for what)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                             :: "s"(to + i * 1024), "v"(off), "s"(rs) : "memory");
            }
        }
    };
    const int nk = (wend + 31) / 32;  // blocks of 32 keys up to the last that this wave computes
    // K: row n of a block, units 2 i + g
    int ka[NS], va[NC];
#pragma unroll
    for (int i = 0; i < NS; ++i) ka[i] = n * RB + (((2 * i + g) ^ (n / RL & (CH - 1))) * 16);
    // V: four keys of 16 columns, turned by the read: a lane of 16 reads four columns of key lane / 4
    const int vk = (lane & 15) / 4;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        va[i] = (4 * g + vk) * RB + (((4 * i + (lane >> 4 & 1) * 2 + (lane & 3) / 2) ^ (4 * (vk / RL) & (CH - 1))) * 16) + (lane & 1) * 8;
    u4 kr[NS];
    auto keys = [&](const char* kf, int kb) {
#pragma unroll
        for (int i = 0; i < NS; ++i) kr[i] = *(const u4*)(kf + ka[i] + kb * 32 * RB);
    };
    auto scores = [&](f16v& s) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, kr[i]), __builtin_bit_cast(b8, q[i]), s, 0, 0, 0);
    };
    auto most = [&](const f16v& s) {
        float mx[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) mx[r] = fmaxf(fmaxf(s[r], s[r + 4]), fmaxf(s[r + 8], s[r + 12]));
        return half_max(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]))) * c;
    };
    // block k's scores made ready: those that are not read at -inf, and the maximum raised to them
    auto settle = [&](f16v& s, int k, uint32_t hv) {
        const int k0 = 32 * k;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int key = 8 * (r / 4) + 4 * g + r % 4;
            s[r] = k0 + key <= pos && (hv >> (r / 8) & 1) ? s[r] : -INFINITY;
        }
        const float mx = most(s);
        if (!__any(mx > m + kLazy)) return;
        const float mn = fmaxf(m, mx), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int i = 0; i < NC; ++i) o[i] *= f;
    };
    // (bf16, half a step of 2^-8 each, as much as the output's own rounding; their sum from before it.  As two numbers
    // each, see split_b8, they take half as many matrix instructions again: 8192 positions 718 us, not 526)
    auto weights = [&](const f16v& s, u4 (&p)[2]) {
        const float base = m == -INFINITY ? 0.f : m;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -base)),
                        y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], c, -base));
            sum[0] += x;
            sum[1] += y;
            p[r / 8][r % 8 / 2] = pack_bf16(x, y);
        }
        return sum[0] + sum[1];
    };
    // Whether a weight exceeds 2^kLazy (or is no number): they are positive, so their bits compare as integers do.
    typedef uint16_t h2 __attribute__((ext_vector_type(2)));
    auto large = [&](const u4 (&p)[2]) {
        h2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_elementwise_max(__builtin_bit_cast(h2, p[0][i]), __builtin_bit_cast(h2, p[1][i]));
        const h2 y = __builtin_elementwise_max(__builtin_elementwise_max(x[0], x[1]), __builtin_elementwise_max(x[2], x[3]));
        return max(y[0], y[1]) > (uint16_t)((127 + kLazy) << 7);
    };
    typedef short h4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) h4* ldsv;
    auto values = [&](u4 (&x)[2][NC], const char* vf, int kb) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const char* p = vf + va[i] + (kb * 32 + 16 * u) * RB;
                const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldsv)p));
                const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldsv)(p + 8 * RB)));
                x[u][i] = u4{lo[0], lo[1], hi[0], hi[1]};
            }
    };
    auto sums = [&](const u4 (&p)[2], const u4 (&x)[2][NC]) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < NC; ++i)
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, x[u][i]), __builtin_bit_cast(b8, p[u]), o[i], 0, 0, 0);
    };
    // (as block_odd; the block's V is 0 afterwards)
    auto odd = [&](const u4 (&p)[2], u4 (&x)[2][NC], int k) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 8 * NC; ++i) any |= odd_bits<uint16_t>(x[i / 4 % 2][i / 8][i % 4]);
        if (!any_odd<uint16_t>(any)) return;
        const int upto = min(32 * k + 32, end) - 1;
#pragma unroll 1
        for (int at = max(wfirst, 32 * k); at <= upto; ++at)
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const int key = unknown(32 * k + 4 * g);
                f16v w = {};
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    u4 y;
#pragma unroll
                    for (int d = 0; d < 4; ++d) y[d] = x[u][i][d] & cut_mask(key + 16 * u + 8 * (d / 2) + d % 2 * 2, at);
                    w = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, y), __builtin_bit_cast(b8, p[u]), w, 0, 0, 0);
                }
                const bool mine = min(pos, upto) == at;
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] += mine ? w[r] : 0.f;
            }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < NC; ++i) x[u][i] = u4{};
    };
    auto meet = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const bool late = wave >= NW / 2;
    const int nkw = (end + 31) / 32;  // of the workgroup
    int pg = named(entry);
    uint64_t have = __ballot(pg >= 0), next = 0;
    load(t0 * KT, pg, t0 & 1);
    entry = entry1;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    // (a negative scale turns into the sign of q, and 0 into q = 0, NaN where it is no finite number: scores that do
    // not count are -inf before they are scaled)
    if (a.scale != 0.f) {
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < NS; ++i) q[i] ^= flip;
    } else {
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) q[i / 4][i % 4] = (odd_bits<uint16_t>(q[i / 4][i % 4]) >> 15 & 0x00010001) * 0x7fc0;
    }
    __syncthreads();
    f16v s;
    u4 x[2][NC];
    if (t0 * NB < nk) {
        keys(ks[t0 & 1], 0);
        scores(s);
        values(x, vs[t0 & 1], 0);
    }
    bool begun = false;  // every query vector has a maximum
    if (late) meet();
    for (int t = t0; t < nt; ++t) {
        const char *kf = ks[t & 1], *vf = vs[t & 1], *kn = ks[(t + 1) & 1], *vn = vs[(t + 1) & 1];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const int k = t * NB + kb;
            if (k >= nkw) break;
            if (kb == 0) {
                pg = named(entry);
                next = __ballot(pg >= 0);
                if (t + 1 < nt) load((t + 1) * KT, pg, (t + 1) & 1);
                entry = look((t + 2) * KT);
            }
            u4 p[2];
            if (k < nk) {
                const uint32_t hv = have >> (2 * kb) & 3;
                bool settled = begun && 32 * k + 31 <= wfirst && hv == 3;
                float sum = 0.f;
                if (settled) {
                    sum = weights(s, p);
                    settled = !__any(large(p));
                }
                if (!settled) {
                    settle(s, k, hv);
                    sum = weights(s, p);
                    begun = !__any(m == -INFINITY);
                    if (32 * k + 31 > wfirst) odd(p, x, k);
                }
                l += sum;
            }
            if (!late && kb == NB - 1) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
            __builtin_amdgcn_s_waitcnt(0xc07f);                             // lgkmcnt(0)
            meet();
            if (k < nk) {
                __builtin_amdgcn_s_setprio(1);
                keys(kb + 1 < NB ? kf : kn, (kb + 1) % NB);
                sums(p, x);
                scores(s);
                values(x, kb + 1 < NB ? vf : vn, (kb + 1) % NB);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an LDS read
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                }
                __builtin_amdgcn_s_setprio(0);
            }
            if (late && kb == NB - 2) __builtin_amdgcn_s_waitcnt(0x0f70);
            meet();
        }
        have = next;
    }
    if (!late) meet();
    const float sum = half_sum(l);
    if (sp.live > 1) {
        if (v >= nqv) return;
        const int64_t slot = ((int64_t)tile * a.c.Hkv + kvh) * d.nspan + span;
        float* po = d.part + (slot * QV + wv - v0 + n) * HD + 4 * g;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) *(f4*)(po + 32 * i + 2 * r) = f4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
        if (g == 0) *(f2*)(d.part + d.ml + (slot * QV + wv - v0 + n) * 2) = f2{m, sum};
        return;
    }
    // the wave's rows through LDS (its own part of what K and V were in, which nobody uses any more), so that
    // whole rows are stored: 8 bytes a lane to 64 rows took 2 to 4 us
    const float inv = inverse(a.c, b, sum, pos, at0 + min(wv + 31, nqv - 1) / G);
    constexpr int OB = RB + 16;
    char* const os = (late ? vs[0] : ks[0]) + wave % (NW / 2) * 32 * OB;
    static_assert(NW / 2 * 32 * OB <= 2 * KT * RB, "the waves' rows fit");
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(u2*)(os + n * OB + (32 * i + 2 * r + 4 * g) * 2) = u2{pack_bf16(o[i][r] * inv, o[i][r + 1] * inv), pack_bf16(o[i][r + 2] * inv, o[i][r + 3] * inv)};
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 32 * CH / 64; ++i) {
        const int row = i * (64 / CH) + lane / CH, w = wv + row;
        if (w < nqv)
            *(u4*)((uint16_t*)a.out + (r0 + w / G) * a.out_stride + (kvh * G + w % G) * HD + lane % CH * 8) = *(const u4*)(os + row * OB + lane % CH * 16);
    }
}

// The same on fp32 matrix instructions (115 TFLOP/s at 4096 positions, 32/8 heads of 128; a large product of torch
// reaches 154), 32 query vectors per wave and tiles of 32 keys, row by row in LDS
// (rows of K four words apart from whole bank rounds).  A lane reads a row of K, or HD / 32 neighbouring
// columns of its keys of V, at a time.
template <int HD>
__global__ __launch_bounds__(256, 2) void k_pprompt_f32(PromptArgs d) {
    constexpr int KT = 32, QV = 128, C4 = HD / 4, KL = HD + 4, VW = HD / 32, NU = KT * C4 / 256;
    __shared__ __attribute__((aligned(16))) float ks[2][KT * KL], vs[2][KT * HD];
    const PagedAttnArgs& a = d.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, g = lane >> 5;
    const int G = a.H / a.c.Hkv;
    const int kvh = blockIdx.x % a.c.Hkv, span = blockIdx.x / a.c.Hkv % d.nspan, tile = blockIdx.x / a.c.Hkv / d.nspan;
    const Tile tl = prompt_tile<QV>(a.r, G, tile);
    const int b = uniform(tl.b), v0 = uniform(tl.v0), r0 = uniform(tl.rows.r0), nrows = uniform(tl.rows.n);
    if (b < 0) return;
    const int nqv = nrows * G;
    if (v0 >= nqv) return;
    const int at0 = uniform(tl.rows.len) - nrows;
    const int wv = v0 + 32 * wave;
    const Span sp = prompt_span(max(min(at0 + min(v0 + QV - 1, nqv - 1) / G + 1, (int64_t)a.c.max_pages << a.c.shift), 0), d.nspan, span_keys(d, KT, tl.rows), span);
    if (span >= sp.live) return;
    const int end = sp.upto;
    const int wfirst = at0 + wv / G, wend = wv < nqv ? min(end, at0 + min(wv + 31, nqv - 1) / G + 1) : 0;
    const float c = a.scale * kLog2e;
    f4 q[HD / 8];
    const int v = wv + n, vc = min(v, nqv - 1), pos = at0 + vc / G;
    {
        const float* p = (const float*)a.q + (r0 + vc / G) * a.q_stride + (kvh * G + vc % G) * HD + 4 * g;
#pragma unroll
        for (int s = 0; s < HD / 8; ++s) q[s] = *(const f4*)(p + 8 * s) * c;
    }
    f16v o[VW];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < VW; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    const int mask = (1 << a.c.shift) - 1;
    u4 st[2][NU];
    auto look = [&](int k0, int (&page)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            page[t] = k0 + 16 * t < end ? __builtin_amdgcn_readfirstlane(paged_page(a.c, b, (k0 + 16 * t) >> a.c.shift)) : -1;
    };
    // unit i of a thread: row i * 1024 / HD + tid / C4, whose group of 16 keys is the same for a wave
    auto load = [&](int k0, const int (&page)[2]) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int t = HD == 32 ? wave >> 1 : i * (1024 / HD) / 16, key = k0 + 16 * t;
            const int pg = HD == 32 ? (t ? page[1] : page[0]) : page[t];
            const int rows = uniform(pg < 0 ? 0 : max(min(end - key, 16), 0));
            const int64_t at = uniform(max(pg, 0) * a.c.page_stride + (((int64_t)kvh << a.c.shift) + (key & mask)) * HD);
            const int off = ((i * (1024 / HD) + tid / C4) % 16 * HD + tid % C4 * 4) * 4;
            st[0][i] = __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc((float*)a.c.k + at, 0, rows * HD * 4, 0x00020000), off, 0, 0);
            st[1][i] = __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc((float*)a.c.v + at, 0, rows * HD * 4, 0x00020000), off, 0, 0);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int row = i * (1024 / HD) + tid / C4, x = tid % C4 * 4;
            *(u4*)(ks[buf] + row * KL + x) = st[0][i];
            *(u4*)(vs[buf] + row * HD + x) = st[1][i];
        }
    };
    const int t0 = sp.from / KT, nt = (end + KT - 1) / KT;
    auto values = [&](const float* vf, int r, float (&x)[VW]) {
        const float* p = vf + (8 * (r / 4) + 4 * g + r % 4) * HD + n * VW;
        if constexpr (VW == 4) *(f4*)x = *(const f4*)p;
        else if constexpr (VW == 2) *(f2*)x = *(const f2*)p;
        else x[0] = *p;
    };
    // Tiles from `from` on.  The first whose V holds infinities or NaN that some rows only read (see odd_bits)
    // and those behind are left to a second, careful pass, apart so that it costs the first no registers.
    int todo = INT32_MAX;
    auto pass = [&](auto careful, int from) {
        constexpr bool kCareful = decltype(careful)::value;
        int pg[2], nx[2];
        look(from * KT, pg);
        look((from + 1) * KT, nx);
        load(from * KT, pg);
        store(from & 1);
        for (int t = from; t < nt; ++t) {
            __syncthreads();
            const int k0 = t * KT;
            const bool whole = k0 + 31 <= wfirst && pg[0] >= 0 && pg[1] >= 0;
            const bool have[2] = {pg[0] >= 0, pg[1] >= 0};
            if (t + 1 < nt) {
                pg[0] = nx[0];
                pg[1] = nx[1];
                load(k0 + KT, pg);
                look(k0 + 2 * KT, nx);
            }
            const float *kf = ks[t & 1], *vf = vs[t & 1];
            if (!kCareful && k0 < wend && k0 + 31 > wfirst && t < todo) {
                uint32_t any = 0;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float x[VW];
                    values(vf, r, x);
#pragma unroll
                    for (int i = 0; i < VW; ++i) any |= odd_bits<float>(__float_as_uint(x[i]));
                }
                if (any_odd<float>(any)) todo = t;
            }
            if (k0 < wend && (kCareful ? t >= todo : t < todo)) {
                f16v s, s1;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = s1[r] = 0.f;
#pragma unroll
                for (int i = 0; i < HD / 8; ++i) {
                    const f4 x = *(const f4*)(kf + n * KL + 8 * i + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], q[i][e], s, 0, 0, 0);
                        s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e + 1], q[i][e + 1], s1, 0, 0, 0);
                    }
                }
                s += s1;
                if (!whole)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = 8 * (r / 4) + 4 * g + r % 4;
                        s[r] = k0 + key <= pos && have[r / 8] ? s[r] : -INFINITY;
                    }
                float mx = s[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
                mx = half_max(mx);
                if (__any(mx > m + kLazy)) {
                    const float mn = fmaxf(m, mx), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                    m = mn;
                    l *= f;
#pragma unroll
                    for (int i = 0; i < VW; ++i) o[i] *= f;
                }
                const float base = m == -INFINITY ? 0.f : m;
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = __builtin_amdgcn_exp2f(s[r] - base);
                    sum += s[r];
                }
                l += sum;
                if constexpr (!kCareful) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float x[VW];
                        values(vf, r, x);
#pragma unroll
                        for (int i = 0; i < VW; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], s[r], o[i], 0, 0, 0);
                    }
                } else {
                    const int upto = min(k0 + 32, end) - 1;
#pragma unroll 1
                    for (int at = max(wfirst, k0); at <= upto; ++at)
#pragma unroll
                        for (int i = 0; i < VW; ++i) {
                            __builtin_amdgcn_sched_barrier(0);
                            const int key = unknown(4 * g), left = at - k0 - key;
                            f16v w = {};
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const float x = vf[(key + 8 * (r / 4) + r % 4) * HD + n * VW + i];
                                w = __builtin_amdgcn_mfma_f32_32x32x2f32(8 * (r / 4) + r % 4 <= left ? x : 0.f, s[r], w, 0, 0, 0);
                            }
                            const bool mine = min(pos, upto) == at;
#pragma unroll
                            for (int r = 0; r < 16; ++r) o[i][r] += mine ? w[r] : 0.f;
                        }
                }
            }
            if (t + 1 < nt) store((t + 1) & 1);
        }
    };
    pass(std::false_type{}, t0);
    if (__syncthreads_or(todo != INT32_MAX)) pass(std::true_type{}, max(t0, (at0 + v0 / G) / KT));
    const float sum = half_sum(l), inv = sp.live > 1 ? 1.f : inverse(a.c, b, sum, pos, at0 + min(wv + 31, nqv - 1) / G);
    if (v >= nqv) return;
    const int64_t at = (((int64_t)tile * a.c.Hkv + kvh) * d.nspan + span) * QV + wv - v0 + n;
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        float y[4 * VW];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < VW; ++i) y[e * VW + i] = o[i][r + e] * inv;
        const int col = (2 * r + 4 * g) * VW;
        if (sp.live > 1) {
#pragma unroll
            for (int i = 0; i < 4 * VW; i += 4) *(f4*)(d.part + at * HD + col + i) = f4{y[i], y[i + 1], y[i + 2], y[i + 3]};
        } else {
            put<float, 4 * VW>(a, r0 + v / G, (kvh * G + v % G) * HD + col, y);
        }
    }
    if (sp.live > 1 && g == 0) *(f2*)(d.part + d.ml + at * 2) = f2{m, sum};
}

// The spans of k_pprompt's tiles joined: a thread per query vector and 4 columns.
template <typename T, int HD, int QV, int KT>
__global__ __launch_bounds__(256) void k_prompt_join(PromptArgs d) {
    constexpr int PER = 256 / (HD / 4), NBK = QV / PER;
    const PagedAttnArgs& a = d.a;
    const int kvh = blockIdx.x / NBK % a.c.Hkv, tile = blockIdx.x / NBK / a.c.Hkv, G = a.H / a.c.Hkv;
    const Tile tl = prompt_tile<QV>(a.r, G, tile);
    if (tl.b < 0) return;
    const int keys = span_keys(d, KT, tl.rows);  // (by whole waves)
    const int v0 = tl.v0, r0 = tl.rows.r0, nqv = tl.rows.n * G;
    const int i = blockIdx.x % NBK * PER + threadIdx.x / (HD / 4), c = threadIdx.x % (HD / 4) * 4;
    if (!__any(v0 + i < nqv)) return;
    const int v = min(v0 + i, nqv - 1);  // (as in k_pjoin)
    const int at0 = tl.rows.len - tl.rows.n;
    const Span sp = prompt_span(max(min(at0 + min(v0 + QV - 1, nqv - 1) / G + 1, (int64_t)a.c.max_pages << a.c.shift), 0), d.nspan, keys, 0);
    if (sp.live == 1) return;
    const int64_t at = ((int64_t)tile * a.c.Hkv + kvh) * d.nspan * QV + v - v0;
    float sum;
    const f4 parts = join_parts(d.part + at * HD + c, d.part + d.ml + at * 2, sp.live, QV, HD, sum);
    const f4 o = parts * inverse(a.c, tl.b, sum, at0 + v / G, at0 + min(v0 + QV - 1, nqv - 1) / G);
    const float y[4] = {o[0], o[1], o[2], o[3]};
    if (v0 + i < nqv) put<T, 4>(a, r0 + v / G, (kvh * G + v % G) * HD + c, y);
}

template <typename T>
constexpr int kPromptQv = sizeof(T) == 2 ? 32 * kPromptWaves : 128;

struct PromptPlan {
    int64_t tiles;
    int nspan, least;
    int64_t ml;
    size_t bytes;
};

// bytes: room for partials.
PromptPlan prompt_plan(const PagedView& c, const PagedRows& r, int H, bool bf16, int64_t max_len, size_t bytes) {
    const int QV = bf16 ? kPromptQv<uint16_t> : kPromptQv<float>;
    const int64_t G = H / c.Hkv, kt = bf16 ? prompt_keys(c.hd) : 32, most = (r.max_rows * G + QV - 1) / QV;
    PromptPlan p{};
    p.tiles = r.row_off ? std::min(r.total_rows * G / QV + r.nseq, r.nseq * most) : r.nseq * most;
    // Workgroups for two rounds of what the CUs hold, one each (head dim 32: two), of at least two tiles; fp32,
    // whose tiles are short: four on each CU, of at least four tiles.  bf16, 4096 positions, 256 / 512 / 1024
    // workgroups: head dim 64 (32/8 heads) 109 / 109 / 168 us, head dim 32 (16 heads) 87 / 74 / 68; fp32, chunks of
    // five sequences, 12 heads of 64, 512 / 768 / 1024 / 1536 / 2048: 74 / 62 / 58 / 56 / 63, but 4096 positions of 32/8
    // heads of 128 take 1195 us with 1024 and 1611 with 2048
    const int64_t groups = std::max<int64_t>(1, p.tiles * c.Hkv), least = kt * (bf16 ? 2 : 4);
    int64_t want = std::max<int64_t>(1, (bf16 && c.hd > 32 ? 512 : 1024) / groups);
    const size_t per = (size_t)groups * QV * (c.hd + 2) * sizeof(float);
    if (want > 1) want = std::min<int64_t>(want, std::max<size_t>(1, bytes / per));
    p.nspan = (int)std::min(want, (max_len + least - 1) / least);
    p.least = (int)least;
    if (p.nspan > 1) {
        p.ml = groups * p.nspan * QV * c.hd;
        p.bytes = per * p.nspan;
    }
    return p;
}

template <typename T, int HD>
hipError_t prompt(hipStream_t s, const PagedAttnArgs& a, const PromptPlan& p, float* ws) {
    const int64_t groups = p.tiles * a.c.Hkv, nj = kPromptQv<T> * (HD / 4) / 256;
    const PromptArgs d{a, (int)p.tiles, p.nspan, p.least, ws, p.ml};
    hipError_t err;
    if constexpr (sizeof(T) == 2) err = launch(k_pprompt_bf16<HD>, dim3((unsigned)(groups * p.nspan)), dim3(64 * kPromptWaves), s, d);
    else err = launch(k_pprompt_f32<HD>, dim3((unsigned)(groups * p.nspan)), dim3(256), s, d);
    if (err != hipSuccess || p.nspan == 1) return err;
    return launch(k_prompt_join<T, HD, kPromptQv<T>, sizeof(T) == 2 ? prompt_keys(HD) : 32>, dim3((unsigned)(groups * nj)), dim3(256), s, d);
}

// Whether a call goes to k_pprompt: by the query vectors of a sequence and KV head that share keys.  k_pdecode reads
// the keys once per 32 of them, k_pprompt once per 256 (fp32: 128) and computes whole tiles.  32/8 heads of
// 128, 16 sequences of 2000 positions / one of 20000, us in k_pdecode and in k_pprompt:
//   bf16:  48: 49 and 49 / 32 and 36    68: 75 and 51 / 37 and 38    132: 82 and 61 / 50 and 46
//   fp32: 128: 184 and 195 / 112 and 130    192: 239 and 310 / 212 and 203    224: 306 and 319 / 252 and 207
bool many_rows(const PagedView& c, const PagedRows& r, int H, bool bf16) {
    return (int64_t)r.max_rows * (H / c.Hkv) > (bf16 ? 64 : 192);
}

// Up to kDirect workgroup steps of expected positions a sequence is one unit, which writes its rows itself:
// 517 positions of 8 KV heads take 7.8 us that way, and 7.3 and 3.5 in two launches.
constexpr int kDirect = 6;

struct DecodePlan {
    int nt, ncg, target, units;
    int64_t ml;  // floats of the sums
    size_t bytes;
};

// bytes: room for partials.
DecodePlan decode_plan(const PagedView& c, const PagedRows& r, int H, bool bf16, int64_t max_len, size_t bytes) {
    DecodePlan p;
    const int qv = std::min<int64_t>((int64_t)r.max_rows * (H / c.Hkv), 1 << 20);
    // (blocks of 32 query vectors as two groups that read the keys once each: 62 us, not 49)
    p.nt = qv <= 16 ? 1 : 2;
    p.ncg = (qv + 16 * p.nt - 1) / (16 * p.nt);
    const int64_t groups = (int64_t)c.Hkv * p.ncg;
    // two workgroups per CU, or as many units again as sequences (for 384 / 512 / 768 workgroups 16 fp32 sequences
    // of 256 to 2048 take 41.4 / 36.4 / 44.6 us, and the 905 MB batch 171 / 159 / 161)
    int64_t target = max_len <= kDirect * kDecodeWaves * (bf16 ? 32 : 16) ? 0 : std::max<int64_t>((512 + groups - 1) / groups, r.nseq);
    const size_t per = (size_t)groups * 16 * p.nt * (c.hd + 2) * sizeof(float);
    if (target && per * (target + r.nseq + 8) > bytes) target = std::max<int64_t>(0, (int64_t)(bytes / per) - r.nseq - 8);
    p.target = (int)target;
    p.units = (int)(target ? target + r.nseq + 8 : r.nseq);
    p.ml = target ? (int64_t)p.units * groups * 16 * p.nt * c.hd : 0;
    p.bytes = target ? per * p.units : 0;
    return p;
}

// Workgroups of k_pjoin for a group of 16 nt query vectors.
constexpr int join_blocks(int hd, int nt) { return (16 * nt + 1024 / hd - 1) / (1024 / hd); }

// Whether both launches of a plan have fewer than 2^32 threads, which is what one may have.
bool fits(const PagedView& c, const PagedRows&, bool bf16, const PromptPlan& p) {
    const int64_t groups = p.tiles * c.Hkv, nj = (bf16 ? kPromptQv<uint16_t> : kPromptQv<float>) * (c.hd / 4) / 256;
    return std::max(groups * p.nspan * (bf16 ? 64 * kPromptWaves : 256), p.nspan > 1 ? groups * nj * 256 : 0) <= UINT32_MAX;
}
bool fits(const PagedView& c, const PagedRows& r, bool, const DecodePlan& p) {
    const int64_t per = ((int64_t)p.units * c.Hkv + 7) / 8 * 8, join = p.target ? (int64_t)r.nseq * c.Hkv * join_blocks(c.hd, p.nt) : 0;
    return std::max(per, join) * p.ncg <= UINT32_MAX / 256;
}

template <typename T, int HD, int NT>
hipError_t run_decode(hipStream_t s, const PagedAttnArgs& a, const DecodePlan& p, float* ws) {
    const DecodeArgs d{a, p.ncg, p.target, kDecodeWaves * kBlockKeys<T>, p.units, ws, p.ml};
    const int64_t per = ((int64_t)p.units * a.c.Hkv + 7) / 8 * 8;
    const hipError_t err = launch(k_pdecode<T, HD, NT>, dim3((unsigned)(per * p.ncg)), dim3(64 * kDecodeWaves), s, d);
    if (err != hipSuccess || !p.target) return err;
    constexpr int nb = join_blocks(HD, NT);
    return launch(k_pjoin<T, HD, NT>, dim3((unsigned)(a.r.nseq * a.c.Hkv * p.ncg * nb)), dim3(256), s, d);
}

template <typename T, int HD>
hipError_t decode(hipStream_t s, const PagedAttnArgs& a, int64_t max_len, float* ws, size_t bytes) {
    if (many_rows(a.c, a.r, a.H, sizeof(T) == 2)) return prompt<T, HD>(s, a, prompt_plan(a.c, a.r, a.H, sizeof(T) == 2, max_len, bytes), ws);
    const DecodePlan p = decode_plan(a.c, a.r, a.H, sizeof(T) == 2, max_len, bytes);
    return p.nt == 1 ? run_decode<T, HD, 1>(s, a, p, ws) : run_decode<T, HD, 2>(s, a, p, ws);
}

}  // namespace

size_t paged_attn_bytes(const PagedView& c, const PagedRows& r, int H, bool bf16, int64_t max_len) {
    if (many_rows(c, r, H, bf16)) {
        const PromptPlan p = prompt_plan(c, r, H, bf16, max_len, SIZE_MAX);
        return fits(c, r, bf16, p) ? std::max<size_t>(p.bytes, 256) : 0;
    }
    const DecodePlan p = decode_plan(c, r, H, bf16, max_len, SIZE_MAX);
    return fits(c, r, bf16, p) ? std::max<size_t>(p.bytes, 256) : 0;
}

hipError_t paged_attn(hipStream_t s, const PagedAttnArgs& a, bool bf16, int64_t max_len, void* ws, size_t ws_bytes) {
    float* const w = (float*)ws;
    if (!a.r.total_rows || !a.r.nseq) return hipSuccess;
    switch (a.c.hd) {
        case 32: return bf16 ? decode<uint16_t, 32>(s, a, max_len, w, ws_bytes) : decode<float, 32>(s, a, max_len, w, ws_bytes);
        case 64: return bf16 ? decode<uint16_t, 64>(s, a, max_len, w, ws_bytes) : decode<float, 64>(s, a, max_len, w, ws_bytes);
        case 128: return bf16 ? decode<uint16_t, 128>(s, a, max_len, w, ws_bytes) : decode<float, 128>(s, a, max_len, w, ws_bytes);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace sd2
