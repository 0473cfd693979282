// Rows into a paged cache of 8 bits: e4m3 numbers, and a power of two for k and for v of every 16 positions of a KV
// head.
//
// A power of two because a number times it is exact in bf16, as is the number's own change of power but for the
// smallest ones: a block of 16 positions whose largest magnitude grows row by row needs no second rounding of what it
// holds above 2^-6 of the scale.  An e4m3 number has four significant bits whatever its magnitude, so that a finer scale
// would gain nothing but range.
//
// A wave has a unit: up to 16 rows of one sequence that share a block, and one KV head.  It loads their k and v (a lane 8
// neighbouring values of 64 / (hd / 8) rows at a time), takes the largest magnitudes over the wave, and writes the
// numbers, 8 bytes a lane, rows of a block one behind the other.  Where all magnitudes are finite and a power reaches them, a
// value costs half an instruction for its magnitude (bf16) and half a one to convert; others are looked at one by one.
//
// Bound by the bytes and, for single rows, by a launch and two to three round trips: 36764 bf16 rows of 8 heads of 128
// (226 MB read and written) 54 us, 4.2 TB/s; one fp32 row of each of 16 sequences 4.1 us.  A wave for k and one for v took
// 78 and 71 us; five workgroups a CU instead of four 54, six (to scratch) 63; groups of 32 or 64 rows 55.
#include <algorithm>

#include "device_common.h"
#include "paged.h"

namespace sd2 {

namespace {

struct Append8Args {
    PagedView c;
    PagedRows r;
    const char *k, *v;
    int64_t k_stride, v_stride;  // bytes
    int group;                   // rows of a workgroup, 1 or 16: those whose blocks begin there are its units
};
constexpr int kAppendBlocks = 1 << 22;
// 2^-100 is far above what fp32 loses, and 448 2^119 is a finite bf16.
constexpr int kLeastPower = -100, kMostPower = 119;

// The least e with 448 2^e >= a = 1.m 2^x: x - 8 for 1.m up to 1.75, as 448 = 1.75 2^8.
__device__ __forceinline__ int power_of(float a) {
    const uint32_t bits = __float_as_uint(a);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000);
    return min(max(e, kLeastPower), kMostPower);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in -126 .. 127

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000) != 0x7f800000; }
__device__ __forceinline__ float e4m3_arg(float x, float inv) {
    const float y = x * inv, z = __builtin_amdgcn_fmed3f(y, -448.f, 448.f);
    return finite(x) ? z : NAN;
}
// 8 values as e4m3 numbers.
__device__ __forceinline__ uint2 e4m3x8(const float (&x)[8], float inv) {
    uint2 w;
    int d = 0;
    d = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(x[0], inv), e4m3_arg(x[1], inv), d, false);
    d = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(x[2], inv), e4m3_arg(x[3], inv), d, true);
    w.x = d;
    d = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(x[4], inv), e4m3_arg(x[5], inv), d, false);
    d = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(x[6], inv), e4m3_arg(x[7], inv), d, true);
    w.y = d;
    return w;
}
__device__ __forceinline__ void of_e4m3x8(uint2 w, float (&x)[8]) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(w.x, 0); x[1] = __builtin_amdgcn_cvt_f32_fp8(w.x, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(w.x, 2); x[3] = __builtin_amdgcn_cvt_f32_fp8(w.x, 3);
    x[4] = __builtin_amdgcn_cvt_f32_fp8(w.y, 0); x[5] = __builtin_amdgcn_cvt_f32_fp8(w.y, 1);
    x[6] = __builtin_amdgcn_cvt_f32_fp8(w.y, 2); x[7] = __builtin_amdgcn_cvt_f32_fp8(w.y, 3);
}

// Eight neighbouring values as they lie in memory.
template <bool BF16>
struct Raw {
    uint32_t w[BF16 ? 4 : 8];
};
template <bool BF16>
__device__ __forceinline__ void load8(const char* p, Raw<BF16>& x) {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) {
        const uint4 w = *(const uint4*)(p + 16 * i);
        x.w[4 * i] = w.x; x.w[4 * i + 1] = w.y; x.w[4 * i + 2] = w.z; x.w[4 * i + 3] = w.w;
    }
}
template <bool BF16>
__device__ __forceinline__ void values(const Raw<BF16>& x, float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = BF16 ? (i % 2 ? bf16_hi(x.w[i / 2]) : bf16_lo(x.w[i / 2])) : __uint_as_float(x.w[BF16 ? 0 : i]);
}
// The bits of the largest magnitude, as those of an fp32 number: they are ordered as the magnitudes are, and behind them all
// infinities and NaN.  (bf16: two at a time.)
typedef uint16_t h2 __attribute__((ext_vector_type(2)));
template <bool BF16>
__device__ __forceinline__ void most_bits(const Raw<BF16>& x, uint32_t& m) {
#pragma unroll
    for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
        if constexpr (BF16) m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(h2, m), __builtin_bit_cast(h2, x.w[i] & 0x7fff7fffu)));
        else m = max(m, x.w[i] & 0x7fffffffu);
    }
}
// Their maximum over a wave, through row operations.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_max(int v) {
    return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_most_bits(uint32_t m) {
    int v = (int)m;
    v = dpp_max<0xB1, 0xf>(v);   // quad_perm [1,0,3,2]
    v = dpp_max<0x4E, 0xf>(v);   // quad_perm [2,3,0,1]
    v = dpp_max<0x141, 0xf>(v);  // row_half_mirror
    v = dpp_max<0x140, 0xf>(v);  // row_mirror
    v = dpp_max<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
    v = dpp_max<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane(v, 63);
}
// Eight values, finite and at most 448 of the scale, as e4m3 numbers of it.
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef short s2 __attribute__((ext_vector_type(2)));
template <bool BF16>
__device__ __forceinline__ uint2 e4m3x8_plain(const Raw<BF16>& x, float scale) {
    s2 d[2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (BF16) {
            d[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(d[i], __builtin_bit_cast(b2, x.w[2 * i]), scale, false);
            d[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(d[i], __builtin_bit_cast(b2, x.w[2 * i + 1]), scale, true);
        } else {
            d[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d[i], __uint_as_float(x.w[4 * i]), __uint_as_float(x.w[4 * i + 1]), scale, false);
            d[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d[i], __uint_as_float(x.w[4 * i + 2]), __uint_as_float(x.w[4 * i + 3]), scale, true);
        }
    }
    return make_uint2(__builtin_bit_cast(uint32_t, d[0]), __builtin_bit_cast(uint32_t, d[1]));
}

// Sequence, position and number of rows left in its 16 positions of the row that begins there; count 0: none does.
struct Start {
    int b, pos, count;
};
__device__ __forceinline__ Start start_of(const SeqRows& s, int b, int row) {
    Start t{b, 0, 0};
    const int i = row - s.r0, p = s.len - s.n + i;
    if (i >= 0 && i < s.n && p >= 0 && (i == 0 || p == 0 || p % 16 == 0)) {
        t.pos = p;
        t.count = min(s.n - i, 16 - p % 16);
    }
    return t;
}
// Those of `rows` rows from row0 on, a lane each.
__device__ __forceinline__ Start starts(const PagedRows& r, int64_t row0, int rows) {
    const int lane = threadIdx.x & 63;
    const int64_t row = row0 + lane;
    const bool mine = lane < rows && row < r.total_rows;
    if (r.row_off && r.nseq < 64) {
        // offsets and lengths of all sequences in one round trip, a lane each, and every row's sequence by counting
        const int off = lane <= r.nseq ? r.row_off[lane] : INT32_MAX, len = lane < r.nseq ? r.lens[lane] : 0;
        const uint64_t real = ((uint64_t)1 << r.nseq) - 1;
        int b = 0;
        for (int i = 0; i < rows; ++i) {
            const int c = __popcll(__ballot(off <= row0 + i) & real);
            if (lane == i) b = max(c - 1, 0);
        }
        SeqRows s;
        s.r0 = min(max(__shfl(off, b, 64), 0), r.total_rows);
        s.n = min(min(max(__shfl(off, b + 1, 64), s.r0), r.total_rows) - s.r0, r.max_rows);
        s.len = max(__shfl(len, b, 64), 0);
        return mine ? start_of(s, b, (int)row) : Start{0, 0, 0};
    }
    if (!mine) return Start{0, 0, 0};
    const int b = paged_seq(r, (int)row);
    return start_of(seq_rows(r, b), b, (int)row);
}

template <bool BF16, int HD>
__global__ __launch_bounds__(256) void k_paged_append8(Append8Args a) {
    constexpr int CH = HD / 8, RP = 64 / CH, PASS = 16 / RP, SIZE = BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = 1 << (a.c.shift - 4);
    const int64_t groups = ((int64_t)a.r.total_rows + a.group - 1) / a.group;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const Start st = starts(a.r, g * a.group, a.group);
        const uint64_t found = __ballot(st.count > 0);
        const int n = __popcll(found) * a.c.Hkv;
        for (int u = blockIdx.y * 4 + wave; u < n; u += gridDim.y * 4) {
            int which = u / a.c.Hkv;
            uint64_t m = found;
            while (which--) m &= m - 1;
            const int l = __builtin_ctzll(m), h = u % a.c.Hkv;
            const int row0 = (int)(g * a.group) + l, p0 = __builtin_amdgcn_readlane(st.pos, l), rows = __builtin_amdgcn_readlane(st.count, l);
            const int page = paged_page(a.c, __builtin_amdgcn_readlane(st.b, l), p0 >> a.c.shift);
            const int lr = lane / CH, lc = lane % CH;
            Raw<BF16> x[2][PASS];
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                for (int i = 0; i < PASS; ++i) {
                    const int r = i * RP + lr;
                    const char* p = kv ? a.v + (row0 + r) * a.v_stride : a.k + (row0 + r) * a.k_stride;
                    if (r < rows) load8(p + (h * HD + 8 * lc) * SIZE, x[kv][i]);
                }
            if (page < 0) continue;
            const int slot = p0 & ((1 << a.c.shift) - 1), blk = slot >> 4, before = slot % 16;
            uint8_t* scale = a.c.scales + page * a.c.scale_stride + ((int64_t)h * blocks + blk) * 2;
            // (from the first slot of a block on: whatever it held is over)
            const int held = before ? *(const uint16_t*)scale : 0;
            int e[2];
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < PASS; ++i)
                    if (i * RP + lr < rows) most_bits(x[kv][i], bits);
                if constexpr (BF16) bits = max(bits & 0xffffu, bits >> 16) << 16;
                bits = wave_most_bits(bits);
                float most = __uint_as_float(bits);
                // (infinities, NaN, and magnitudes that no power reaches are looked at one by one)
                const bool plain = bits <= __float_as_uint(448.f) + (kMostPower << 23);
                if (!plain) {
                    most = 0.f;
#pragma unroll
                    for (int i = 0; i < PASS; ++i) {
                        float y[8];
                        values(x[kv][i], y);
                        if (i * RP + lr < rows)
#pragma unroll
                            for (int j = 0; j < 8; ++j) most = fmaxf(most, finite(y[j]) ? fabsf(y[j]) : 0.f);
                    }
                    most = wave_max(most);
                }
                const int was = before ? min(max((held >> 8 * kv & 255) - 127, kLeastPower), kMostPower) : kLeastPower;
                e[kv] = max(power_of(most), was);
                char* to = (char*)(kv ? a.c.v : a.c.k) + page * a.c.page_stride + (((int64_t)h << a.c.shift) + (blk << 4)) * HD;
                if (before && e[kv] > was) {
                    const float by = pow2(max(was - e[kv], -126));  // (beyond 2^-126 nothing is left either way)
#pragma unroll
                    for (int i = 0; i < PASS; ++i) {
                        const int r = i * RP + lr;
                        if (r >= before) continue;
                        uint2* at = (uint2*)(to + r * HD + 8 * lc);
                        float y[8];
                        of_e4m3x8(*at, y);
                        *at = e4m3x8(y, by);
                    }
                }
                const float scale_up = pow2(e[kv]), inv = pow2(-e[kv]);
#pragma unroll
                for (int i = 0; i < PASS; ++i) {
                    const int r = i * RP + lr;
                    uint2 w;
                    if (plain) {
                        w = e4m3x8_plain(x[kv][i], scale_up);
                    } else {
                        float y[8];
                        values(x[kv][i], y);
                        w = e4m3x8(y, inv);
                    }
                    if (r < rows) *(uint2*)(to + (before + r) * HD + 8 * lc) = w;
                }
            }
            if (lane == 0) *(uint16_t*)scale = (uint16_t)(e[0] + 127 | (e[1] + 127) << 8);
        }
    }
}

template <bool BF16>
hipError_t append8(hipStream_t s, const Append8Args& a) {
    const int64_t groups = ((int64_t)a.r.total_rows + a.group - 1) / a.group;
    const dim3 grid((unsigned)std::min<int64_t>(groups, kAppendBlocks / 4), (unsigned)std::min((a.c.Hkv + 3) / 4, 4));
    switch (a.c.hd) {
        case 32: return launch(k_paged_append8<BF16, 32>, grid, dim3(256), s, a);
        case 64: return launch(k_paged_append8<BF16, 64>, grid, dim3(256), s, a);
        case 128: return launch(k_paged_append8<BF16, 128>, grid, dim3(256), s, a);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t paged_append8(hipStream_t s, const PagedView& c, const PagedRows& r, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, bool bf16) {
    if (!r.total_rows || !r.nseq) return hipSuccess;
    const int size = bf16 ? 2 : 4;
    const Append8Args a{c, r, (const char*)k, (const char*)v, k_stride * size, v_stride * size, r.max_rows < 16 ? 1 : 16};
    return bf16 ? append8<true>(s, a) : append8<false>(s, a);
}

}  // namespace sd2
