// Rows into a paged cache of 8 bits: e4m3 numbers, and a power of two for k and for v of every 16 positions of a KV
// head.
//
// A power of two because a number times it is exact in bf16, as is the number's own change of power but for the
// smallest ones: a block of 16 positions whose largest magnitude grows row by row needs no second rounding of what it
// holds above 2^-6 of the scale.  An e4m3 number has four significant bits whatever its magnitude, so that a finer scale
// would gain nothing but range.
//
// A wave has a unit: up to 16 rows of one sequence that share a block, one KV head, k or v.  It loads them (a lane 8
// neighbouring values of 64 / (hd / 8) rows at a time), takes the largest magnitude over the wave, and writes the
// numbers, 8 bytes a lane, rows of a block one behind the other.
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

__device__ __forceinline__ void load8(const char* p, bool bf16, float (&x)[8]) {
    if (bf16) {
        const uint4 w = *(const uint4*)p;
        const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(d[i]);
            x[2 * i + 1] = bf16_hi(d[i]);
        }
    } else {
        const float4 a = *(const float4*)p, b = *(const float4*)(p + 16);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

template <bool BF16, int HD>
__global__ __launch_bounds__(256) void k_paged_append8(Append8Args a) {
    constexpr int CH = HD / 8, RP = 64 / CH, PASS = 16 / RP, SIZE = BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = 1 << (a.c.shift - 4);
    const int64_t groups = ((int64_t)a.r.total_rows + a.group - 1) / a.group;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        // a lane per row of the group: its position, and whether it is its sequence's first one in a block
        const int64_t mine = g * a.group + lane;
        int pos = -1, b = 0, count = 0;
        if (lane < a.group && mine < a.r.total_rows) {
            b = paged_seq(a.r, (int)mine);
            const SeqRows s = seq_rows(a.r, b);
            const int i = (int)mine - s.r0, p = s.len - s.n + i;
            if (i >= 0 && i < s.n && p >= 0 && (i == 0 || p == 0 || p % 16 == 0)) {
                pos = p;
                count = min(s.n - i, 16 - p % 16);
            }
        }
        uint64_t starts = __ballot(pos >= 0);
        const int n = __popcll(starts) * 2 * a.c.Hkv;
        for (int u = blockIdx.y * 4 + wave; u < n; u += gridDim.y * 4) {
            int which = u / (2 * a.c.Hkv);
            uint64_t m = starts;
            while (which--) m &= m - 1;
            const int l = __builtin_ctzll(m), h = u % (2 * a.c.Hkv) >> 1, kv = u & 1;
            const int row0 = (int)(g * a.group) + l, p0 = __builtin_amdgcn_readlane(pos, l), rows = __builtin_amdgcn_readlane(count, l);
            const int sb = __builtin_amdgcn_readlane(b, l);
            const char* src = kv ? a.v : a.k;
            const int64_t stride = kv ? a.v_stride : a.k_stride;
            const int lr = lane / CH, lc = lane % CH;
            float x[PASS][8];
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < PASS; ++i) {
                const int r = i * RP + lr;
                if (r < rows) load8(src + (row0 + r) * stride + (h * HD + 8 * lc) * SIZE, BF16, x[i]);
            }
            const int page = paged_page(a.c, sb, p0 >> a.c.shift);
            if (page < 0) continue;
            const int slot = p0 & ((1 << a.c.shift) - 1), blk = slot >> 4;
            uint8_t* scale = a.c.scales + page * a.c.scale_stride + ((int64_t)h * blocks + blk) * 2 + kv;
            // (the first slot of a block: whatever it held is over)
            const int was = slot % 16 ? min(max((int)*scale - 127, kLeastPower), kMostPower) : kLeastPower;
#pragma unroll
            for (int i = 0; i < PASS; ++i)
                if (i * RP + lr < rows)
#pragma unroll
                    for (int e = 0; e < 8; ++e) most = fmaxf(most, finite(x[i][e]) ? fabsf(x[i][e]) : 0.f);
            most = wave_max(most);
            const int e = max(power_of(most), was);
            char* to = (char*)(kv ? a.c.v : a.c.k) + page * a.c.page_stride + (((int64_t)h << a.c.shift) + (blk << 4)) * HD;
            if (slot % 16 && e > was) {
                const float by = pow2(max(was - e, -126));  // (beyond 2^-126 nothing is left either way)
#pragma unroll
                for (int i = 0; i < PASS; ++i) {
                    const int r = i * RP + lr;
                    if (r >= slot % 16) continue;
                    uint2* at = (uint2*)(to + r * HD + 8 * lc);
                    float y[8];
                    of_e4m3x8(*at, y);
                    *at = e4m3x8(y, by);
                }
            }
            const float inv = pow2(-e);
#pragma unroll
            for (int i = 0; i < PASS; ++i) {
                const int r = i * RP + lr;
                if (r < rows) *(uint2*)(to + (slot % 16 + r) * HD + 8 * lc) = e4m3x8(x[i], inv);
            }
            if (lane == 0) *scale = (uint8_t)(e + 127);
        }
    }
}

template <bool BF16>
hipError_t append8(hipStream_t s, const Append8Args& a) {
    const int64_t groups = ((int64_t)a.r.total_rows + a.group - 1) / a.group;
    const dim3 grid((unsigned)std::min<int64_t>(groups, kAppendBlocks / 4), (unsigned)std::min((a.c.Hkv + 1) / 2, 4));
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
