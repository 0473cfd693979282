// Causal grouped-query attention over a paged K/V cache.
#include <math.h>

#include "device_common.h"
#include "paged.h"
#include "pgemm.h"

namespace sd2 {

template <typename T>
__device__ __forceinline__ void paged_put1(const PagedAttnArgs& a, int row, int c, float v);
template <>
__device__ __forceinline__ void paged_put1<float>(const PagedAttnArgs& a, int row, int c, float v) {
    if (a.planes) pg_put1(a.planes, a.Mp, row, c, v);
    else ((float*)a.out)[row * a.out_stride + c] = v;
}
template <>
__device__ __forceinline__ void paged_put1<uint16_t>(const PagedAttnArgs& a, int row, int c, float v) {
    const __bf16 h = (__bf16)v;
    ((uint16_t*)a.out)[row * a.out_stride + c] = __builtin_bit_cast(uint16_t, h);
}

// One wave per row and head, a key at a time.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_attn(PagedAttnArgs a) {
    constexpr int E = (HD + 63) / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x;
    const int b = paged_seq(a.r, row);
    int n;
    const int r0 = paged_rows(a.r, b, n);
    if (row < r0 || row >= r0 + n) return;
    const int pos = paged_len(a.r, b, r0, n) - n + (row - r0);
    const int G = a.H / a.c.Hkv;
    for (int h = wave; h < a.H; h += 4) {
        const int kvh = h / G;
        float q[E], o[E], m = -INFINITY, l = 0.f;
        for (int e = 0; e < E; ++e) {
            const int d = lane + 64 * e;
            q[e] = d < HD ? load_scalar<T>((const T*)a.q, row * a.q_stride + h * HD + d) * a.scale : 0.f;
            o[e] = 0.f;
        }
        for (int j = 0; j <= pos; ++j) {
            const int p = paged_page(a.c, b, j >> a.c.shift);
            if (p < 0) continue;
            const int64_t at = p * a.c.page_stride + (((int64_t)kvh << a.c.shift) + (j & ((1 << a.c.shift) - 1))) * HD;
            float s = 0.f;
            for (int e = 0; e < E; ++e) {
                const int d = lane + 64 * e;
                if (d < HD) s += q[e] * load_scalar<T>((const T*)a.c.k, at + d);
            }
            s = wave_sum(s);
            const float mn = fmaxf(m, s), w = expf(s - mn), f = m == -INFINITY ? 0.f : expf(m - mn);
            m = mn;
            l = l * f + w;
            for (int e = 0; e < E; ++e) {
                const int d = lane + 64 * e;
                if (d < HD) o[e] = o[e] * f + w * load_scalar<T>((const T*)a.c.v, at + d);
            }
        }
        for (int e = 0; e < E; ++e) {
            const int d = lane + 64 * e;
            if (d < HD) paged_put1<T>(a, row, h * HD + d, l > 0.f ? o[e] / l : 0.f);
        }
    }
}

size_t paged_attn_bytes(const PagedView&, const PagedRows&, int, bool, int64_t) { return 256; }

hipError_t paged_attn(hipStream_t s, const PagedAttnArgs& a, bool bf16, int64_t, void*, size_t, hipEvent_t, hipEvent_t) {
    if (!a.r.total_rows || !a.r.nseq) return hipSuccess;
    const dim3 grid(a.r.total_rows), block(256);
    switch (a.c.hd) {
        case 32: return launch(bf16 ? k_paged_attn<uint16_t, 32> : k_paged_attn<float, 32>, grid, block, s, a);
        case 64: return launch(bf16 ? k_paged_attn<uint16_t, 64> : k_paged_attn<float, 64>, grid, block, s, a);
        case 128: return launch(bf16 ? k_paged_attn<uint16_t, 128> : k_paged_attn<float, 128>, grid, block, s, a);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace sd2
