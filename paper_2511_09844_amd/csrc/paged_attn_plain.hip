// Attention over a paged cache of 8 bits, or under a window: a wave per row and head, a lane per key.
#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "paged.h"

namespace sd2 {

namespace {

__device__ __forceinline__ float value(const PagedAttnArgs& a, bool bf16, const void* pool, int which, int page, int h, int slot, int i) {
    const int64_t at = page * a.c.page_stride + (((int64_t)h << a.c.shift) + slot) * a.c.hd + i;
    if (!a.c.scales) return bf16 ? bf16_to_f32(((const uint16_t*)pool)[at]) : ((const float*)pool)[at];
    const int b = a.c.scales[page * a.c.scale_stride + (((int64_t)h << (a.c.shift - 4)) + (slot >> 4)) * 2 + which];
    return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)pool)[at], 0) * __uint_as_float((uint32_t)b << 23);
}

__global__ __launch_bounds__(256) void k_attn_plain(PagedAttnArgs a, bool bf16) {
    const int lane = threadIdx.x & 63, hd = a.c.hd, mask = (1 << a.c.shift) - 1;
    const int64_t n = (int64_t)a.r.total_rows * a.H;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < n; u += (int64_t)gridDim.x * 4) {
        const int row = u / a.H, h = u % a.H, kvh = h / (a.H / a.c.Hkv), b = paged_seq(a.r, row);
        const SeqRows s = seq_rows(a.r, b);
        if (row < s.r0 || row >= s.r0 + s.n) continue;
        const int pos = s.len - s.n + row - s.r0;
        const int end = (int)min((int64_t)pos + 1, (int64_t)a.c.max_pages << a.c.shift);
        auto qv = [&](int i) {
            const int64_t at = row * a.q_stride + h * hd + i;
            return bf16 ? bf16_to_f32(((const uint16_t*)a.q)[at]) : ((const float*)a.q)[at];
        };
        float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
        bool any = false;
        for (int k0 = 0; k0 < end; k0 += 64) {
            const int j = k0 + lane;
            const bool read = j < end && (!a.window || pos - j < a.window || j < a.sinks);
            const int page = read ? paged_page(a.c, b, j >> a.c.shift) : -1;
            float sc = -INFINITY;
            if (page >= 0) {
                sc = 0.f;
                for (int i = 0; i < hd; ++i) sc += qv(i) * value(a, bf16, a.c.k, 0, page, kvh, j & mask, i);
                sc *= a.scale;
            }
            any |= __any(page >= 0);
            const float mn = fmaxf(m, wave_max(sc)), base = mn == -INFINITY ? 0.f : mn, f = expf(m - base);
            const float w = page >= 0 ? expf(sc - base) : 0.f;
            m = mn;
            l = l * f + wave_sum(w);
            o[0] *= f;
            o[1] *= f;
            for (int t = 0; t < 64 && k0 + t < end; ++t) {
                const int pg = __shfl(page, t, 64);
                const float wt = __shfl(w, t, 64);
                if (pg < 0) continue;
                for (int i = 0; i < 2; ++i)
                    if (lane + 64 * i < hd) o[i] += wt * value(a, bf16, a.c.v, 1, pg, kvh, (k0 + t) & mask, lane + 64 * i);
            }
        }
        for (int i = 0; i < 2; ++i)
            if (lane + 64 * i < hd) {
                const float y = l > 0.f ? o[i] / l : l == l && !any ? 0.f : NAN;
                const int64_t at = row * a.out_stride + h * hd + lane + 64 * i;
                if (bf16) ((__bf16*)a.out)[at] = (__bf16)y;
                else ((float*)a.out)[at] = y;
            }
    }
}

}  // namespace

hipError_t paged_attn_plain(hipStream_t s, const PagedAttnArgs& a, bool bf16) {
    const int64_t n = ((int64_t)a.r.total_rows * a.H + 3) / 4;
    return launch(k_attn_plain, dim3((unsigned)std::min<int64_t>(n, 1 << 20)), dim3(256), s, a, bf16);
}

}  // namespace sd2
