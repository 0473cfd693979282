// Attention over paged caches of the rows' own type, every position read (paged_attn_kernels.h), and how calls of all kinds
// are planned.
#include "paged_attn_kernels.h"

namespace sd2 {

size_t paged_attn_bytes(const PagedView& c, const PagedRows& r, int H, bool bf16, int64_t max_len, int window, int sinks) {
    max_len = keys_expected(r, max_len, window, sinks);
    if (many_rows(c, r, H, bf16)) {
        const PromptPlan p = prompt_plan(c, r, H, bf16, max_len, SIZE_MAX);
        return fits(c, r, bf16, p) ? std::max<size_t>(p.bytes, 256) : 0;
    }
    const DecodePlan p = decode_plan(c, r, H, bf16, max_len, SIZE_MAX, c.scales || window);
    return fits(c, r, bf16, p) ? std::max<size_t>(p.bytes, 256) : 0;
}

hipError_t paged_attn(hipStream_t s, const PagedAttnArgs& a, bool bf16, int64_t max_len, void* ws, size_t ws_bytes) {
    float* const w = (float*)ws;
    if (!a.r.total_rows || !a.r.nseq) return hipSuccess;
    if (a.c.scales) return bf16 ? paged_attn_scaled_bf16(s, a, max_len, w, ws_bytes) : paged_attn_scaled_f32(s, a, max_len, w, ws_bytes);
    if (a.window) return paged_attn_window(s, a, bf16, max_len, w, ws_bytes);
    return bf16 ? attn_of<uint16_t, uint16_t, false>(s, a, max_len, w, ws_bytes) : attn_of<float, float, false>(s, a, max_len, w, ws_bytes);
}

}  // namespace sd2
