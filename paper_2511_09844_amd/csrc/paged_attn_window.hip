// Attention over paged caches of the rows' own type, under a window.
#include "paged_attn_kernels.h"

namespace sd2 {

hipError_t paged_attn_window(hipStream_t s, const PagedAttnArgs& a, bool bf16, int64_t max_len, float* ws, size_t bytes) {
    return bf16 ? attn_of<uint16_t, uint16_t, true>(s, a, max_len, ws, bytes) : attn_of<float, float, true>(s, a, max_len, ws, bytes);
}

}  // namespace sd2
