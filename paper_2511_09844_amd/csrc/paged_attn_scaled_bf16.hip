// Attention of bf16 rows over paged caches of 8 bits.
#include "paged_attn_kernels.h"

namespace sd2 {

hipError_t paged_attn_scaled_bf16(hipStream_t s, const PagedAttnArgs& a, int64_t max_len, float* ws, size_t bytes) {
    return a.window ? attn_of<uint16_t, uint8_t, true>(s, a, max_len, ws, bytes) : attn_of<uint16_t, uint8_t, false>(s, a, max_len, ws, bytes);
}

}  // namespace sd2
