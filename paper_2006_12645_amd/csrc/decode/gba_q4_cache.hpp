// gba_q4_cache.hpp -- the cache in 4 bits: sizes and checks of its stored form.
#pragma once

#include "gba_decode.hpp"

namespace gba {

// Below this the inverse of a scale may be infinite: such a group is stored as
// its lowest value.
constexpr float SMALLEST_SCALE = 0x1p-100f;

// The offset of a group before its rounding: low + 8 scale, rounded once.  8 scale
// has no place in fp32 where a group spans nearly all of bf16, so the product is
// part of the sum whatever the compiler contracts.
__host__ __device__ __forceinline__ float q4_offset(float low, float scale) { return __builtin_fmaf(8.f, scale, low); }

// Elements of a stored row: dim, padded.
inline int q4_width(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

inline gba_status validate_q4_cache(const gba_q4_cache &c)
{
    if (!is_dtype(c.dtype) || (c.group != 32 && c.group != 64 && c.group != 128)) return GBA_EINVAL;
    if (c.num_blocks < 0 || c.block_size < 1 || c.heads < 0 || c.dim < 0) return GBA_EINVAL;
    if (c.num_blocks > INT_MAX || c.block_size > INT_MAX || c.heads > 65535 || c.num_blocks * c.block_size > INT_MAX ||
        c.block_size % 16 != 0 || c.dim % 8 != 0 || c.dim > 256)
        return GBA_EUNSUPPORTED;
    if (c.num_blocks == 0 || c.heads == 0 || c.dim == 0) return GBA_OK;
    if (c.k_codes == nullptr || c.v_codes == nullptr || c.k_scales == nullptr || c.v_scales == nullptr) return GBA_EINVAL;
    if (!aligned_to(c.k_codes, 16) || !aligned_to(c.v_codes, 16) || !aligned_to(c.k_scales, 16) || !aligned_to(c.v_scales, 16))
        return GBA_EUNSUPPORTED;
    return GBA_OK;
}

}  // namespace gba
