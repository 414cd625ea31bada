// Device helpers of the operators on a cache held in 8 bits.
//
// Codes lie in the pool as a layout view arranges bf16 rows, one byte an element; token t's plane of head h (of the row) has the scale
//   scales[block][plane][(slot / B_base) * row_heads + h],
// B_base tokens of a head to a scale, n_kv_heads scales a plane under every view (B(p) / B_base groups of H_row heads).
#pragma once

#include "decode_common.h"

namespace kvq8 {

using namespace kvdec;

constexpr int kE4M3 = KV_Q8_E4M3, kInt8 = KV_Q8_INT8;

// What a kernel needs to know of a view beside kv_view_dev (whose elements are bytes here).
struct q8_view {
    int32_t base_tokens;   // B_base
    int32_t base_shift;    // log2, or -1
    int32_t row_heads;     // heads in a stored row
    int32_t row_head0;     // the first exposed one
    int32_t block_scales;  // scales of a block, both planes
};
static inline q8_view q8_view_of(const kv_view* v)
{
    q8_view x;
    x.base_tokens = v->geom.base_block_size;
    x.base_shift = -1;
    for (int s = 0; s < 31; ++s)
        if ((1 << s) == x.base_tokens) x.base_shift = s;
    x.row_heads = v->row_heads;
    x.row_head0 = v->row_head0;
    x.block_scales = 2 * v->geom.n_kv_heads;
    return x;
}
static inline bool q8_format_ok(int format) { return format == kE4M3 || format == kInt8; }

// Place of the scale of local head h, plane 0, of the tokens around `slot` of a block (plane 1: block_scales / 2 on).
__device__ __forceinline__ int64_t q8_scale_at(const q8_view& x, int64_t block, int slot, int h)
{
    const int group = x.base_shift >= 0 ? slot >> x.base_shift : slot / x.base_tokens;
    return block * x.block_scales + group * x.row_heads + x.row_head0 + h;
}

// Two codes of a dword (HI: the upper two) as two bf16: exact in either format (e4m3 has four significant bits, int8 eight).
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t two_bf16(uint32_t codes)
{
    if constexpr (FMT == kE4M3) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, HI));
    } else {
        const int lo = (int)(int8_t)(codes >> (HI ? 16 : 0)), hi = (int)(int8_t)(codes >> (HI ? 24 : 8));
        return pack_bf16x2((float)lo, (float)hi);
    }
}
// The same as floats.
template <int FMT, bool HI>
__device__ __forceinline__ f32x2 two_f32(uint32_t codes)
{
    if constexpr (FMT == kE4M3) {
        return __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, HI);
    } else {
        return f32x2{(float)(int)(int8_t)(codes >> (HI ? 16 : 0)), (float)(int)(int8_t)(codes >> (HI ? 24 : 8))};
    }
}

// Four numbers, no larger than the largest code but for a rounding, to the nearest codes (ties to the even one).
template <int FMT>
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d)
{
    if constexpr (FMT == kE4M3) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
    } else {
        const uint32_t i = (uint8_t)(int)rintf(a), j = (uint8_t)(int)rintf(b), k = (uint8_t)(int)rintf(c), l = (uint8_t)(int)rintf(d);
        return i | j << 8 | k << 16 | l << 24;
    }
}

// The scale for numbers of up to an absolute value (its bits; infinities and NaN lie above): the smallest power of two that brings it
// down to the largest code, 448 = 1.75 2^8 or 127 = 1.984375 2^6, at least 2^-120; NaN where a number is not finite.
constexpr int kLeastExponent = -120;
constexpr uint32_t kNaNBits = 0x7fc00000u;
template <int FMT>
__device__ __forceinline__ float scale_for(uint32_t top)
{
    if (top >= 0x7f800000u) return __uint_as_float(kNaNBits);
    const int e = (int)(top >> 23) - 127;
    const uint32_t part = top & 0x7fffffu;
    const int s = FMT == kE4M3 ? e - 8 + (part > 0x600000u) : e - 6 + (part > 0x7e0000u);
    return __uint_as_float((uint32_t)(max(s, kLeastExponent) + 127) << 23);
}

// K's scale as attention takes it: NaN for an infinity.  (A score times an infinity may be -inf, whose weight is 0: the group would be left out.)
__device__ __forceinline__ float key_scale(float s)
{
    return (__float_as_uint(s) & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(kNaNBits) : s;
}

}  // namespace kvq8
