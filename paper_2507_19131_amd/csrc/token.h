// int8 codes with one scale a row (a token, or a channel of weights): what the quantizer, the linear layers and the group norm share.
#pragma once
#include "activations.h"
#include "scaled.h"

namespace mixaq {

constexpr float I8_MAX = 127.0f;

// ---- the scale of a row: NaN if it holds a NaN or an infinity -----------------------------------------------------------------
struct RowScale { float scale, inv; };
__device__ __forceinline__ RowScale row_scale(unsigned largest)
{
    RowScale s;
    s.scale = fmaxf(__uint_as_float(largest), LEAST_MAGNITUDE) / I8_MAX;
    s.inv = 1.0f / s.scale;
    if (largest >= 0x7f800000u) {
        s.scale = __uint_as_float(0x7fc00000u);
        s.inv = 0.0f;
    }
    return s;
}
// Four codes, the first in the low byte.  v * inv may pass 127 by its roundings, by 2^-22 of it: the nearest integer is 127 all the same.  Of a row without
// a scale inv is 0, as it is of no other: all codes 0.
__device__ __forceinline__ int int_codes4(float a, float b, float c, float d, float inv)
{
    const int w = pack4(__float_as_int(a * inv + RND_MAGIC), __float_as_int(b * inv + RND_MAGIC), __float_as_int(c * inv + RND_MAGIC),
                        __float_as_int(d * inv + RND_MAGIC));
    return inv == 0.0f ? 0 : w;
}
template <bool TINY>
__device__ __forceinline__ void store_int_codes8(int8_t* row, Eight c, int C, const float v[8], float inv)
{
    const int w[2] = {int_codes4(v[0], v[1], v[2], v[3], inv), int_codes4(v[4], v[5], v[6], v[7], inv)};
    int8_t t[8];
    __builtin_memcpy(t, w, 8);
    put8<TINY>(row, c, C, t);
}

// ---- host ---------------------------------------------------------------------------------------------------------
enum { VALUES = 1, CODES = 2 };
// The matrix `m` as an argument called `name`; allowed: of VALUES and CODES
int check_token_rows(const mixaq_rows* m, const char* name, int32_t columns, int allowed);
inline Extent token_scales_of(const mixaq_rows& m, int32_t rows)                          // (no rows where there are none)
{
    return {(uintptr_t)m.scales, (long long)rows * 4, m.type == MIXAQ_I8 ? 1 : 0, (long long)rows * 4};
}
inline Extent memory_of(const void* p, long long bytes) { return {(uintptr_t)p, bytes, p ? 1 : 0, bytes}; }
inline int round_up16(int v) { return (v + 15) / 16 * 16; }
inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
// mixaq_token_quantize behind its checks
int launch_token_quantize(const mixaq_rows& x, int32_t rows, int32_t columns, const mixaq_rows& q, hipStream_t st);

}  // namespace mixaq
