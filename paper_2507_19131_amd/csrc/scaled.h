// 8-bit float codes with a scale per block of 128 columns: what the quantizer, the linear layers and the norms share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mixaq.h"
#include "mixaq_dev.h"

namespace mixaq {

int fail(int code, const char* fmt, ...);

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int SBLOCK = 128;              // columns that share a scale = the depth of one 16 x 16 x 128 matrix instruction
constexpr float E4M3_MAX = 448.0f;
constexpr float LEAST_MAGNITUDE = 0x1p-100f;      // scales stay normal numbers, their inverses too

// ---- values of the three float types, eight at a time -------------------------------------------------------
template <int TYPE> struct TypeOf;
template <> struct TypeOf<MIXAQ_F32> { using T = float; };
template <> struct TypeOf<MIXAQ_F16> { using T = _Float16; };
template <> struct TypeOf<MIXAQ_BF16> { using T = __bf16; };

// n of the eight values from p on (all of them: n >= 8), zero for the others.  Global memory takes vector accesses at any address, so
// rows of odd stride need no form of their own; only the values that lie behind the row's end are taken one by one.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float v[8])
{
    T t[8];
    if (n >= 8) {
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? (float)p[e] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float v[8])
{
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (T)v[e];
    if (n >= 8) {
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = t[e];
    }
}

// ---- the scale of a block -------------------------------------------------------------------------------------
// Magnitudes are compared as bit patterns, which order like the numbers with infinity and then NaN on top: a block that holds one
// cannot hide it.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ unsigned max_magnitude(const float v[8])
{
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[e]));
    return m;
}
struct BlockScale { float scale, inv; };           // both NaN for a block that holds a NaN or an infinity
__device__ __forceinline__ BlockScale block_scale(unsigned largest)
{
    BlockScale s;
    s.scale = fmaxf(__uint_as_float(largest), LEAST_MAGNITUDE) / E4M3_MAX;
    s.inv = 1.0f / s.scale;
    if (largest >= 0x7f800000u) s.scale = s.inv = __uint_as_float(0x7fc00000u);
    return s;
}
// four codes, the first in the low byte.  v * inv may pass 448 by its rounding: clamped, as the conversion would make it a NaN.
__device__ __forceinline__ int codes4(float a, float b, float c, float d, float inv)
{
    const auto q = [&](float v) { return __builtin_amdgcn_fmed3f(v * inv, -E4M3_MAX, E4M3_MAX); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), w, true);
    return inv == inv ? w : 0x7f7f7f7f;
}
__device__ __forceinline__ void store_codes8(uint8_t* p, int n, const float v[8], float inv)
{
    const int w[2] = {codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv)};
    if (n >= 8) {
        __builtin_memcpy(p, w, 8);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
    }
}
// over the 16 lanes that hold a block of 128 columns, eight each
__device__ __forceinline__ unsigned max16(unsigned m)
{
#pragma unroll
    for (int d = 8; d; d >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, d, 64));
    return m;
}

// ---- host ---------------------------------------------------------------------------------------------------------
constexpr long long MOST_THREADS = 1LL << 32;      // of one launch

inline int size_of(int type) { return type == MIXAQ_F32 ? 4 : type == MIXAQ_E4M3 ? 1 : 2; }
inline int blocks_of(int columns) { return (columns + SBLOCK - 1) / SBLOCK; }

// The matrix `m` as an argument called `name`: `columns` values or codes a row, scales for `scale_rows` rows.
int check_rows(const mixaq_rows* m, const char* name, int32_t columns, bool codes_allowed, int32_t scale_rows);
// Whether writing one matrix touches the other.  Column ranges of one larger matrix do not.
bool rows_overlap(const mixaq_rows& a, int32_t rows_a, int32_t columns_a, const mixaq_rows& b, int32_t rows_b, int32_t columns_b);
// mixaq_scaled_quantize behind its checks
int launch_quantize(const mixaq_rows& x, int32_t rows, int32_t columns, int32_t block_rows, const mixaq_rows& q, hipStream_t st);

}  // namespace mixaq
