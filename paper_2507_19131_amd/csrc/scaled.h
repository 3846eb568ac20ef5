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
template <> struct TypeOf<MIXAQ_E4M3> { using T = uint8_t; };

// A lane's eight columns.  The last lane of a row of C columns takes its last eight, and of those only the ones from `first` on are its
// own; lanes behind the row take the same and own none.  So every load is whole and in the row, without a branch between it and the next one, and
// rows of any stride and length take the same path: global memory takes vector accesses at any address.  (Of fewer than eight columns lane 0 owns
// all, one by one: TINY.)
struct Eight { int at, first; };
template <bool TINY>
__device__ __forceinline__ Eight place8(int col, int C)
{
    if (TINY) return {0, col == 0 ? 0 : 8};
    const int at = min(col, C - 8);
    return {at, min(col - at, 8)};
}
template <bool TINY, typename T>
__device__ __forceinline__ void load8(const T* row, Eight c, int C, T t[8])
{
    if constexpr (TINY) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = e < C ? row[e] : (T)0.0f;
    } else {
        __builtin_memcpy(t, row + c.at, 8 * sizeof(T));
    }
}
template <bool TINY, typename T>
__device__ __forceinline__ void load8f(const T* row, Eight c, int C, float v[8])
{
    T t[8];
    load8<TINY>(row, c, C, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
}
// whether element e of a lane's eight is its own
template <bool TINY>
__device__ __forceinline__ bool own8(Eight c, int e, int C) { return e >= c.first && (!TINY || e < C); }

template <bool TINY, typename T>
__device__ __forceinline__ void put8(T* row, Eight c, int C, const T t[8])
{
    if (!TINY && c.first == 0) {
        __builtin_memcpy(row + c.at, t, 8 * sizeof(T));
    } else if (c.first < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (own8<TINY>(c, e, C)) row[c.at + e] = t[e];
    }
}
template <bool TINY, typename T>
__device__ __forceinline__ void store8(T* row, Eight c, int C, const float v[8])
{
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (T)v[e];
    put8<TINY>(row, c, C, t);
}

// ---- the scale of a block -------------------------------------------------------------------------------------
// Magnitudes are compared as bit patterns, which order like the numbers with infinity and then NaN on top: a block that holds one
// cannot hide it.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
template <bool TINY>
__device__ __forceinline__ unsigned max_magnitude(Eight c, int C, const float v[8])
{
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, own8<TINY>(c, e, C) ? magnitude(v[e]) : 0u);
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
// four codes, the first in the low byte.  v * inv may pass 448 by its roundings, by 2^-22 of it: the nearest code is 448 all the same.
__device__ __forceinline__ int codes4(float a, float b, float c, float d, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
    return inv == inv ? w : 0x7f7f7f7f;
}
template <bool TINY>
__device__ __forceinline__ void store_codes8(uint8_t* row, Eight c, int C, const float v[8], float inv)
{
    const int w[2] = {codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv)};
    uint8_t t[8];
    __builtin_memcpy(t, w, 8);
    put8<TINY>(row, c, C, t);
}

// ---- exchanges between lanes, all in the vector unit ------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int LANES, typename Op>
__device__ __forceinline__ unsigned over_few(unsigned v, Op op)       // of 4 or 16 neighbouring lanes
{
    static_assert(LANES == 4 || LANES == 16, "");
    v = op(v, dpp<0xB1>(v));                                          // neighbours
    v = op(v, dpp<0x4E>(v));                                          // pairs
    if constexpr (LANES == 4) return v;
    v = op(v, dpp<0x141>(v));                                         // quads, by the mirror of eight lanes
    return op(v, dpp<0x140>(v));                                      // eights, by the mirror of 16
}
template <typename Op>
__device__ __forceinline__ unsigned over16(unsigned v, Op op) { return over_few<16>(v, op); }
template <typename Op>
__device__ __forceinline__ unsigned over4rows(unsigned v, Op op)      // of the four lanes l, l + 16, l + 32, l + 48
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return op(b[0], b[1]);
}
template <typename Op>
__device__ __forceinline__ unsigned over64(unsigned v, Op op) { return over4rows(over16(v, op), op); }
struct MaxOf { __device__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); } };
struct SumOf { __device__ unsigned operator()(unsigned a, unsigned b) const { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); } };
__device__ __forceinline__ unsigned max16(unsigned m) { return over16(m, MaxOf()); }

// ---- host ---------------------------------------------------------------------------------------------------------
// A call that fails (a creation without memory) leaves its error with the runtime, where the caller's next launch would find it.
#define HIP_TRY(expr)                                                                                        \
    do {                                                                                                     \
        hipError_t e_ = (expr);                                                                              \
        if (e_ != hipSuccess) {                                                                              \
            (void)hipGetLastError();                                                                         \
            return fail(MIXAQ_E_HIP, "%s failed: %s", #expr, hipGetErrorString(e_));                         \
        }                                                                                                    \
    } while (0)

constexpr long long MOST_THREADS = 1LL << 32;      // of one launch

inline int size_of(int type) { return type == MIXAQ_F32 ? 4 : type >= MIXAQ_E4M3 ? 1 : 2; }
inline int blocks_of(int columns) { return (columns - 1) / SBLOCK + 1; }       // of at least one; up to the largest int

// The matrix `m` as an argument called `name`: `columns` values or codes a row, scales for `scale_rows` rows.
int check_rows(const mixaq_rows* m, const char* name, int32_t columns, bool codes_allowed, int32_t scale_rows);
constexpr int32_t MOST_ROWS = 1 << 30;
// Memory of an argument: `rows` runs of `width` bytes, `stride` apart.
struct Extent {
    uintptr_t at;
    long long stride, rows, width;
};
inline Extent extent_of(const mixaq_rows& m, int32_t rows, int32_t columns)
{
    return {(uintptr_t)m.data, (long long)m.stride * size_of(m.type), rows, (long long)columns * size_of(m.type)};
}
inline Extent scales_of(const mixaq_rows& m, int32_t scale_rows, int32_t columns)        // (no rows where there are none)
{
    return {(uintptr_t)m.scales, (long long)m.scale_stride * 4, m.type == MIXAQ_E4M3 ? blocks_of(columns) : 0, (long long)scale_rows * 4};
}
// Whether writing one touches the other.  Column ranges of one larger matrix do not.
bool overlap(const Extent& a, const Extent& b);
// mixaq_scaled_quantize behind its checks
int launch_quantize(const mixaq_rows& x, int32_t rows, int32_t columns, int32_t block_rows, const mixaq_rows& q, hipStream_t st);

}  // namespace mixaq
