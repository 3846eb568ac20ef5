// Values to int8 codes with one scale a row, and the checks of such matrices.
#include "token.h"

#include <algorithm>

using namespace mixaq;

namespace mixaq {

int check_token_rows(const mixaq_rows* m, const char* name, int32_t columns, int allowed)
{
    if (!m || !m->data) return fail(MIXAQ_E_NULL, "%s is NULL", name);
    if (m->type != MIXAQ_I8) {
        if (m->type == MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "%s: e4m3 codes are not int8 codes", name);
        if (!(allowed & VALUES)) return fail(MIXAQ_E_SHAPE, "%s must be int8 codes", name);
        return check_rows(m, name, columns, false, 0);
    }
    if (!(allowed & CODES)) return fail(MIXAQ_E_SHAPE, "%s must be values", name);
    if (m->stride < columns) return fail(MIXAQ_E_SHAPE, "%s: stride %lld of %d columns", name, (long long)m->stride, columns);
    if (m->stride > (1LL << 40)) return fail(MIXAQ_E_SHAPE, "%s: stride %lld is too large", name, (long long)m->stride);
    if (!m->scales) return fail(MIXAQ_E_NULL, "%s: scales is NULL", name);
    if ((uintptr_t)m->scales % 4) return fail(MIXAQ_E_SHAPE, "%s: scales are not aligned", name);
    if ((uintptr_t)m->data % 16 || m->stride % 16)
        return fail(MIXAQ_E_SHAPE, "%s: codes and their stride must be multiples of 16 bytes (stride %lld)", name, (long long)m->stride);
    return MIXAQ_OK;
}

}  // namespace mixaq

namespace {

struct QuantArgs {
    const void* x;
    long long ldx;
    int8_t* codes;
    long long ldc;
    float* scales;
    int rows, cols;
};

// The largest magnitude of a row that G neighbouring lanes hold; of more than a wave through LDS (`part`: a place per wave; the caller's rows are a
// barrier apart).
template <int G>
__device__ __forceinline__ unsigned row_top(unsigned m, unsigned* part)
{
    if constexpr (G == 16) return max16(m);
    m = over64(m, MaxOf());
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
        m = part[0];
#pragma unroll
        for (int w = 1; w < G / 64; ++w) m = max(m, part[w]);
    }
    return m;
}

// A row is V times eight values in each of G lanes, held in registers between its maximum and its codes: one read of the values.  What bounds it is memory: 68208 x
// 384 of bf16 13.3 us, 5.9 TB/s (inputs in turn that the last-level cache holds in part), 16384 x 4096 36.6, 5.5 TB/s.  (Codes stored past the caches: 13.1 and 34.9,
// but the layer that reads them then takes longer by far, 1024 inputs a row through two layers 313 us instead of 214.)
template <typename T, int G, int V, bool TINY>
__global__ __launch_bounds__(256) void token_quantize_kernel(QuantArgs A)
{
    __shared__ unsigned part[4];
    const int l = threadIdx.x % G;
    const long long row = (long long)blockIdx.x * (256 / G) + threadIdx.x / G, at = min(row, (long long)A.rows - 1);
    const T* const from = (const T*)A.x + at * A.ldx;
    Eight c[V];
    float v[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        c[j] = place8<TINY>((j * G + l) * 8, A.cols);
        load8f<TINY>(from, c[j], A.cols, v[j]);
    }
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) m = max(m, max_magnitude<TINY>(c[j], A.cols, v[j]));
    const RowScale s = row_scale(row_top<G>(m, part));
    if (row >= A.rows) return;
#pragma unroll
    for (int j = 0; j < V; ++j) store_int_codes8<TINY>(A.codes + row * A.ldc, c[j], A.cols, v[j], s.inv);
    if (l == 0) A.scales[row] = s.scale;
}

// Rows that no workgroup's registers hold: read twice.
template <typename T>
__global__ __launch_bounds__(1024) void token_quantize_wide_kernel(QuantArgs A)
{
    __shared__ unsigned part[16];
    const long long row = blockIdx.x;
    const T* const from = (const T*)A.x + row * A.ldx;
    float v[8];
    unsigned m = 0;
    for (long long col = threadIdx.x * 8; col < A.cols; col += 8192) {
        load8f<false>(from, place8<false>((int)col, A.cols), A.cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[e]));
    }
    const RowScale s = row_scale(row_top<1024>(m, part));
    for (long long col = threadIdx.x * 8; col < A.cols; col += 8192) {
        const Eight c = place8<false>((int)col, A.cols);
        load8f<false>(from, c, A.cols, v);
        store_int_codes8<false>(A.codes + row * A.ldc, c, A.cols, v, s.inv);
    }
    if (threadIdx.x == 0) A.scales[row] = s.scale;
}

template <typename T, int G, int V, bool TINY = false>
long long launch(const QuantArgs& A, hipStream_t st)
{
    const long long blocks = ((long long)A.rows + 256 / G - 1) / (256 / G);
    if (blocks * 256 >= MOST_THREADS) return blocks;
    hipLaunchKernelGGL((token_quantize_kernel<T, G, V, TINY>), dim3((unsigned)blocks), dim3(256), 0, st, A);
    return 0;
}
template <int TYPE>
long long launch_type(const QuantArgs& A, hipStream_t st)         // 0, or the workgroups that are too many
{
    using T = typename TypeOf<TYPE>::T;
    const int C = A.cols;
    if (C < 8) return launch<T, 16, 1, true>(A, st);
    if (C <= 128) return launch<T, 16, 1>(A, st);
    if (C <= 256) return launch<T, 16, 2>(A, st);
    if (C <= 384) return launch<T, 16, 3>(A, st);
    if (C <= 512) return launch<T, 16, 4>(A, st);
    if (C <= 1024) return launch<T, 64, 2>(A, st);
    if (C <= 1536) return launch<T, 64, 3>(A, st);
    if (C <= 2048) return launch<T, 64, 4>(A, st);
    if (C <= 4096) return launch<T, 256, 2>(A, st);
    if (C <= 8192) return launch<T, 256, 4>(A, st);
    if (A.rows * 1024LL >= MOST_THREADS) return A.rows;
    hipLaunchKernelGGL((token_quantize_wide_kernel<T>), dim3((unsigned)A.rows), dim3(1024), 0, st, A);
    return 0;
}

}  // namespace

namespace mixaq {

int launch_token_quantize(const mixaq_rows& x, int32_t rows, int32_t columns, const mixaq_rows& q, hipStream_t st)
{
    const QuantArgs A = {x.data, (long long)x.stride, (int8_t*)q.data, (long long)q.stride, q.scales, rows, columns};
    const long long over = x.type == MIXAQ_F32 ? launch_type<MIXAQ_F32>(A, st) : x.type == MIXAQ_F16 ? launch_type<MIXAQ_F16>(A, st) : launch_type<MIXAQ_BF16>(A, st);
    if (over) return fail(MIXAQ_E_SHAPE, "%d rows of %d columns are too many for one call", rows, columns);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // namespace mixaq

extern "C" int mixaq_token_quantize(const mixaq_rows* x, int32_t rows, int32_t columns, const mixaq_rows* q, void* stream)
{
    if (rows < 0 || rows > MOST_ROWS || columns < 1) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 and columns >= 1 (got %d, %d)", rows, columns);
    if (rows == 0) return MIXAQ_OK;
    int rc = check_token_rows(x, "x", columns, VALUES);
    if (!rc) rc = check_token_rows(q, "q", columns, CODES);
    if (rc) return rc;
    const Extent from = extent_of(*x, rows, columns), codes = extent_of(*q, rows, columns), scales = token_scales_of(*q, rows);
    if (overlap(codes, from) || overlap(scales, from)) return fail(MIXAQ_E_SHAPE, "x and q overlap");
    if (overlap(codes, scales)) return fail(MIXAQ_E_SHAPE, "codes and scales of q overlap");
    return launch_token_quantize(*x, rows, columns, *q, (hipStream_t)stream);
}
