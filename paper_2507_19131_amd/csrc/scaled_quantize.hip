// Values to 8-bit float codes with one scale per block of 1 x 128 or 128 x 128 values, and the checks of matrices of rows.
#include "scaled.h"

#include <algorithm>

using namespace mixaq;

namespace mixaq {

int check_rows(const mixaq_rows* m, const char* name, int32_t columns, bool codes_allowed, int32_t scale_rows)
{
    if (!m || !m->data) return fail(MIXAQ_E_NULL, "%s is NULL", name);
    if (m->type < MIXAQ_F32 || m->type > MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "%s: unknown type %d", name, m->type);
    if (m->type == MIXAQ_E4M3 && !codes_allowed) return fail(MIXAQ_E_SHAPE, "%s must be values", name);
    if (m->stride < columns) return fail(MIXAQ_E_SHAPE, "%s: stride %lld of %d columns", name, (long long)m->stride, columns);
    if (m->stride > (1LL << 40)) return fail(MIXAQ_E_SHAPE, "%s: stride %lld is too large", name, (long long)m->stride);
    if ((uintptr_t)m->data % size_of(m->type)) return fail(MIXAQ_E_SHAPE, "%s is not aligned to its values", name);
    if (m->type == MIXAQ_E4M3) {
        if (!m->scales) return fail(MIXAQ_E_NULL, "%s: scales is NULL", name);
        if ((uintptr_t)m->scales % 4) return fail(MIXAQ_E_SHAPE, "%s: scales are not aligned", name);
        if ((uintptr_t)m->data % 16 || m->stride % 16)
            return fail(MIXAQ_E_SHAPE, "%s: codes and their stride must be multiples of 16 bytes (stride %lld)", name, (long long)m->stride);
        if (m->scale_stride < scale_rows || m->scale_stride > (1LL << 40))
            return fail(MIXAQ_E_SHAPE, "%s: scale_stride %lld of %d rows", name, (long long)m->scale_stride, scale_rows);
    }
    return MIXAQ_OK;
}

bool overlap(const Extent& a, const Extent& b)
{
    if (!a.rows || !b.rows) return false;
    const __int128 pa = a.at, pb = b.at;
    if (pa + (__int128)(a.rows - 1) * a.stride + a.width <= pb || pb + (__int128)(b.rows - 1) * b.stride + b.width <= pa) return false;
    if (a.stride == b.stride && a.stride > 0) {          // two column ranges of one matrix
        const __int128 d = ((pb - pa) % a.stride + a.stride) % a.stride;           // b's first column behind a's
        if (d >= a.width && d + b.width <= a.stride) return false;
    }
    return true;
}

}  // namespace mixaq

namespace {

struct QuantArgs {
    const void* x;
    long long ldx;
    uint8_t* codes;
    long long ldc;
    float* scales;
    long long lds;
    int rows, cols, nb, units;        // units: groups of 16 rows x blocks of columns
    FastDiv by_nb;
};

// One block of a row is 16 lanes with eight values each; a wave takes 16 rows of one block of columns, four at a time, and the waves
// beside it the next blocks of the same rows.  What bounds it is memory: 68208 x 384 of bf16 14.7 us, 5.4 TB/s.
template <typename T, bool TINY>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs A)
{
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
    for (int u = blockIdx.x * 4 + (threadIdx.x >> 6); u < A.units; u += gridDim.x * 4) {
        const int rg = A.by_nb(u), b = u - rg * A.nb;
        const Eight c = place8<TINY>(b * SBLOCK + l * 8, A.cols);
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) load8f<TINY>((const T*)A.x + (long long)min(rg * 16 + j * 4 + g, A.rows - 1) * A.ldx, c, A.cols, v[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = rg * 16 + j * 4 + g;
            const BlockScale s = block_scale(max16(max_magnitude<TINY>(c, A.cols, v[j])));
            if (row < A.rows) {
                store_codes8<TINY>(A.codes + (long long)row * A.ldc, c, A.cols, v[j], s.inv);
                if (l == 0) A.scales[b * A.lds + row] = s.scale;
            }
        }
    }
}

// A workgroup per 128 x 128 tile, held in registers between its maximum and its codes: one read of the values.  4000 x 1000 of f32 6.6 us, a tile
// a CU: the launch, a round trip of 64 KB, the maximum's and the stores; more tiles overlap.
template <typename T, bool TINY>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(QuantArgs A)
{
    __shared__ unsigned part[4];
    const int tr = A.by_nb(blockIdx.x), b = blockIdx.x - tr * A.nb;
    const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
    const Eight c = place8<TINY>(b * SBLOCK + l * 8, A.cols);
    float v[8][8];
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) load8f<TINY>((const T*)A.x + (long long)min(tr * SBLOCK + j * 16 + g, A.rows - 1) * A.ldx, c, A.cols, v[j]);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, max_magnitude<TINY>(c, A.cols, v[j]));        // (the last row once more is no other maximum)
    m = over64(m, MaxOf());
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    const BlockScale s = block_scale(max(max(part[0], part[1]), max(part[2], part[3])));
    if (threadIdx.x == 0) A.scales[b * A.lds + tr] = s.scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = tr * SBLOCK + j * 16 + g;
        if (row < A.rows) store_codes8<TINY>(A.codes + (long long)row * A.ldc, c, A.cols, v[j], s.inv);
    }
}

template <typename T, bool TINY>
void launch(const QuantArgs& A, int block_rows, hipStream_t st)
{
    if (block_rows == 1) hipLaunchKernelGGL((quantize_rows_kernel<T, TINY>), dim3(std::min((A.units + 3) / 4, 1 << 22)), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((quantize_tiles_kernel<T, TINY>), dim3(A.units), dim3(256), 0, st, A);
}
template <int TYPE>
void launch_type(const QuantArgs& A, int block_rows, hipStream_t st)
{
    using T = typename TypeOf<TYPE>::T;
    if (A.cols < 8) launch<T, true>(A, block_rows, st);
    else launch<T, false>(A, block_rows, st);
}

}  // namespace

namespace mixaq {

int launch_quantize(const mixaq_rows& x, int32_t rows, int32_t columns, int32_t block_rows, const mixaq_rows& q, hipStream_t st)
{
    QuantArgs A;
    A.x = x.data; A.ldx = x.stride;
    A.codes = (uint8_t*)q.data; A.ldc = q.stride;
    A.scales = q.scales; A.lds = q.scale_stride;
    A.rows = rows; A.cols = columns; A.nb = blocks_of(columns);
    const int per = block_rows == 1 ? 16 : SBLOCK;
    const long long units = ((long long)rows + per - 1) / per * A.nb;
    if (units >= (1LL << 30) || (block_rows > 1 && units * 256 >= MOST_THREADS))
        return fail(MIXAQ_E_SHAPE, "%d rows of %d columns are too many for one call", rows, columns);
    A.units = (int)units;
    A.by_nb = FastDiv(A.nb);
    switch (x.type) {
    case MIXAQ_F32: launch_type<MIXAQ_F32>(A, block_rows, st); break;
    case MIXAQ_F16: launch_type<MIXAQ_F16>(A, block_rows, st); break;
    default: launch_type<MIXAQ_BF16>(A, block_rows, st); break;
    }
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // namespace mixaq

extern "C" int mixaq_scaled_quantize(const mixaq_rows* x, int32_t rows, int32_t columns, int32_t block_rows, const mixaq_rows* q,
                                     void* stream)
{
    if (rows < 0 || rows > MOST_ROWS || columns < 1) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 and columns >= 1 (got %d, %d)", rows, columns);
    if (block_rows != 1 && block_rows != SBLOCK) return fail(MIXAQ_E_SHAPE, "block_rows must be 1 or 128 (got %d)", block_rows);
    if (rows == 0) return MIXAQ_OK;
    const int32_t scale_rows = block_rows == 1 ? rows : blocks_of(rows);
    int rc = check_rows(x, "x", columns, false, 0);
    if (!rc) rc = check_rows(q, "q", columns, true, scale_rows);
    if (rc) return rc;
    if (q->type != MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "q must be codes");
    const Extent from = extent_of(*x, rows, columns), codes = extent_of(*q, rows, columns), scales = scales_of(*q, scale_rows, columns);
    if (overlap(codes, from) || overlap(scales, from)) return fail(MIXAQ_E_SHAPE, "x and q overlap");
    if (overlap(codes, scales)) return fail(MIXAQ_E_SHAPE, "codes and scales of q overlap");
    return launch_quantize(*x, rows, columns, block_rows, *q, (hipStream_t)stream);
}
