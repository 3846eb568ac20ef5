// y = act(group norm of x) on channels-last maps: the mean and the variance of every group of neighbouring channels over all rows of an image.
#include "token.h"

#include <algorithm>
#include <cmath>

using namespace mixaq;

namespace {

constexpr int MOST_GROUPS = 1024, MOST_CHANNELS = 8192, THREADS = 1024;

// Sums over values less a pivot, the first value of their image and group: squares of differences from one of the values are at most as many times the
// variance as there are values, so that binary64 keeps the variance whatever the mean is.
struct Sums { double v, q; };

struct GroupArgs {
    const void* x;
    void* y;
    float* scales;
    long long ldx, ldy;
    int C, groups, per_group;         // channels of a group
    int rows, chunks, chunk_rows;     // of an image
    int units, lanes, act, y_type;    // units: of eight channels; lanes: of a row, of the kernel that writes
    float eps;
    const float *gamma, *beta;
    Sums* part;                       // [images][chunks][groups]
    float* pivots;                    // [images][groups]: x may be written over
};

__device__ __forceinline__ double shfl_xor64(double v, int d)
{
    const long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__shfl_xor((int)b, d, 64), hi = (unsigned)__shfl_xor((int)(b >> 32), d, 64);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}

// The sums of one chunk of rows.  A thread keeps to eight channels, so that the threads of a workgroup read whole rows one behind the other.  WHOLE: a
// group is a multiple of eight channels, whose sums a thread takes together.
template <typename T, bool TINY, bool WHOLE>
__global__ __launch_bounds__(THREADS) void group_sums_kernel(GroupArgs A)
{
    constexpr int E = WHOLE ? 1 : 8;
    __shared__ double red[E][THREADS];
    const int image = blockIdx.x / A.chunks, chunk = blockIdx.x - image * A.chunks;
    const int slots = THREADS / A.units, slot = threadIdx.x / A.units, u = threadIdx.x - slot * A.units;
    const Eight c = place8<TINY>(u * 8, A.C);
    const T* const map = (const T*)A.x + (long long)image * A.rows * A.ldx;
    double pivot[E], v[E] = {}, q[E] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) pivot[e] = (double)(float)map[min(c.at + e, A.C - 1) / A.per_group * A.per_group];
    if (slot < slots) {
        const int end = min((chunk + 1) * A.chunk_rows, A.rows);
        for (int r = chunk * A.chunk_rows + slot; r < end; r += slots) {
            float x[8];
            load8f<TINY>(map + (long long)r * A.ldx, c, A.C, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = (double)x[e] - pivot[WHOLE ? 0 : e];
                v[WHOLE ? 0 : e] += d;
                q[WHOLE ? 0 : e] = fma(d, d, q[WHOLE ? 0 : e]);
            }
        }
    }
    // a group's lanes: a power of two, with about eight values each
    const int per = WHOLE ? A.per_group / 8 : A.per_group, count = slots * per;
    int lanes = 1;
    while (lanes < 64 && lanes * 8 < count) lanes *= 2;
    double total[2];
    for (int round = 0; round * (THREADS / lanes) < A.groups; ++round) {
        const int g = round * (THREADS / lanes) + threadIdx.x / lanes, l = threadIdx.x % lanes;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();                                                 // (one kind of sums at a time lies in LDS)
#pragma unroll
            for (int e = 0; e < E; ++e) red[e][threadIdx.x] = which ? q[e] : v[e];
            __syncthreads();
            double s = 0.0;
            if (g < A.groups)
                for (int i = l; i < count; i += lanes) {
                    const int at = i / per, channel = g * per + i - at * per;            // (WHOLE: unit)
                    if constexpr (WHOLE) s += red[0][at * A.units + channel];
                    else {
                        const int unit = channel / 8, from = place8<TINY>(unit * 8, A.C).at;
                        s += red[channel - from][at * A.units + unit];
                    }
                }
            for (int d = 1; d < lanes; d <<= 1) s += shfl_xor64(s, d);
            total[which] = s;
        }
        if (g < A.groups && l == 0) {
            A.part[((long long)image * A.chunks + chunk) * A.groups + g] = {total[0], total[1]};
            if (chunk == 0) A.pivots[(long long)image * A.groups + g] = (float)map[g * A.per_group];
        }
    }
}

// Chunk by chunk again: every workgroup adds up its image's sums first, in the order of the chunks.  `lanes` lanes a row: for values as many as it has units of
// eight channels, for codes a power of two, whose maximum goes through the lanes and, of more than a wave, through LDS.
template <typename T, bool TINY>
__global__ __launch_bounds__(THREADS) void group_norm_kernel(GroupArgs A)
{
    __shared__ float mean_hi[MOST_GROUPS], mean_lo[MOST_GROUPS], factor[MOST_GROUPS];
    __shared__ unsigned part[2][THREADS / 64];
    const int image = blockIdx.x / A.chunks, chunk = blockIdx.x - image * A.chunks;
    const T* const map = (const T*)A.x + (long long)image * A.rows * A.ldx;
    {
        int lanes = 1;                                                       // of a group
        while (lanes < 64 && lanes * 2 <= A.chunks && lanes * 2 * A.groups <= THREADS) lanes *= 2;
        for (int g0 = 0; g0 < A.groups; g0 += THREADS / lanes) {
            const int g = g0 + threadIdx.x / lanes, l = threadIdx.x % lanes;
            double v = 0.0, q = 0.0;
            if (g < A.groups)
                for (int i = l; i < A.chunks; i += lanes) {
                    const Sums s = A.part[((long long)image * A.chunks + i) * A.groups + g];
                    v += s.v;
                    q += s.q;
                }
            for (int d = 1; d < lanes; d <<= 1) {
                v += shfl_xor64(v, d);
                q += shfl_xor64(q, d);
            }
            if (g < A.groups && l == 0) {
                const double n = 1.0 / ((double)A.rows * A.per_group), off = v * n, mean = (double)A.pivots[(long long)image * A.groups + g] + off;
                const double variance = q * n - off * off;
                mean_hi[g] = (float)mean;
                mean_lo[g] = (float)(mean - (double)mean_hi[g]);
                factor[g] = (float)(1.0 / sqrt((variance < 0.0 ? 0.0 : variance) + (double)A.eps));        // (a NaN stays one)
            }
        }
    }
    __syncthreads();
    const int slots = THREADS / A.lanes, slot = threadIdx.x / A.lanes, u = threadIdx.x - slot * A.lanes;
    const Eight c = place8<TINY>(u * 8, A.C);
    float hi[8], a[8], b[8];                                                 // y = (x - hi) a + b
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int channel = min(c.at + e, A.C - 1), g = channel / A.per_group;
        hi[e] = mean_hi[g];
        a[e] = factor[g] * (A.gamma ? A.gamma[channel] : 1.0f);
        b[e] = fmaf(-mean_lo[g], a[e], A.beta ? A.beta[channel] : 0.0f);
    }
    const int end = min((chunk + 1) * A.chunk_rows, A.rows);
    int turn = 0;
    for (int r0 = chunk * A.chunk_rows; r0 < end; r0 += slots) {
        const bool real = slot < slots && r0 + slot < end;
        const int r = min(r0 + slot, end - 1);
        float v[8];
        load8f<TINY>(map + (long long)r * A.ldx, c, A.C, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e] - hi[e], a[e], b[e]);
        activate(v, A.act);
        const long long row = (long long)image * A.rows + r;
        if (A.y_type == MIXAQ_I8) {
            unsigned m = max_magnitude<TINY>(c, A.C, v);
            for (int d = 1; d < A.lanes && d < 64; d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d, 64));
            if (A.lanes > 64) {                                              // (two places in turn: who writes one again has passed the other's barrier)
                if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = m;
                __syncthreads();
                const int first = slot * (A.lanes / 64);
                for (int w = 0; w < A.lanes / 64; ++w) m = max(m, part[turn][first + w]);
                turn ^= 1;
            }
            const RowScale s = row_scale(m);
            if (real) {
                store_int_codes8<TINY>((int8_t*)A.y + row * A.ldy, c, A.C, v, s.inv);
                if (u == 0) A.scales[row] = s.scale;
            }
        } else if (real) {
            if (A.y_type == MIXAQ_F32) store8<TINY>((float*)A.y + row * A.ldy, c, A.C, v);
            else if (A.y_type == MIXAQ_F16) store8<TINY>((_Float16*)A.y + row * A.ldy, c, A.C, v);
            else store8<TINY>((__bf16*)A.y + row * A.ldy, c, A.C, v);
        }
    }
}

// Chunks of an image: about two workgroups a CU in all, each with rows for several turns.
struct Chunks { int count, rows; };
Chunks chunks_of(int rows, int images, int units)
{
    const int turn = THREADS / units;
    const long long most = ((long long)rows + 4LL * turn - 1) / (4LL * turn), wanted = std::max(1, (512 + images - 1) / images);
    const int count = (int)std::min(most, wanted), per = (rows + count - 1) / count;
    return {(rows + per - 1) / per, per};
}

int check_desc(const mixaq_group_norm_desc* d)
{
    if (!d) return fail(MIXAQ_E_NULL, "descriptor is NULL");
    if (d->C < 1 || d->C > MOST_CHANNELS) return fail(MIXAQ_E_SHAPE, "C=%d outside 1..%d", d->C, MOST_CHANNELS);
    if (d->groups < 1 || d->groups > MOST_GROUPS || d->C % d->groups) return fail(MIXAQ_E_SHAPE, "groups=%d: need 1..%d, a divisor of C=%d", d->groups, MOST_GROUPS, d->C);
    if (d->rows_per_image < 1 || d->rows_per_image > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "rows_per_image=%d outside 1..2^30", d->rows_per_image);
    if (d->activation < ACT_NONE || d->activation > ACT_RELU) return fail(MIXAQ_E_SHAPE, "unknown activation %d", d->activation);
    if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return fail(MIXAQ_E_SHAPE, "eps must be positive");
    return MIXAQ_OK;
}
int check_count(const mixaq_group_norm_desc* d, int32_t rows)
{
    if (rows < 0 || rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 (got %d)", rows);
    if (rows % d->rows_per_image) return fail(MIXAQ_E_SHAPE, "%d rows are no whole images of %d", rows, d->rows_per_image);
    return MIXAQ_OK;
}
int units_of(int C) { return (C + 7) / 8; }
size_t sums_bytes(const mixaq_group_norm_desc& d, int images)
{
    return (size_t)images * chunks_of(d.rows_per_image, images, units_of(d.C)).count * d.groups * sizeof(Sums);
}
size_t workspace_of(const mixaq_group_norm_desc& d, int images) { return images ? sums_bytes(d, images) + (size_t)images * d.groups * sizeof(float) : 0; }

template <typename T, bool TINY>
void launch(const GroupArgs& A, unsigned blocks, hipStream_t st)
{
    if (A.per_group % 8 == 0) hipLaunchKernelGGL((group_sums_kernel<T, TINY, true>), dim3(blocks), dim3(THREADS), 0, st, A);
    else hipLaunchKernelGGL((group_sums_kernel<T, TINY, false>), dim3(blocks), dim3(THREADS), 0, st, A);
    hipLaunchKernelGGL((group_norm_kernel<T, TINY>), dim3(blocks), dim3(THREADS), 0, st, A);
}
template <int TYPE>
void launch_type(const GroupArgs& A, unsigned blocks, hipStream_t st)
{
    using T = typename TypeOf<TYPE>::T;
    if (A.C < 8) launch<T, true>(A, blocks, st);
    else launch<T, false>(A, blocks, st);
}

}  // namespace

extern "C" {

int mixaq_group_norm_workspace_bytes(const mixaq_group_norm_desc* desc, int32_t rows, size_t* bytes)
{
    if (!bytes) return fail(MIXAQ_E_NULL, "bytes is NULL");
    int rc = check_desc(desc);
    if (!rc) rc = check_count(desc, rows);
    if (rc) return rc;
    *bytes = workspace_of(*desc, rows / desc->rows_per_image);
    return MIXAQ_OK;
}

int mixaq_group_norm(const mixaq_group_norm_desc* desc, const mixaq_group_norm_params* params, const mixaq_rows* x, const mixaq_rows* y, int32_t rows,
                     void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_desc(desc);
    if (rc) return rc;
    if (!params) return fail(MIXAQ_E_NULL, "params is NULL");
    const mixaq_group_norm_desc& d = *desc;
    rc = check_count(desc, rows);
    if (rc || rows == 0) return rc;
    rc = check_token_rows(x, "x", d.C, VALUES);
    if (!rc) rc = check_token_rows(y, "y", d.C, VALUES | CODES);
    if (rc) return rc;
    const int images = rows / d.rows_per_image;
    const size_t need = workspace_of(d, images);
    if (!workspace) return fail(MIXAQ_E_NULL, "workspace is NULL (%zu bytes needed)", need);
    if (workspace_bytes < need) return fail(MIXAQ_E_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    if ((uintptr_t)workspace & 255) return fail(MIXAQ_E_WORKSPACE, "workspace must be 256-byte aligned");
    const Extent from = extent_of(*x, rows, d.C), to = extent_of(*y, rows, d.C), scales = token_scales_of(*y, rows), ws = memory_of(workspace, (long long)need);
    const bool in_place = x->data == y->data && x->stride == y->stride && x->type == y->type;
    if ((!in_place && overlap(to, from)) || overlap(scales, from)) return fail(MIXAQ_E_SHAPE, "x and y overlap");
    if (overlap(to, scales)) return fail(MIXAQ_E_SHAPE, "codes and scales of y overlap");
    if (overlap(ws, from) || overlap(ws, to) || overlap(ws, scales)) return fail(MIXAQ_E_SHAPE, "the workspace overlaps x or y");
    const float* const vectors[2] = {params->gamma, params->beta};
    const char* const names[2] = {"gamma", "beta"};
    for (int i = 0; i < 2; ++i) {
        if ((uintptr_t)vectors[i] % 4) return fail(MIXAQ_E_SHAPE, "%s is not aligned", names[i]);
        const Extent v = memory_of(vectors[i], d.C * 4LL);
        if (overlap(to, v) || overlap(scales, v) || overlap(ws, v)) return fail(MIXAQ_E_SHAPE, "%s overlaps y or the workspace", names[i]);
    }
    GroupArgs A = {};
    A.x = x->data; A.ldx = x->stride;
    A.y = y->data; A.ldy = y->stride; A.scales = y->scales; A.y_type = y->type;
    A.C = d.C; A.groups = d.groups; A.per_group = d.C / d.groups;
    A.units = A.lanes = units_of(d.C);
    if (y->type == MIXAQ_I8)
        for (A.lanes = 1; A.lanes < A.units;) A.lanes *= 2;
    const Chunks ch = chunks_of(d.rows_per_image, images, A.units);
    A.rows = d.rows_per_image; A.chunks = ch.count; A.chunk_rows = ch.rows;
    A.act = d.activation; A.eps = d.eps;
    A.gamma = params->gamma; A.beta = params->beta;
    A.part = (Sums*)workspace;
    A.pivots = (float*)((char*)workspace + sums_bytes(d, images));
    const long long blocks = (long long)images * ch.count;
    if (blocks * THREADS >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d images are too many for one call", images);
    if (x->type == MIXAQ_F32) launch_type<MIXAQ_F32>(A, (unsigned)blocks, (hipStream_t)stream);
    else if (x->type == MIXAQ_F16) launch_type<MIXAQ_F16>(A, (unsigned)blocks, (hipStream_t)stream);
    else launch_type<MIXAQ_BF16>(A, (unsigned)blocks, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // extern "C"
