// y = act(group norm of x) on channels-last maps: the mean and the variance of every group of neighbouring channels over all rows of an image.
#include "token.h"

#include <algorithm>
#include <cmath>

using namespace mixaq;

namespace {

constexpr int MOST_GROUPS = 1024, MOST_CHANNELS = 8192;

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
    bool aligned;                     // rows of y that are values start at multiples of 16 bytes
    float eps;
    double inv_count;                 // of a group's values
    FastDiv by_group;                 // per_group
    const float *gamma, *beta;
    Sums* part;                       // [images][chunks][groups]
    float* pivots;                    // [images][groups]: x may be written over
};

__device__ __forceinline__ double shfl64(double v, int from)
{
    const long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__shfl((int)b, from, 64), hi = (unsigned)__shfl((int)(b >> 32), from, 64);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}

// Which rows and channels a thread takes: slot < slots of those that take any.
struct Place { int u, slot, slots; };
template <int THREADS>
__device__ __forceinline__ Place place_of(int units)
{
    Place p;
    p.slots = THREADS / units;
    p.slot = threadIdx.x / units;
    p.u = threadIdx.x - p.slot * units;
    return p;
}

// Adds up what the threads of a workgroup have for each group, of a unit's eight channels together (WHOLE) or each for itself: of many rows of sums those that are `left`
// apart, then 16 lanes a group the rows that are left.  (Exchanges between lanes in place of the first step pass LDS as well, and more often: 49 x 96 with three
// channels a group 12.1 us instead of 7.2.)  One thread a group calls to(g, sums).  The order goes by the sizes alone.
template <int THREADS, bool TINY, bool WHOLE, int E, typename To>
__device__ __forceinline__ void add_up(const double (&v)[E], const double (&q)[E], const Place& p, int units, int per_group, int groups, int C, Sums (*red)[THREADS * 9 / 8], To to)
{
    constexpr int LANES = 16;
    const int left = p.slots <= 2 * LANES ? p.slots : LANES * (p.slots >= 512 ? 8 : p.slots >= 128 ? 4 : 1);
    const int stride = units < 8 ? units : units | 1;                        // odd, so that the rows of a unit lie in different banks
    if (p.slot < p.slots) {
#pragma unroll
        for (int e = 0; e < E; ++e) red[e][p.slot * stride + p.u] = {v[e], q[e]};
    }
    __syncthreads();
    if (left < p.slots) {
        const int row = left * stride;
        for (int i = threadIdx.x; i < E * row; i += THREADS) {               // (the only thread that reads or writes these rows of this channel)
            const int e = E == 1 ? 0 : i / row;
            Sums s = {0.0, 0.0};
            for (int at = i - e * row; at < p.slots * stride; at += row) {
                s.v += red[e][at].v;
                s.q += red[e][at].q;
            }
            red[e][i - e * row] = s;
        }
        __syncthreads();
    }
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < groups; g0 += THREADS / LANES) {
        const int g = g0 + threadIdx.x / LANES, l = threadIdx.x % LANES;
        Sums s = {0.0, 0.0};
        if (g < groups) {
            auto more = [&](const Sums& o) {
                s.v += o.v;
                s.q += o.q;
            };
            for (int r = l; r < left; r += LANES) {
                if constexpr (WHOLE) {
                    for (int i = g * (per_group / 8); i < (g + 1) * (per_group / 8); ++i) more(red[0][r * stride + i]);
                } else {
                    for (int i = g * per_group; i < (g + 1) * per_group; ++i) {
                        const int unit = i / 8, at = place8<TINY>(unit * 8, C).at;
                        more(red[i - at][r * stride + unit]);
                    }
                }
            }
        }
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) {
            s.v += shfl64(s.v, lane ^ d);
            s.q += shfl64(s.q, lane ^ d);
        }
        if (g < groups && l == 0) to(g, s);
    }
}
template <bool WHOLE, int E>
__device__ __forceinline__ void add(double (&v)[E], double (&q)[E], const float (&x)[8], const double (&pivot)[E])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double d = (double)x[e] - pivot[WHOLE ? 0 : e];
        v[WHOLE ? 0 : e] += d;
        q[WHOLE ? 0 : e] = fma(d, d, q[WHOLE ? 0 : e]);
    }
}

// What becomes of a group's values: (x - hi) a + b, a = r gamma, b = beta - lo a; hi + lo is the mean.
struct Factors { float hi, lo, r; };
__device__ __forceinline__ Factors factors_of(Sums s, double n, float pivot, float eps)
{
    const double off = s.v * n, mean = (double)pivot + off, variance = s.q * n - off * off;
    Factors f;
    f.hi = (float)mean;
    f.lo = (float)(mean - (double)f.hi);
    f.r = (float)(1.0 / sqrt((variance < 0.0 ? 0.0 : variance) + (double)eps));          // (a NaN stays one)
    return f;
}
template <bool TINY>
__device__ __forceinline__ void load_vectors(const GroupArgs& A, Eight c, float (&gamma)[8], float (&beta)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        gamma[e] = 1.0f;
        beta[e] = 0.0f;
    }
    if (A.gamma) load8f<TINY>(A.gamma, c, A.C, gamma);
    if (A.beta) load8f<TINY>(A.beta, c, A.C, beta);
}
// a: gamma, b: beta
__device__ __forceinline__ void coefficients(const GroupArgs& A, Eight c, const Factors* of, int first, float (&hi)[8], float (&a)[8], float (&b)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const Factors f = of[A.by_group(min(c.at + e, A.C - 1)) - first];
        hi[e] = f.hi;
        a[e] *= f.r;
        b[e] = fmaf(-f.lo, a[e], b[e]);
    }
}
template <typename T>
__device__ __forceinline__ void apply(const T (&x)[8], const float (&hi)[8], const float (&a)[8], const float (&b)[8], int act, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf((float)x[e] - hi[e], a[e], b[e]);
    activate(v, act);
}
// PAST: past the caches, where rows start at multiples of 16 bytes.
template <bool TINY, bool PAST, typename Y>
__device__ __forceinline__ void store_row(Y* row, Eight c, int C, bool aligned, const float (&v)[8])
{
    if (PAST && !TINY && aligned && c.first == 0) {
        Y t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (Y)v[e];
        v4i p[sizeof(Y) / 2];
        __builtin_memcpy(p, t, sizeof(t));
#pragma unroll
        for (int i = 0; i < (int)sizeof(Y) / 2; ++i) __builtin_nontemporal_store(p[i], (v4i*)(row + c.at) + i);
    } else store8<TINY>(row, c, C, v);
}
template <bool TINY, bool PAST>
__device__ __forceinline__ void store_values(const GroupArgs& A, long long row, Eight c, const float (&v)[8])
{
    if (A.y_type == MIXAQ_F32) store_row<TINY, PAST>((float*)A.y + row * A.ldy, c, A.C, A.aligned, v);
    else if (A.y_type == MIXAQ_F16) store_row<TINY, PAST>((_Float16*)A.y + row * A.ldy, c, A.C, A.aligned, v);
    else store_row<TINY, PAST>((__bf16*)A.y + row * A.ldy, c, A.C, A.aligned, v);
}

// Small maps in one kernel: a workgroup holds its channels of an image, whole groups and whole units, in registers.  What bounds it: a launch, a round trip and the
// reductions (1050 x 256 of f16 6.7 us of a graph replay; 4200 x 768, in the two kernels of larger maps, 12).
constexpr int HELD = 4;                           // rows of a thread
template <typename T, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void group_small_kernel(GroupArgs A, int parts)
{
    constexpr int E = WHOLE ? 1 : 8;
    __shared__ Sums red[E][THREADS * 9 / 8];
    __shared__ Factors factor[8];                                            // (of lcm(8, per_group) channels)
    const int image = blockIdx.x / parts, part = blockIdx.x - image * parts, width = A.C / parts, units = width / 8;
    const Place p = place_of<THREADS>(units);
    const int slots = p.slots, slot = p.slot, first = part * width / A.per_group;
    const Eight c = {part * width + p.u * 8, 0};
    const T* const map = (const T*)A.x + (long long)image * A.rows * A.ldx;
    T x[HELD][8];
#pragma unroll
    for (int k = 0; k < HELD; ++k) load8<false>(map + (long long)min(slot + k * slots, A.rows - 1) * A.ldx, c, A.C, x[k]);
    float hi[8], a[8], b[8];
    load_vectors<false>(A, c, a, b);
    double pivot[E], v[E] = {}, q[E] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) pivot[e] = (double)(float)map[A.by_group(c.at + e) * A.per_group];
    const float mine = (float)map[(first + min((int)threadIdx.x, width / A.per_group - 1)) * A.per_group];         // the pivot of group threadIdx.x
    __shared__ float pivots[8];
    if (threadIdx.x < 8) pivots[threadIdx.x] = mine;
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (slot < slots && slot + k * slots < A.rows) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = (float)x[k][e];
            add<WHOLE>(v, q, f, pivot);
        }
    add_up<THREADS, false, WHOLE>(v, q, p, units, A.per_group, width / A.per_group, width, red, [&](int g, Sums s) {
        factor[g] = factors_of(s, A.inv_count, pivots[g], A.eps);
    });
    __syncthreads();                                                         // (every value has been read: y may be x)
    coefficients(A, c, factor, first, hi, a, b);
    if (slot >= slots) return;
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        if (slot + k * slots >= A.rows) break;
        float f[8];
        apply(x[k], hi, a, b, A.act, f);
        store_values<false, false>(A, (long long)image * A.rows + slot + k * slots, c, f);
    }
}

constexpr int AHEAD = 8;                          // rows of a thread that are on their way at one time (of 32 bits half as many)

// The sums of one chunk of rows.  A thread keeps to eight channels, so that the threads of a workgroup read whole rows one behind the other.  WHOLE: a
// group is a multiple of eight channels, whose sums a thread takes together.  4 x 65536 x 128 of bf16 15.9 us, 4.2 TB/s, 67200 x 96 of f32 8.6, 3.0 TB/s: less than
// memory gives (the quantizer moves 5.9), and sums in binary32 instead of binary64 save nothing.  A workgroup a CU, so two waves a SIMD, each with one turn of loads on its
// way; more of them were not tried.
template <typename T, bool TINY, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void group_sums_kernel(GroupArgs A)
{
    constexpr int E = WHOLE ? 1 : 8, TURN = AHEAD / (sizeof(T) == 4 ? 2 : 1) / (THREADS == 1024 ? 2 : 1);
    __shared__ Sums red[E][THREADS * 9 / 8];
    const int image = blockIdx.x / A.chunks, chunk = blockIdx.x - image * A.chunks;
    const Place p = place_of<THREADS>(A.units);
    const int slots = p.slots, slot = p.slot;
    const Eight c = place8<TINY>(p.u * 8, A.C);
    const T* const map = (const T*)A.x + (long long)image * A.rows * A.ldx;
    double pivot[E], v[E] = {}, q[E] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) pivot[e] = (double)(float)map[A.by_group(min(c.at + e, A.C - 1)) * A.per_group];
    if (slot < slots) {
        const int end = min((chunk + 1) * A.chunk_rows, A.rows);
        int r = chunk * A.chunk_rows + slot;
        for (; r + (TURN - 1) * slots < end; r += TURN * slots) {
            T x[TURN][8];
#pragma unroll
            for (int k = 0; k < TURN; ++k) load8<TINY>(map + (long long)(r + k * slots) * A.ldx, c, A.C, x[k]);
#pragma unroll
            for (int k = 0; k < TURN; ++k) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (float)x[k][e];
                add<WHOLE>(v, q, f, pivot);
            }
        }
        for (; r < end; r += slots) {
            float f[8];
            load8f<TINY>(map + (long long)r * A.ldx, c, A.C, f);
            add<WHOLE>(v, q, f, pivot);
        }
    }
    add_up<THREADS, TINY, WHOLE>(v, q, p, A.units, A.per_group, A.groups, A.C, red, [&](int g, Sums s) {
        A.part[((long long)image * A.chunks + chunk) * A.groups + g] = s;
        if (chunk == 0) A.pivots[(long long)image * A.groups + g] = (float)map[g * A.per_group];
    });
}

// Chunk by chunk again, from its last rows, which the caches are likely to hold, to the first: every workgroup adds up its image's sums first, in an order that goes
// by the sizes alone, while its first rows are on their way.  `lanes` lanes a row: for values as many as it has units of eight channels, for codes a power of
// two, whose maximum goes through the lanes and, of more than a wave, through LDS.  Values go past the caches, which the map is in.  What bounds it is memory, with a SiLU in
// part the vector unit: 4 x 65536 x 128 of bf16 27.5 us, 4.9 TB/s of read and write (through the caches 33.9, without the SiLU 28.9 there), 67200 x 96 of
// f32 12.2; before that 2 to 3 us for the image's sums, which other XCDs wrote, eight loads at a time (one after the other 7 more).  In place of two kernels one with
// the map held on the chip would need the workgroups to wait for one another.
template <typename T, bool TINY, int THREADS>
__global__ __launch_bounds__(THREADS) void group_norm_kernel(GroupArgs A)
{
    constexpr int TURN = AHEAD / (sizeof(T) == 4 ? 2 : 1) / (THREADS == 1024 ? 2 : 1);
    __shared__ Sums merge[THREADS];
    __shared__ Factors factor[MOST_GROUPS];
    __shared__ unsigned part[2][THREADS / 64];
    const int image = blockIdx.x / A.chunks, chunk = blockIdx.x - image * A.chunks;
    const T* const map = (const T*)A.x + (long long)image * A.rows * A.ldx;
    const int slots = THREADS / A.lanes, slot = threadIdx.x / A.lanes, u = threadIdx.x - slot * A.lanes;
    const Eight c = place8<TINY>(u * 8, A.C);
    const int first = chunk * A.chunk_rows, end = min(first + A.chunk_rows, A.rows), step = TURN * slots;
    T x[TURN][8];
    auto row_of = [&](int r0, int k) { return r0 + k * slots + slot; };
    auto request = [&](int r0) {                                             // (spare lanes take the last row along)
#pragma unroll
        for (int k = 0; k < TURN; ++k) load8<TINY>(map + (long long)min(row_of(r0, k), end - 1) * A.ldx, c, A.C, x[k]);
    };
    int r0 = first + (end - 1 - first) / step * step;
    request(r0);
    float hi[8], a[8], b[8];
    load_vectors<TINY>(A, c, a, b);
    {
        const int at_once = min(A.groups, THREADS), teams = THREADS / at_once, l = threadIdx.x / at_once;
        int fold = 1;                                                        // the largest power of two up to teams and chunks
        while (fold * 2 <= teams && fold * 2 <= A.chunks) fold *= 2;
        for (int g = threadIdx.x - l * at_once; g < A.groups; g += at_once) {            // (once, unless a thread has a group or two)
            Sums s = {0.0, 0.0};
            if (l < fold) {
                const Sums* const from = A.part + (long long)image * A.chunks * A.groups + g;
                for (int i = l; i < A.chunks; i += 8 * fold) {               // (each from beyond the L2: eight on their way at one time)
                    Sums o[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] = from[(long long)min(i + k * fold, A.chunks - 1) * A.groups];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const bool one = i + k * fold < A.chunks;
                        s.v += one ? o[k].v : 0.0;
                        s.q += one ? o[k].q : 0.0;
                    }
                }
                merge[threadIdx.x] = s;
            }
            for (int d = fold / 2; d; d /= 2) {
                __syncthreads();
                if (l < d) {
                    merge[threadIdx.x].v += merge[threadIdx.x + d * at_once].v;
                    merge[threadIdx.x].q += merge[threadIdx.x + d * at_once].q;
                }
            }
            if (l == 0) factor[g] = factors_of(merge[threadIdx.x], A.inv_count, A.pivots[(long long)image * A.groups + g], A.eps);
        }
    }
    __syncthreads();
    coefficients(A, c, factor, 0, hi, a, b);
    int turn = 0;
    for (;;) {
        float v[TURN][8];
#pragma unroll
        for (int k = 0; k < TURN; ++k) apply(x[k], hi, a, b, A.act, v[k]);
        const int now = r0;
        r0 -= step;
        if (r0 >= first) request(r0);
#pragma unroll
        for (int k = 0; k < TURN; ++k) {
            const bool real = slot < slots && row_of(now, k) < end;
            const long long row = (long long)image * A.rows + row_of(now, k);
            if (A.y_type == MIXAQ_I8) {
                unsigned m = max_magnitude<TINY>(c, A.C, v[k]);
                for (int d = 1; d < A.lanes && d < 64; d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d, 64));
                if (A.lanes > 64) {                                          // (two places in turn: who writes one again has passed the other's barrier)
                    if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = m;
                    __syncthreads();
                    const int wave = slot * (A.lanes / 64);
                    for (int w = 0; w < A.lanes / 64; ++w) m = max(m, part[turn][wave + w]);
                    turn ^= 1;
                }
                const RowScale s = row_scale(m);
                if (real) {
                    store_int_codes8<TINY>((int8_t*)A.y + row * A.ldy, c, A.C, v[k], s.inv);
                    if (u == 0) A.scales[row] = s.scale;
                }
            } else if (real) store_values<TINY, true>(A, row, c, v[k]);
        }
        if (r0 < first) break;
    }
}

// Chunks of an image: a workgroup a CU in all (what every one adds up first grows with their number), each with rows for a turn of AHEAD or more.
constexpr int THREADS = 512, MOST_THREADS_EACH = 1024;                       // of a workgroup, of one for more than 4096 channels
int threads_of(int units) { return units > THREADS ? MOST_THREADS_EACH : THREADS; }
struct Chunks { int count, rows; };
long long most_chunks(int rows, int units)                                   // of an image
{
    const int turn = threads_of(units) / units;
    return ((long long)rows + AHEAD * turn - 1) / (AHEAD * turn);
}
Chunks chunks_of(int rows, int images, int units)
{
    const long long wanted = std::max(1, (256 + images - 1) / images);
    const int count = (int)std::min(most_chunks(rows, units), wanted), per = (rows + count - 1) / count;
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
// What a call uses.
size_t needed(const mixaq_group_norm_desc& d, int images) { return sums_bytes(d, images) + (size_t)images * d.groups * sizeof(float); }
// Enough for up to `images`: the chunks of all of them rise and fall with their number (256 of 4 images, 258 of 3), but are never more than images + 255.
size_t workspace_of(const mixaq_group_norm_desc& d, int images)
{
    const size_t chunks = (size_t)std::min(images * most_chunks(d.rows_per_image, units_of(d.C)), images + 255LL);
    return images ? chunks * d.groups * sizeof(Sums) + (size_t)images * d.groups * sizeof(float) : 0;
}

// Of how many parts an image's channels are, whole groups and whole units of eight each, where a workgroup holds the rows of one; 0 where none does, or where the
// workgroups of all images are more than a launch takes.  us of graph replays, bf16, images x rows x channels (groups):
//   In one kernel / in two, up to the line of HELD: 1 x 49 x 256 (32) 5.5 / 8.1    1 x 4096 x 32 (4) 8.0 / 10.7    1 x 1364 x 48 (16) 9.1 / 11.0    1 x 1050 x 256 (32) 6.6 / 11.1
//     1 x 1024 x 1024 (32) 8.0 / 11.4    1 x 256 x 1024 (8) 7.4 / 11.0    1 x 128 x 2048 (8) 9.2 / 11.7; not so 1 x 4096 x 256 (32) 15.7 / 11.3, of f32 22.4 / 11.7 (32 workgroups
//     of 16 bytes a row)
//   Behind it (HELD 8 / two): 1 x 8192 x 32 (4) 11.5 / 10.8    1 x 4200 x 256 (32) 16.3 / 11.2    1 x 2048 x 1024 (32) 11.3 / 11.6    1 x 512 x 1024 (8) 9.9 / 11.2    1 x 256 x 2048 (8)
//     11.5 / 11.8    8 x 8192 x 256 (32) 60 / 19.5
//   The number of images is not looked at, nor how many threads of a workgroup have rows; many images take longer in one kernel, 256 (32): 4 x 1024 9.9 / 10.9    8 x 1024
//     12.4 / 11.1    16 x 196 9.5 / 9.9    64 x 196 26 / 11.3    64 x 49 21 / 8.7    1000 x 49 270 / 26
int parts_of(const mixaq_group_norm_desc& d, int images)
{
    int width = d.C / d.groups;
    while (width % 8) width += d.C / d.groups;                               // (after at most eight)
    if (d.C % 8 || d.C % width || width / 8 > 1024 || (d.rows_per_image - 1LL) / (1024 / (width / 8)) >= HELD) return 0;
    return (long long)images * (d.C / width) * 1024 < MOST_THREADS ? d.C / width : 0;
}

template <typename T>
void launch_small(const GroupArgs& A, int parts, unsigned blocks, hipStream_t st)
{
    if (A.per_group % 8 == 0) hipLaunchKernelGGL((group_small_kernel<T, true, 1024>), dim3(blocks), dim3(1024), 0, st, A, parts);
    else hipLaunchKernelGGL((group_small_kernel<T, false, 1024>), dim3(blocks), dim3(1024), 0, st, A, parts);
}
template <typename T, bool TINY, int THREADS>
void launch(const GroupArgs& A, unsigned blocks, hipStream_t st)
{
    if (A.per_group % 8 == 0) hipLaunchKernelGGL((group_sums_kernel<T, TINY, true, THREADS>), dim3(blocks), dim3(THREADS), 0, st, A);
    else hipLaunchKernelGGL((group_sums_kernel<T, TINY, false, THREADS>), dim3(blocks), dim3(THREADS), 0, st, A);
    hipLaunchKernelGGL((group_norm_kernel<T, TINY, THREADS>), dim3(blocks), dim3(THREADS), 0, st, A);
}
template <int TYPE>
void launch_type(const GroupArgs& A, int parts, unsigned blocks, hipStream_t st)
{
    using T = typename TypeOf<TYPE>::T;
    if (parts) launch_small<T>(A, parts, blocks, st);
    else if (A.C < 8) launch<T, true, THREADS>(A, blocks, st);
    else if (A.units <= THREADS) launch<T, false, THREADS>(A, blocks, st);
    else launch<T, false, MOST_THREADS_EACH>(A, blocks, st);
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
    const size_t need = needed(d, images);
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
    A.aligned = (uintptr_t)y->data % 16 == 0 && y->stride * size_of(y->type) % 16 == 0;
    A.gamma = params->gamma; A.beta = params->beta;
    A.inv_count = 1.0 / ((double)d.rows_per_image * A.per_group);
    A.by_group = FastDiv(A.per_group);
    A.part = (Sums*)workspace;
    A.pivots = (float*)((char*)workspace + sums_bytes(d, images));
    const int parts = y->type == MIXAQ_I8 ? 0 : parts_of(d, images);
    const long long blocks = (long long)images * (parts ? parts : ch.count);
    if (blocks * (parts ? 1024 : threads_of(A.units)) >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d images are too many for one call", images);
    if (x->type == MIXAQ_F32) launch_type<MIXAQ_F32>(A, parts, (unsigned)blocks, (hipStream_t)stream);
    else if (x->type == MIXAQ_F16) launch_type<MIXAQ_F16>(A, parts, (unsigned)blocks, (hipStream_t)stream);
    else launch_type<MIXAQ_BF16>(A, parts, (unsigned)blocks, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // extern "C"
