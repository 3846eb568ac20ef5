// Linear layers on 8-bit float codes with a scale per 128 columns: y = act(x w^T + bias), the products on the e4m3 matrix
// instruction of gfx950, 128 deep, which is one block of scales.
#include "scaled.h"

#include <algorithm>
#include <new>

#include "arena.h"

using namespace mixaq;

struct mixaq_scaled_linear {
    mixaq_scaled_linear_desc d;
    int KB, NB, device;               // blocks of 128 inputs and outputs
    uint8_t* packed = nullptr;        // [NB][KB][8 tiles][2 halves][64 lanes] x 16 bytes, zero beyond K and N
    float* scales = nullptr;          // [KB][NB]
    float* bias = nullptr;            // [NB * 128], zeros beyond N or without a bias
    void* memory = nullptr;
    ~mixaq_scaled_linear() { if (memory) (void)hipFree(memory); }
};

namespace {

#define HIP_TRY(expr)                                                                                   \
    do {                                                                                                \
        hipError_t e_ = (expr);                                                                         \
        if (e_ != hipSuccess) return fail(MIXAQ_E_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

struct LinearArgs {
    const uint8_t* x;                 // codes
    const float* sx;
    const uint8_t* w;
    const float* sw;
    const float* bias;
    void* y;
    float* sy;
    long long ldx, ldsx, ldy, ldsy;
    int M, N, K, KB, NB, y_type, gelu, tiles;
    FastDiv by_NB;
};

// ---- layouts --------------------------------------------------------------------------------------------------------
// Weights are the row operand, activations the column operand, so that a lane's results are outputs of ONE row of x: its scale is a
// value of the lane.  The instruction takes of lane l row (or column) l % 16 and two times 16 bytes of k; which k they are does
// not matter as long as both operands agree: 16-byte chunk l / 16 of the 128, and the same chunk of the second half.  Its result r of lane l is
// row 4 * (l / 16) + r.  The rows of the 8 tiles of a block of 128 outputs are dealt so that a lane ends up with two runs of 16
// neighbouring outputs: whole 16-byte stores of codes.
constexpr int TILE_BYTES = 2048;                  // of packed weights: 16 outputs x 128 inputs
__device__ __forceinline__ int output_of(int tile, int row) { return (tile >> 2) * 64 + (row >> 2) * 16 + (tile & 3) * 4 + (row & 3); }

__global__ __launch_bounds__(256) void pack_kernel(const uint8_t* w, long long ldw, int N, int K, int KB, int NB, v4i* packed, int total)
{
    const int i = blockIdx.x * 256 + threadIdx.x;               // one 16-byte piece
    if (i >= total) return;
    const int lane = i & 63, half = (i >> 6) & 1, tile = (i >> 7) & 7, block = i >> 10, kb = block % KB, nb = block / KB;
    const int n = nb * SBLOCK + output_of(tile, lane & 15), k = kb * SBLOCK + half * 64 + (lane >> 4) * 16;
    uint8_t b[16] = {};
    if (n < N)
        for (int e = 0; e < 16; ++e)
            if (k + e < K) b[e] = w[(long long)n * ldw + k + e];
    v4i v;
    __builtin_memcpy(&v, b, 16);
    packed[i] = v;
}
__global__ __launch_bounds__(256) void pack_vectors_kernel(const float* s, long long lds, const float* bias, int N, int KB, int NB, float* scales, float* out)
{
    for (int i = blockIdx.x * 256 + threadIdx.x; i < KB * NB; i += gridDim.x * 256) scales[i] = s[(long long)(i / NB) * lds + i % NB];
    for (int i = blockIdx.x * 256 + threadIdx.x; i < NB * SBLOCK; i += gridDim.x * 256) out[i] = bias && i < N ? bias[i] : 0.0f;
}

// ---- the end of a tile ------------------------------------------------------------------------------------------------
// GELU(v) = max(v, 0) - |v| erfc(|v| / sqrt 2) / 2, the erfc by Abramowitz and Stegun 7.1.26 (at most 1.5e-7 off): no
// difference of near values, as 1 + erf would be for negative v.  From |v| = 30 on the second term is 0; a NaN stays one.
__device__ __forceinline__ float gelu(float v)
{
    const float a = fminf(fabsf(v), 30.0f), z = a * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.0f));
    float p = fmaf(t, 1.061405429f, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float e = __builtin_amdgcn_exp2f(z * z * -1.44269504f);
    return (v < 0.0f ? 0.0f : v) - 0.5f * a * (p * t * e);
}

template <typename T>
__device__ __forceinline__ void store16(T* p, int n, const float* v)
{
    store8(p, n, v);
    store8(p + 8, n - 8, v + 8);
}

// The outputs of one row that a lane holds: RUNS runs of 16 neighbouring ones, run i from `col` + offset(i) on; `LANES` lanes
// (l, l + LANE_STEP, ..) hold a whole block of 128.
template <int RUNS, int LANE_STEP, typename Offset>
__device__ __forceinline__ void finish(const LinearArgs& A, float (&v)[16 * RUNS], int nb, int row, Offset offset)
{
    const int col = nb * SBLOCK;
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            v[i * 16 + e] += A.bias[col + offset(i) + e];
            if (A.gelu) v[i * 16 + e] = gelu(v[i * 16 + e]);
        }
    if (A.y_type == MIXAQ_E4M3) {
        unsigned m = 0;                                   // outputs beyond N are gelu(0) = 0 (or NaN where the whole row is)
#pragma unroll
        for (int e = 0; e < 16 * RUNS; ++e) m = max(m, magnitude(v[e]));
#pragma unroll
        for (int d = LANE_STEP; d < 64; d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d, 64));
        const BlockScale s = block_scale(m);
        if (row >= A.M) return;
        if ((threadIdx.x & 63) < LANE_STEP) A.sy[nb * A.ldsy + row] = s.scale;
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            const int n = A.N - col - offset(i);
            uint8_t* p = (uint8_t*)A.y + row * A.ldy + col + offset(i);
            store_codes8(p, n, v + i * 16, s.inv);
            store_codes8(p + 8, n - 8, v + i * 16 + 8, s.inv);
        }
        return;
    }
    if (row >= A.M) return;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        const int n = A.N - col - offset(i);
        const long long at = row * A.ldy + col + offset(i);
        if (A.y_type == MIXAQ_F32) store16((float*)A.y + at, n, v + i * 16);
        else if (A.y_type == MIXAQ_F16) store16((_Float16*)A.y + at, n, v + i * 16);
        else store16((__bf16*)A.y + at, n, v + i * 16);
    }
}

// 16 bytes of a row's codes from byte k on; bytes from K on are zero, so that what stands there takes no part (a NaN there, times a zero
// weight, would).
__device__ __forceinline__ v4i load_codes(const uint8_t* row, int k, int K)
{
    v4i v = {0, 0, 0, 0};
    if (k < K) v = *(const v4i*)(row + k);
    if (k + 16 > K) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int left = K - k - 4 * q;
            v[q] = left >= 4 ? v[q] : left <= 0 ? 0 : v[q] & ((1 << (8 * left)) - 1);
        }
    }
    return v;
}

// ---- products of one block of 128 -----------------------------------------------------------------------------------------
// The 8-bit instruction sums groups of eight neighbouring products at the exponent of the largest of them and keeps 14 bits of each
// (measured: of 2^16 + 2^s within a group s = 3 arrives and s = 2 does not; across groups 24 bits do): up to 7 * 2^-13 of a group's largest product,
// 1.5e-5 of the results' root mean square on normal values, 2.8e-5 with an outlier channel.  That is a hundredth of what rounding to bf16
// costs and a tenth of f16's, but not binary32: results of 32 bits, and those that become codes, whose scale is kept in 32 bits, are summed
// by the f16 instruction (e4m3 values are f16 values, their products exact, 1e-8), which takes twice the time.
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v8h widen(int lo, int hi)
{
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return (v8h){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <bool EXACT>
__device__ __forceinline__ v4f product(v4i w0, v4i w1, v4i x0, v4i x1)
{
    v4f d = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (EXACT) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(w0[0], w0[1]), widen(x0[0], x0[1]), d, 0, 0, 0);
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(w0[2], w0[3]), widen(x0[2], x0[3]), d, 0, 0, 0);
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(w1[0], w1[1]), widen(x1[0], x1[1]), d, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(w1[2], w1[3]), widen(x1[2], x1[3]), d, 0, 0, 0);
    } else {
        const v8i w = __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7), x = __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, d, 0, 0, 0, 0, 0, 0);
    }
}

// A wave per 16 rows and 128 outputs, operands straight from memory.
template <bool EXACT>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs A)
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int rt = A.by_NB(blockIdx.x), nb = blockIdx.x - rt * A.NB;
    const int row = rt * 64 + (threadIdx.x >> 6) * 16 + (lane & 15), r = min(row, A.M - 1);
    float v[32] = {};
    for (int kb = 0; kb < A.KB; ++kb) {
        const uint8_t* xr = A.x + r * A.ldx;
        const v4i x0 = load_codes(xr, kb * SBLOCK + g * 16, A.K), x1 = load_codes(xr, kb * SBLOCK + 64 + g * 16, A.K);
        const float s = A.sx[kb * A.ldsx + r] * A.sw[kb * A.NB + nb];
        const v4i* w = (const v4i*)(A.w + ((long long)nb * A.KB + kb) * 8 * TILE_BYTES) + lane;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const v4f d = product<EXACT>(w[t * 128], w[t * 128 + 64], x0, x1);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[t * 4 + e] = fmaf(d[e], s, v[t * 4 + e]);
        }
    }
    finish<2, 16>(A, v, nb, row, [&](int i) { return i * 64 + g * 16; });
}

// ---- both operands through LDS ------------------------------------------------------------------------------------------
// A workgroup of WM x WN waves computes 32 MT WM rows times 128 WN outputs, a wave 32 MT rows times one block of 128 outputs: the product of a
// block's two scales is then a value per lane, and a row's codes need no exchange but between the two halves of a wave.  K goes in stages
// of one block of 128 through two LDS buffers filled by direct loads; a stage travels under the products of the one before it.
// Instructions of 32 x 32: the packed tiles 2 T and 2 T + 1 are rows 0 .. 31 of the T-th, lane half h takes the 16-byte chunks
// h, 2 + h, 4 + h and 6 + h of a row's 128 bytes.  Rows of x lie in LDS as 8 chunks whose places are turned by the row, so that the lanes that are
// served together (eight rows, one chunk) meet all banks.
// The direct loads are asm: as a builtin every LDS read behind them waits for all of them.
__device__ __forceinline__ void request16(const void* uniform_src, unsigned lane_bytes, unsigned lds_dst)
{
    int m0;                                                              // given back: the compiler does not let an asm statement change it
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds_dst), "v"(lane_bytes), "s"(uniform_src) : "memory");
}
__device__ __forceinline__ void request4(const void* uniform_src, unsigned lane_bytes, unsigned lds_dst)
{
    int m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds_dst), "v"(lane_bytes), "s"(uniform_src) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(size_t)(const __attribute__((address_space(3))) char*)p; }

typedef float v16f __attribute__((ext_vector_type(16)));

template <bool EXACT>
__device__ __forceinline__ v16f product32(const v4i (&w)[4], const v4i (&x)[4])
{
    v16f d = {};
    if constexpr (EXACT) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(w[j][0], w[j][1]), widen(x[j][0], x[j][1]), d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(w[j][2], w[j][3]), widen(x[j][2], x[j][3]), d, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const v8i a = __builtin_shufflevector(w[j], w[j + 1], 0, 1, 2, 3, 4, 5, 6, 7), b = __builtin_shufflevector(x[j], x[j + 1], 0, 1, 2, 3, 4, 5, 6, 7);
            d = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, d, 0, 0, 0, 0, 0, 0);
        }
    }
    return d;
}

constexpr int MOST_KB = 65536 / SBLOCK;
constexpr int GROUP_M = 8;                        // row tiles that run beside one another

template <bool EXACT, int MT, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 1) void tile_kernel(LinearArgs A, int tiles_m, int tiles_n, FastDiv by_group)
{
    constexpr int W = WM * WN, TM = 32 * MT * WM;
    constexpr int XP = TM * 8 / 64, WP = WN * 16, LPW = (XP + WP) / W;       // 1 KB pieces of a stage: of x, of w, and a wave's
    static_assert((XP + WP) % W == 0 && TM / 64 <= W && LPW < 60, "whole pieces a wave");
    __shared__ v4i xs[2][XP * 64], ws[2][WP * 64];
    __shared__ float sxs[2][TM], sws[WN][MOST_KB];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, h = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    // a run of tiles per XCD, in groups of GROUP_M row tiles with all their outputs, so that what its CUs read at one time meets in its L2
    const int tiles = tiles_m * tiles_n, per_xcd = (tiles + 7) / 8;
    const int t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || t >= tiles) return;             // the whole workgroup
    const int group = by_group(t), in = t - group * GROUP_M * tiles_n, gm = min(GROUP_M, tiles_m - group * GROUP_M);
    const int tn = in / gm, tm = group * GROUP_M + in - tn * gm;
    const int row0 = tm * TM, nb0 = tn * WN, nb = nb0 + wn;

    const uint8_t* xb = A.x + (long long)row0 * A.ldx;
    const float* sxb = A.sx + row0;
    unsigned at[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int p = wave * LPW + i;                                        // this wave's i-th piece
        const int r = p * 8 + (lane >> 3), chunk = (lane & 7) ^ (r & 7);
        at[i] = p < XP ? (unsigned)(min(r, A.M - 1 - row0) * (int)A.ldx + chunk * 16) : lane * 16;
    }
    const unsigned srow = (unsigned)min(wave * 64 + lane, A.M - 1 - row0) * 4;
    const unsigned lx = lds_address(xs), lw = lds_address(ws), ls = lds_address(sxs);
    auto request = [&](int kb) {
        const int b = kb & 1;
        const bool tail = (kb + 1) * SBLOCK > A.K;                           // chunks behind a row's end: any of the row, the weights there are zero
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int p = wave * LPW + i;
            if (p < XP) {
                unsigned o = at[i];
                const int chunk = (lane & 7) ^ ((p * 8 + (lane >> 3)) & 7);
                if (tail && kb * SBLOCK + chunk * 16 >= A.K) o -= chunk * 16;
                request16(xb + kb * SBLOCK, o, lx + (b * XP + p) * 1024);
            } else {
                const int q = p - XP, n = min(nb0 + q / 16, A.NB - 1);
                request16(A.w + ((long long)n * A.KB + kb) * (8 * TILE_BYTES) + (q % 16) * 1024, at[i], lw + (b * WP + q) * 1024);
            }
        }
        if (wave < TM / 64) request4(sxb + kb * A.ldsx, srow, ls + (b * TM + wave * 64) * 4);
    };
    request(0);
    for (int i = tid; i < WN * A.KB; i += W * 64) {
        const int n = i / A.KB, kb = i - n * A.KB;
        sws[n][kb] = A.sw[kb * A.NB + min(nb0 + n, A.NB - 1)];
    }
    v16f acc[MT][4] = {};
    const int m0 = wm * 32 * MT;
    for (int kb = 0; kb < A.KB; ++kb) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");          // this stage has landed, this wave's reads of the last one have returned
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kb + 1 < A.KB) request(kb + 1);
        const int b = kb & 1;
        v4i x[MT][4];
        float s[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int r = m0 + m * 32 + j;
#pragma unroll
            for (int c = 0; c < 4; ++c) x[m][c] = xs[b][r * 8 + ((2 * c + h) ^ (r & 7))];
            s[m] = sxs[b][r] * sws[wn][kb];
        }
        if ((A.K & 15) && kb == A.KB - 1) {                                  // what stands behind a row's end takes no part
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int left = A.K - kb * SBLOCK - (2 * c + h) * 16 - 4 * q;
                    const int mask = left >= 4 ? -1 : left <= 0 ? 0 : (1 << (8 * left)) - 1;
#pragma unroll
                    for (int m = 0; m < MT; ++m) x[m][c][q] &= mask;
                }
        }
#pragma unroll
        for (int T = 0; T < 4; ++T) {
            v4i w[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = ws[b][wn * 1024 + ((2 * T + (j >> 4)) * 2 + (c >> 1)) * 64 + ((2 * c + h) & 3) * 16 + (j & 15)];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const v16f d = product32<EXACT>(w, x[m]);
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[m][T][e] = fmaf(d[e], s[m], acc[m][T][e]);
            }
        }
    }
    if (nb >= A.NB) return;
    // result e of the T-th instruction is its row 8 (e / 4) + 4 h + e % 4: of the outputs, with output_of, number 4 (2 (T % 2) + e / 8) + e % 4 of
    // run 2 (e / 4 % 2) + h of 16, in half T / 2 of the block
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float v[64];
#pragma unroll
        for (int T = 0; T < 4; ++T)
#pragma unroll
            for (int e = 0; e < 16; ++e) v[((T >> 1) * 2 + (e >> 2 & 1)) * 16 + ((T & 1) * 2 + (e >> 3)) * 4 + (e & 3)] = acc[m][T][e];
        finish<4, 32>(A, v, nb, row0 + m0 + m * 32 + j, [&](int i) { return (i >> 1) * 64 + (2 * (i & 1) + h) * 16; });
    }
}

template <bool EXACT, int MT, int WM, int WN>
int launch_tiles(const LinearArgs& A, hipStream_t st)
{
    constexpr int TM = 32 * MT * WM;
    const int tiles_m = (int)(((long long)A.M + TM - 1) / TM), tiles_n = (A.NB + WN - 1) / WN;
    const long long blocks = ((long long)tiles_m * tiles_n + 7) / 8 * 8;
    if (blocks * WM * WN * 64 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", A.M, A.N);
    hipLaunchKernelGGL((tile_kernel<EXACT, MT, WM, WN>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0, st, A, tiles_m, tiles_n, FastDiv(GROUP_M * tiles_n));
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

int round_up16(int v) { return (v + 15) / 16 * 16; }
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// the workspace: codes and scales of x, where it is given as values
size_t workspace_of(const mixaq_scaled_linear* h, int32_t rows, int32_t x_type)
{
    if (x_type == MIXAQ_E4M3 || rows == 0) return 0;
    return align256((size_t)rows * round_up16(h->d.K)) + align256((size_t)rows * h->KB * 4);
}

int create(const mixaq_scaled_linear_desc* desc, const mixaq_scaled_linear_params* p, hipStream_t st, mixaq_scaled_linear** out)
{
    if (!out) return fail(MIXAQ_E_NULL, "out is NULL");
    *out = nullptr;
    if (!desc) return fail(MIXAQ_E_NULL, "descriptor is NULL");
    if (!p) return fail(MIXAQ_E_NULL, "params is NULL");
    const int K = desc->K, N = desc->N;
    if (K < 1 || K > 65536 || N < 1 || N > 65536) return fail(MIXAQ_E_SHAPE, "K=%d, N=%d outside 1..65536", K, N);
    if (desc->activation != 0 && desc->activation != 1) return fail(MIXAQ_E_SHAPE, "unknown activation %d", desc->activation);
    if (p->w.type != MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "w must be codes");
    int rc = check_rows(&p->w, "w", K, true, blocks_of(N));
    if (rc) return rc;
    mixaq_scaled_linear* h = new (std::nothrow) mixaq_scaled_linear();
    if (!h) return fail(MIXAQ_E_HIP, "out of host memory");
    struct Owner {                       // frees a half-built layer on every early return
        mixaq_scaled_linear* h;
        ~Owner() { delete h; }
    } owner{h};
    h->d = *desc;
    h->KB = blocks_of(K);
    h->NB = blocks_of(N);
    HIP_TRY(hipGetDevice(&h->device));
    const size_t codes = (size_t)h->NB * h->KB * 8 * TILE_BYTES, scales = align256((size_t)h->NB * h->KB * 4);
    HIP_TRY(hipMalloc(&h->memory, codes + scales + (size_t)h->NB * SBLOCK * 4));
    h->packed = (uint8_t*)h->memory;
    h->scales = (float*)(h->packed + codes);
    h->bias = (float*)(h->packed + codes + scales);
    const int pieces = (int)(codes / 16);                // at most 2^28
    hipLaunchKernelGGL(pack_kernel, dim3((pieces + 255) / 256), dim3(256), 0, st, (const uint8_t*)p->w.data, (long long)p->w.stride, N, K, h->KB,
                       h->NB, (v4i*)h->packed, pieces);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(pack_vectors_kernel, dim3(std::min((h->NB * std::max(h->KB, SBLOCK) + 255) / 256, 1024)), dim3(256), 0, st, p->w.scales,
                       (long long)p->w.scale_stride, p->bias, N, h->KB, h->NB, h->scales, h->bias);
    HIP_TRY(hipGetLastError());
    HIP_TRY(hipStreamSynchronize(st));
    owner.h = nullptr;
    *out = h;
    return MIXAQ_OK;
}

}  // namespace

extern "C" {

int mixaq_scaled_linear_create(const mixaq_scaled_linear_desc* desc, const mixaq_scaled_linear_params* params, void* stream,
                               mixaq_scaled_linear** out)
{
    return create(desc, params, (hipStream_t)stream, out);
}

int mixaq_scaled_linear_destroy(mixaq_scaled_linear* h)
{
    delete h;
    return MIXAQ_OK;
}

int mixaq_scaled_linear_workspace_bytes(const mixaq_scaled_linear* h, int32_t rows, int32_t x_type, int32_t y_type, size_t* bytes)
{
    if (!h || !bytes) return fail(MIXAQ_E_NULL, "layer or bytes is NULL");
    if (rows < 0) return fail(MIXAQ_E_SHAPE, "rows must not be negative (got %d)", rows);
    for (int t : {x_type, y_type})
        if (t < MIXAQ_F32 || t > MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "unknown type %d", t);
    *bytes = workspace_of(h, rows, x_type);
    return MIXAQ_OK;
}

int mixaq_scaled_linear_forward(const mixaq_scaled_linear* h, const mixaq_rows* x, int32_t rows, const mixaq_rows* y, void* workspace,
                                size_t workspace_bytes, void* stream)
{
    if (!h) return fail(MIXAQ_E_NULL, "layer is NULL");
    if (rows < 0) return fail(MIXAQ_E_SHAPE, "rows must not be negative (got %d)", rows);
    if (rows == 0) return MIXAQ_OK;
    const int K = h->d.K, N = h->d.N;
    int rc = check_rows(x, "x", K, true, rows);
    if (!rc) rc = check_rows(y, "y", N, true, rows);
    if (rc) return rc;
    if (rows_overlap(*x, rows, K, *y, rows, N)) return fail(MIXAQ_E_SHAPE, "x and y overlap");
    int device = -1;
    HIP_TRY(hipGetDevice(&device));
    if (device != h->device) return fail(MIXAQ_E_SHAPE, "the layer was created on device %d, device %d is current", h->device, device);
    const hipStream_t st = (hipStream_t)stream;
    mixaq_rows codes = *x;
    const size_t need = workspace_of(h, rows, x->type);
    if (need) {
        if (!workspace) return fail(MIXAQ_E_NULL, "workspace is NULL (%zu bytes needed)", need);
        if (workspace_bytes < need) return fail(MIXAQ_E_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
        if ((uintptr_t)workspace & 255) return fail(MIXAQ_E_WORKSPACE, "workspace must be 256-byte aligned");
        const mixaq_rows ws = {workspace, (int64_t)need, MIXAQ_E4M3, nullptr, 0};
        if (rows_overlap(ws, 1, (int32_t)std::min<size_t>(need, INT32_MAX), *x, rows, K) ||
            rows_overlap(ws, 1, (int32_t)std::min<size_t>(need, INT32_MAX), *y, rows, N))
            return fail(MIXAQ_E_SHAPE, "the workspace overlaps x or y");
        codes = {workspace, round_up16(K), MIXAQ_E4M3, (float*)((char*)workspace + align256((size_t)rows * round_up16(K))), rows};
    }
    LinearArgs A;
    A.x = (const uint8_t*)codes.data; A.ldx = codes.stride;
    A.sx = codes.scales; A.ldsx = codes.scale_stride;
    A.w = h->packed; A.sw = h->scales; A.bias = h->bias;
    A.y = y->data; A.ldy = y->stride;
    A.sy = y->scales; A.ldsy = y->scale_stride;
    A.M = rows; A.N = N; A.K = K; A.KB = h->KB; A.NB = h->NB;
    A.y_type = y->type; A.gelu = h->d.activation == 1;
    A.by_NB = FastDiv(h->NB);
    const long long tiles = (long long)((rows + 63LL) / 64) * h->NB;
    if (tiles * 256 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", rows, N);
    A.tiles = (int)tiles;
    if (need) {
        rc = launch_quantize(*x, rows, K, 1, codes, st);
        if (rc) return rc;
    }
    const bool exact = y->type == MIXAQ_F32 || y->type == MIXAQ_E4M3;
    if ((long long)((rows + 255) / 256) * ((h->NB + 1) / 2) >= 256 && h->KB >= 4 && A.ldx < (1 << 22))
        return exact ? launch_tiles<true, 1, 8, 1>(A, st) : launch_tiles<false, 2, 4, 2>(A, st);
    if (exact) hipLaunchKernelGGL(linear_kernel<true>, dim3(A.tiles), dim3(256), 0, st, A);
    else hipLaunchKernelGGL(linear_kernel<false>, dim3(A.tiles), dim3(256), 0, st, A);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // extern "C"
