// Linear layers on 8-bit float codes with a scale per 128 columns: y = act(x w^T + bias), the products on the e4m3 matrix
// instruction of gfx950, 128 deep, which is one block of scales.
#include "activations.h"
#include "scaled.h"
#include "scaled_forms.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

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

struct LinearArgs {
    const uint8_t* x;                 // codes (split_kernel: or values)
    const float* sx;
    const uint8_t* w;
    const float* sw;
    const float* bias;
    void* y;
    float* sy;
    long long ldx, ldsx, ldy, ldsy;
    int M, N, K, KB, NB, gelu;
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
// The end of a wave's ROWS rows and 128 outputs: a lane holds those of one row, the bias in them, in RUNS runs of 16 neighbouring ones, run i from
// column offset(i) of block nb on; the lanes l, l + ROWS, .. hold the whole row.  Through LDS (`turn`: 16 or 32 rows x 256 bytes of the
// wave's own), so that a store covers whole lines: from the lanes themselves it would touch 32 rows with 32 bytes each (268324 x 128 x 512 of bf16
// 115 us instead of 90, 100000 x 96 x 384 of f32 66 instead of 35).  Its 16-byte pieces are turned by the row, so that neither side meets a
// bank twice.  A block that ends beyond N is stored value by value.
template <int YT, int RUNS, int ROWS, typename Offset>
__device__ __forceinline__ void finish(const LinearArgs& A, float (&v)[16 * RUNS], int nb, long long row0, v4i* turn, Offset offset)
{
    using T = typename TypeOf<YT>::T;
    constexpr int ES = sizeof(T), ROW_BYTES = 128 * ES < 256 ? 128 * ES : 256, PASSES = 128 * ES / ROW_BYTES, PIECES = ROW_BYTES / 16;
    const int lane = threadIdx.x & 63, own = lane % ROWS, col = nb * SBLOCK;
    const long long row = row0 + own;
    if (A.gelu) {
#pragma unroll
        for (int e = 0; e < 16 * RUNS; ++e) v[e] = gelu(v[e]);
    }
    T t[RUNS][16];
    if constexpr (YT == MIXAQ_E4M3) {
        // two maxima of the bits, three values an instruction: of the positive numbers as integers, of the negative ones without a sign
        int up = 0;
        unsigned down = 0;
#pragma unroll
        for (int e = 0; e < 16 * RUNS; e += 2) {
            up = max(max(up, __float_as_int(v[e])), __float_as_int(v[e + 1]));
            down = max(max(down, __float_as_uint(v[e])), __float_as_uint(v[e + 1]));
        }
        unsigned largest = max((unsigned)up, (down >> 31) * (down & 0x7fffffffu));       // outputs beyond N are gelu(0) = 0 (or NaN where the row is)
#pragma unroll
        for (int d = ROWS; d < 64; d <<= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, d, 64));
        const BlockScale s = block_scale(largest);
        if (row < A.M && lane < ROWS) A.sy[nb * A.ldsy + row] = s.scale;
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
            for (int q = 0; q < 16; q += 4) {
                const int w = codes4(v[i * 16 + q], v[i * 16 + q + 1], v[i * 16 + q + 2], v[i * 16 + q + 3], s.inv);
                __builtin_memcpy(&t[i][q], &w, 4);
            }
    } else {
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) t[i][e] = (T)v[i * 16 + e];
    }
    if (col + SBLOCK > A.N) {
        if (row >= A.M) return;
        T* const y = (T*)A.y + row * A.ldy + col;
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (col + offset(i) + e < A.N) y[offset(i) + e] = t[i][e];
        return;
    }
    auto place = [](int r, int p) { return r * PIECES + (PIECES == 16 ? p ^ (r & 15) : p ^ (r >> 1 & 7)); };
    auto in_order = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };           // among the lanes of the wave, which runs in step
    uint8_t* const y = (uint8_t*)A.y + (row0 * A.ldy + col) * ES;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
#pragma unroll
        for (int i = pass * RUNS / PASSES; i < (pass + 1) * RUNS / PASSES; ++i) {
            const int p = offset(i) * ES % ROW_BYTES / 16;
#pragma unroll
            for (int q = 0; q < ES; ++q) __builtin_memcpy(&turn[place(own, p + q)], (const uint8_t*)t[i] + q * 16, 16);
        }
        in_order();
#pragma unroll
        for (int k = 0; k < ROWS * PIECES / 64; ++k) {
            const int r = (k * 64 + lane) / PIECES, p = (k * 64 + lane) % PIECES;
            const v4i piece = turn[place(r, p)];
            if (row0 + r < A.M) __builtin_memcpy(y + r * A.ldy * ES + pass * ROW_BYTES + p * 16, &piece, 16);
        }
        in_order();
    }
}

// 16 bytes of a row's codes from byte k on; bytes from K on are zero, so that what stands there takes no part (a NaN there, times a zero
// weight, would).
__device__ __forceinline__ void cut(v4i& c, int left)      // of the row's bytes from the chunk on
{
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] &= left >= 4 * q + 4 ? -1 : left <= 4 * q ? 0 : (1 << (8 * (left - 4 * q))) - 1;
}
__device__ __forceinline__ v4i load_codes(const uint8_t* row, int k, int K)
{
    v4i v = {0, 0, 0, 0};
    if (k < K) v = *(const v4i*)(row + k);
    cut(v, K - k);
    return v;
}

// ---- products of one block of 128 -----------------------------------------------------------------------------------------
// The 8-bit instruction sums groups of eight neighbouring products at the exponent of the largest of them and keeps 14 bits of each
// (measured: of 2^16 + 2^s within a group s = 3 arrives and s = 2 does not; across groups 24 bits do): up to 7 * 2^-13 of a group's largest product
// is lost, whatever is left of it when it cancels.  Of normal values that is 2e-5 of the results' root mean square, with a channel 12 times as large as
// the others 3e-5, 1000 times 1.1e-4: 1, 2 and 7 % of what rounding to bf16 costs, and results in bf16 are summed so.  Of f16's rounding it would be
// 10, 16 and 50 %; results in f16, those of 32 bits and those that become codes, whose scale is kept in 32 bits, are summed by the f16 instruction
// (e4m3 values are f16 values, their products exact, 1e-8), which takes twice the time (16384 x 4096 x 3840 480 us, to bf16 230).
constexpr bool exact_sums(int y_type) { return y_type != MIXAQ_BF16; }

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

// ---- operands straight from memory, K split over the waves --------------------------------------------------------------------
// A workgroup of NW waves computes 16 MR rows times NR tiles of 16 outputs, wave w the blocks w, w + NW, .. of K; the waves' sums meet in LDS,
// in the order of the waves.  For products of few tiles: a lone row at K = 1024 is one round trip to memory.  A block's scale meets
// its product where both are of one row, so x may be given as values: a lane holds 32 of the 128 values of its row, the other three
// lanes of the row the rest, and what it needs as operand is the codes of its own.  What bounds it: a launch and two round trips (1 x 1024 x 4096
// 2.7 us from codes, 3.7 from values; 4.2 MB of weights would take 0.8), with more rows the operands' way through the caches, each workgroup for
// itself (64 x 4096 x 4096 in 32 x 32 7.9 us: 34 MB of weights and as much of x, 8.5 TB/s; 1001 x 1000 x 333 in 16 x 16 6.0 us: 24 and 21 MB).
template <int XT>
__device__ __forceinline__ void operand_of(const LinearArgs& A, int row, int kb, int g, v4i (&x)[2], float& scale)
{
    const int k0 = kb * SBLOCK + g * 16;
    if constexpr (XT == MIXAQ_E4M3) {
        const uint8_t* const from = A.x + (long long)row * A.ldx;
        if ((kb + 1) * SBLOCK <= A.K) {
            x[0] = *(const v4i*)(from + k0);
            x[1] = *(const v4i*)(from + k0 + 64);
        } else {
            x[0] = load_codes(from, k0, A.K);
            x[1] = load_codes(from, k0 + 64, A.K);
        }
        scale = A.sx[kb * A.ldsx + row];
    } else {
        using T = typename TypeOf<XT>::T;
        const T* const from = (const T*)A.x + (long long)row * A.ldx;
        T t[2][16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if ((kb + 1) * SBLOCK <= A.K) __builtin_memcpy(t[h], from + k0 + h * 64, sizeof(t[h]));
            else
#pragma unroll
                for (int e = 0; e < 16; ++e) t[h][e] = k0 + h * 64 + e < A.K ? from[k0 + h * 64 + e] : (T)0.0f;
        }
        unsigned largest = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) largest = max(largest, magnitude((float)t[e >> 4][e & 15]));
        const BlockScale s = block_scale(over4rows(largest, MaxOf()));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) x[h][q] = codes4((float)t[h][4 * q], (float)t[h][4 * q + 1], (float)t[h][4 * q + 2], (float)t[h][4 * q + 3], s.inv);
        scale = s.scale;
    }
}

template <int XT, int YT, int MR, int NR, int NW>
__global__ __launch_bounds__(NW * 64) void split_kernel(LinearArgs A, int row_tiles, FastDiv by_rows, int groups)
{
    constexpr bool EXACT = exact_sums(YT);
    constexpr int FR = MR * NR;                                              // 16 x 16 results of the workgroup
    __shared__ v4f part[NW][FR][64];
    __shared__ unsigned top[YT == MIXAQ_E4M3 ? FR : 1][16];
    static_assert(YT != MIXAQ_E4M3 || NR == 8, "a row's codes need its whole block");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // a run of workgroups per XCD, the row tiles of one run of weights beside one another
    const int per_xcd = (groups + 7) / 8, t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || t >= groups) return;            // the whole workgroup
    const int nt = by_rows(t), rt = t - nt * row_tiles, nb = nt * NR / 8, tile0 = nt * NR % 8;
    if (nb * SBLOCK + output_of(tile0, 0) >= A.N) return;                    // (the tiles of the last block may all lie beyond)
    int row[MR];
#pragma unroll
    for (int m = 0; m < MR; ++m) row[m] = min(rt * 16 * MR + m * 16 + c, A.M - 1);
    v4f acc[MR][NR] = {};
    struct Operands {
        v4i x[MR][2], w[NR][2];
        float s[MR];
    };
    auto load = [&](int kb, Operands& o) {
        const v4i* const w = (const v4i*)(A.w + (((long long)nb * A.KB + kb) * 8 + tile0) * TILE_BYTES) + lane;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            o.w[n][0] = w[n * 128];
            o.w[n][1] = w[n * 128 + 64];
        }
        const float sw = A.sw[kb * A.NB + nb];
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            operand_of<XT>(A, row[m], kb, g, o.x[m], o.s[m]);
            o.s[m] *= sw;
        }
    };
    auto multiply = [&](const Operands& o) {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                const v4f d = product<EXACT>(o.w[n][0], o.w[n][1], o.x[m][0], o.x[m][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][n][e] = fmaf(d[e], o.s[m], acc[m][n][e]);
            }
    };
    if (wave < A.KB) {                                                       // one block's operands travel under the products of the last one
        Operands now;
        load(wave, now);
        for (int kb = wave + NW; kb < A.KB; kb += NW) {
            Operands next;
            load(kb, next);
            multiply(now);
            now = next;
        }
        multiply(now);
    }
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int n = 0; n < NR; ++n) part[wave][m * NR + n][lane] = acc[m][n];
    __syncthreads();
    constexpr int MINE = (FR + NW - 1) / NW;                                 // results that a wave sums and finishes
    v4f y[MINE];
    const int used = min(NW, A.KB);
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int f = wave + i * NW;
        if (f >= FR) break;
        v4f v = part[0][f][lane];
        for (int w = 1; w < used; ++w) v += part[w][f][lane];
        const int n0 = nb * SBLOCK + output_of(tile0 + f % NR, 4 * g);
        v4f b;
        __builtin_memcpy(&b, A.bias + n0, sizeof(b));
        v += b;
        if (A.gelu) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = gelu(v[e]);
        }
        y[i] = v;
        if constexpr (YT == MIXAQ_E4M3) {
            unsigned m = 0;                                                  // (outputs beyond N are gelu(0) = 0, or NaN where the whole row is)
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, magnitude(v[e]));
            m = over4rows(m, MaxOf());
            if (g == 0) top[f][c] = m;
        }
    }
    if constexpr (YT == MIXAQ_E4M3) __syncthreads();
    using T = typename TypeOf<YT>::T;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int f = wave + i * NW;
        if (f >= FR) break;
        const int r = rt * 16 * MR + f / NR * 16 + c, n0 = nb * SBLOCK + output_of(tile0 + f % NR, 4 * g);
        T out[4];
        if constexpr (YT == MIXAQ_E4M3) {
            unsigned m = 0;
#pragma unroll
            for (int n = 0; n < NR; ++n) m = max(m, top[f / NR * NR + n][c]);
            const BlockScale s = block_scale(m);
            const int w = codes4(y[i][0], y[i][1], y[i][2], y[i][3], s.inv);
            __builtin_memcpy(out, &w, 4);
            if (r < A.M && g == 0 && f % NR == 0) A.sy[nb * A.ldsy + r] = s.scale;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = (T)y[i][e];
        }
        if (r >= A.M) continue;
        T* const to = (T*)A.y + (long long)r * A.ldy + n0;
        if (n0 + 4 <= A.N) __builtin_memcpy(to, out, sizeof(out));
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n0 + e < A.N) to[e] = out[e];
    }
}

// ---- both operands through LDS ------------------------------------------------------------------------------------------
// A workgroup of WM x WN waves computes 32 MT WM rows times 128 WN outputs, a wave 32 MT rows times one block of 128 outputs: the product of a
// block's two scales is then a value per lane, and a row's codes need no exchange beyond the wave.  K goes in stages
// of one block of 128 through two LDS buffers filled by direct loads; a stage travels under the products of the one before it.
// Rows of x lie in LDS as 8 chunks of 16 bytes whose places are turned by half the row's number, so that the 16 lanes that are served
// together (16 rows, one chunk) meet all 64 banks.
// What bounds it: of 16384 x 4096 x 3840 to bf16 (240 to 280 us by card, 2.1 PFLOP/s; a library product without scales 2.4) the matrix instructions are
// busy in 52 % of the clocks and vector instructions in 41 %, and beside operands of 16 x 16 x 128 they hardly overlap; of codes out the vector
// instructions (61 %, with a GELU at K = 128 82 %).
// The direct loads are asm: as a builtin every LDS read behind them waits for all of them.  They do nothing for stages from `end` on, which the asm finds out: a branch around it would be one in the middle of a stage.
#define MIXAQ_REQUEST(SIZE_)                                                                                                              \
    int m0; /* given back: the compiler does not let an asm statement change it */                                                       \
    asm volatile("s_cmp_ge_i32 %4, %5\n\ts_cbranch_scc1 .Lskip%=\n\ts_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_" SIZE_ \
                 " %2, %3\n\ts_mov_b32 m0, %0\n.Lskip%=:" : "=&s"(m0) : "s"(lds_dst), "v"(lane_bytes), "s"(uniform_src), "s"(stage), "s"(end) : "memory", "scc")
__device__ __forceinline__ void request16(const void* uniform_src, unsigned lane_bytes, unsigned lds_dst, int stage, int end) { MIXAQ_REQUEST("dwordx4"); }
__device__ __forceinline__ void request4(const void* uniform_src, unsigned lane_bytes, unsigned lds_dst, int stage, int end) { MIXAQ_REQUEST("dword"); }
#undef MIXAQ_REQUEST
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(size_t)(const __attribute__((address_space(3))) char*)p; }

typedef float v16f __attribute__((ext_vector_type(16)));

// one half of an exact product of a block: the chunks 2 HALF and 2 HALF + 1 of a lane
template <int HALF>
__device__ __forceinline__ v16f half_product(const v4i (&w)[4], const v4i (&x)[4], v16f d)
{
#pragma unroll
    for (int j = 2 * HALF; j < 2 * HALF + 2; ++j) {
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(w[j][0], w[j][1]), widen(x[j][0], x[j][1]), d, 0, 0, 0);
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen(w[j][2], w[j][3]), widen(x[j][2], x[j][3]), d, 0, 0, 0);
    }
    return d;
}

// Of instructions of 32 x 32 the packed tiles 2 T and 2 T + 1 are rows 0 .. 31 of the T-th, and lane half h takes the 16-byte chunks h, 2 + h, 4 + h
// and 6 + h of a row's 128 bytes.  Result e is row 8 (e / 4) + 4 h + e % 4: of the outputs, by output_of, number 4 (2 (T % 2) + e / 8) + e % 4 of
// run 2 (e / 4 % 2) + h of 16, in half T / 2 of the block.
__device__ __forceinline__ int run_of(int i, int h) { return (i >> 1) * 64 + (2 * (i & 1) + h) * 16; }
__device__ __forceinline__ void in_runs(const v16f (&acc)[4], float (&v)[64])
{
#pragma unroll
    for (int T = 0; T < 4; ++T)
#pragma unroll
        for (int e = 0; e < 16; ++e) v[((T >> 1) * 2 + (e >> 2 & 1)) * 16 + ((T & 1) * 2 + (e >> 3)) * 4 + (e & 3)] = acc[T][e];
}
__device__ __forceinline__ void bias_of(const float* bias, int T, int h, v16f& acc)      // of the block's 128, for the results of the T-th
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v4f b;
        __builtin_memcpy(&b, bias + run_of((T >> 1) * 2 + (q & 1), h) + ((T & 1) * 2 + (q >> 1)) * 4, 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[q * 4 + e] = b[e];
    }
}

constexpr int MOST_KB = 65536 / SBLOCK;
constexpr int GROUP_M = 4;                        // row tiles that run beside one another

template <int YT, int MT, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 2) void tile_kernel(LinearArgs A, int tiles_m, int tiles_n, FastDiv by_group)
{
    constexpr bool EXACT = exact_sums(YT);
    constexpr int W = WM * WN, TM = 32 * MT * WM;
    constexpr int XP = TM * 8 / 64, WP = WN * 16, XL = XP / W, WL = WP / W;  // 1 KB pieces of a stage, of x and of w, and a wave's
    static_assert(XP % W == 0 && WP % W == 0 && TM / 64 <= W, "whole pieces a wave");
    __shared__ v4i xs[2][XP * 64], ws[2][WP * 64];
    __shared__ float sxs[2][TM], sws[WN][MOST_KB + 1];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, h = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    // a run of tiles per XCD, in groups of GROUP_M row tiles with all their outputs, so that what its CUs read at one time meets in its L2
    const int tiles = tiles_m * tiles_n, per_xcd = (tiles + 7) / 8;
    const int t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || t >= tiles) return;             // the whole workgroup
    const int group = by_group(t), in = t - group * GROUP_M * tiles_n, gm = min(GROUP_M, tiles_m - group * GROUP_M);
    const int tn = in / gm, tm = group * GROUP_M + in - tn * gm;
    const int row0 = tm * TM, nb0 = tn * WN, nb = nb0 + wn, KB = A.KB;

    // what this wave requests: rows (wave XL + i) 8 + lane / 8 of x, whose lanes take the chunk that belongs in their place, and pieces
    // wave WL + i of w; the first waves the scales of 64 rows each
    const uint8_t* xb = A.x + (long long)row0 * A.ldx;
    const float* sxb = A.sx + row0;
    static_assert(XL % 2 == 0, "the parity of a piece is that of i");
    const int chunk[2] = {((lane & 7) ^ (lane >> 4)) * 16, ((lane & 7) ^ (lane >> 4) ^ 4) * 16};     // of even and of odd pieces
    unsigned at[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) at[i] = (unsigned)(min((wave * XL + i) * 8 + (lane >> 3), A.M - 1 - row0) * (int)A.ldx + chunk[i & 1]);
    const uint8_t* wb = A.w + (long long)min(nb0 + wave * WL / 16, A.NB - 1) * KB * (8 * TILE_BYTES) + wave * WL % 16 * 1024;
    const int swave = wave % (TM / 64);                                      // (where there are more waves, twice)
    const unsigned srow = (unsigned)min(swave * 64 + lane, A.M - 1 - row0) * 4;
    const unsigned lx = lds_address(xs), lw = lds_address(ws), ls = lds_address(sxs);
    const int kb_tail = A.K % SBLOCK ? KB - 1 : KB;                          // chunks behind a row's end: the row's first, the weights there are zero
    auto request_x = [&](int kb, int i) {
        unsigned o = at[i];
        if (kb >= kb_tail && kb * SBLOCK + chunk[i & 1] >= A.K) o -= chunk[i & 1];
        request16(xb + kb * SBLOCK, o, lx + ((kb & 1) * XP + wave * XL + i) * 1024, kb, KB);
    };
    auto request_w = [&](int kb, int i) { request16(wb + (long long)kb * (8 * TILE_BYTES) + i * 1024, lane * 16, lw + ((kb & 1) * WP + wave * WL + i) * 1024, kb, KB); };
    auto request_s = [&](int kb) { request4(sxb + kb * A.ldsx, srow, ls + ((kb & 1) * TM + swave * 64) * 4, kb, KB); };
    auto landed = [&] {                                                      // every wave's requests, and its reads of the other buffer have returned
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < XL; ++i) request_x(0, i);
#pragma unroll
    for (int i = 0; i < WL; ++i) request_w(0, i);
    request_s(0);
    for (int i = tid; i < WN * KB; i += W * 64) {
        const int n = i / KB, kb = i - n * KB;
        sws[n][kb] = A.sw[kb * A.NB + min(nb0 + n, A.NB - 1)];
    }
    const int m0 = wm * 32 * MT;
    static_assert(2 * XP * 64 >= W * 512, "room for a wave's 32 rows of 256 bytes");
    v4i* const turn = &xs[0][0] + wave * 512;                                // (at the end)
    auto scale_of = [&](int kb, int row) { return sxs[kb & 1][row] * sws[wn][kb]; };
    landed();
#pragma unroll
    for (int i = 0; i < XL; ++i) request_x(1, i);
#pragma unroll
    for (int i = 0; i < WL; ++i) request_w(1, i);
    request_s(1);
    // The stages.  Beside a product run the sums of an earlier one, whose result is there by then: matrix and vector work of a wave side by side.  What
    // a product needs of LDS is read some products ahead; behind the last read of a stage the waves meet, and its buffer is requested anew.
    // (Without branches in a stage: the compiler moves the sums behind any, away from the matrix instructions.)
    if constexpr (!EXACT) {
        // instructions of 16 x 16 x 128, one a block: tile T of the packed eight, rows 16 i .. of the wave's; lane group g takes chunks g and 4 + g
        constexpr int MI = 2 * MT, P = 8 * MI, BEHIND = 2;
        static_assert(MI >= BEHIND, "the products of a stage that are added in the next one");
        const int c = lane & 15, g = lane >> 4;
        v4f acc[MI][8], d[4] = {};
#pragma unroll
        for (int T = 0; T < 8; ++T) {
            __builtin_memcpy(&acc[0][T], A.bias + min(nb, A.NB - 1) * SBLOCK + output_of(T, 4 * g), 16);
#pragma unroll
            for (int i = 1; i < MI; ++i) acc[i][T] = acc[0][T];
        }
        v4i x[MI][2], w[3][2];
        float s[MI], s_last[BEHIND] = {};
        const v4i* const xr[2] = {&xs[0][(m0 + c) * 8 + (g ^ (c >> 1))], &xs[0][(m0 + c) * 8 + ((g + 4) ^ (c >> 1))]};
        const v4i* const wr = &ws[0][wn * 1024 + lane];
        auto read_x = [&](int kb, int i) {
            x[i][0] = xr[0][(kb & 1) * (XP * 64) + i * 128];
            x[i][1] = xr[1][(kb & 1) * (XP * 64) + i * 128];
        };
        auto read_w = [&](int kb, int T, int to) {
            w[to][0] = wr[(kb & 1) * (WP * 64) + T * 128];
            w[to][1] = wr[(kb & 1) * (WP * 64) + T * 128 + 64];
        };
        auto add = [&](int p, float scale) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[p % MI][p / MI][e] = fmaf(d[p & 3][e], scale, acc[p % MI][p / MI][e]);
        };
        read_w(0, 0, 0);
        read_w(0, 1, 1);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            read_x(0, i);
            s[i] = scale_of(0, m0 + i * 16 + c);
        }
        auto stage = [&](int kb, auto more) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int T = p / MI, i = p % MI, behind = (p + P - BEHIND) % P;
                if (i == 0 && T < 6) read_w(kb, T + 2, (T + 2) % 3);
                if (i == 0 && T == 6 && more) landed();
                if (i == 0 && T >= 6 && more) read_w(kb + 1, T - 6, (T + 2) % 3);
                __builtin_amdgcn_sched_barrier(0);
                d[p & 3] = product<false>(w[T % 3][0], w[T % 3][1], x[i][0], x[i][1]);
                __builtin_amdgcn_sched_barrier(0);
                add(behind, p < BEHIND ? s_last[p] : s[behind % MI]);
                if (T == 7 && more) read_x(kb + 1, i);
                if (T >= 6 && more) {                                     // a request a product
                    const int q = p - 6 * MI, per = (XL + WL + 2 * MI - 1) / (2 * MI);
#pragma unroll
                    for (int k = q * per; k < (q + 1) * per; ++k) {
                        if (k < XL) request_x(kb + 2, k);
                        else if (k < XL + WL) request_w(kb + 2, k - XL);
                    }
                    if (q == 2 * MI - 1) request_s(kb + 2);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // w of the next stage's first tiles lie where (8 + T) % 3 says: back to their places
            const v4i a0 = w[2][0], a1 = w[2][1], b0 = w[0][0], b1 = w[0][1];
            w[0][0] = a0; w[0][1] = a1; w[1][0] = b0; w[1][1] = b1;
#pragma unroll
            for (int b = 0; b < BEHIND; ++b) s_last[b] = s[MI - BEHIND + b];
#pragma unroll
            for (int i = 0; i < MI; ++i)
                if (more) s[i] = scale_of(kb + 1, m0 + i * 16 + c);
        };
        auto cut_rows = [&] {                                                // what stands behind a row's end takes no part
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                cut(x[i][0], A.K - (KB - 1) * SBLOCK - g * 16);
                cut(x[i][1], A.K - (KB - 1) * SBLOCK - g * 16 - 64);
            }
        };
        // Of the large tile the stage stands here once, and the last one reads on like the others, for nobody: with a copy of its own some sums
        // would lie in scratch memory at the end, and a launch with scratch costs the more (16384 x 1024 x 4096 113 -> 84 us).  Small tiles
        // of few stages are faster with it (268324 x 128 x 512 of bf16 97 -> 88).
        constexpr bool ONCE = MT > 1;
#pragma unroll 1
        for (int kb = 0; kb < (ONCE ? KB : KB - 1); ++kb) {
            if (ONCE && kb == KB - 1 && (A.K & 15)) cut_rows();
            stage(kb, std::true_type());
        }
        if constexpr (!ONCE) {
            if (A.K & 15) cut_rows();
            stage(KB - 1, std::false_type());
        }
#pragma unroll
        for (int b = 0; b < BEHIND; ++b) add(P - BEHIND + b, s_last[b]);
        __syncthreads();                                                     // the last stage has been read
        if (nb >= A.NB) return;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            float v[32];
#pragma unroll
            for (int T = 0; T < 8; ++T)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[T * 4 + e] = acc[i][T][e];
            finish<YT, 2, 16>(A, v, nb, row0 + m0 + i * 16, turn, [&](int r) { return r * 64 + g * 16; });
        }
    } else {
        // instructions of 32 x 32 x 16: those of 16 x 16 have half their rate
        constexpr int P = 4 * MT;
        v16f acc[MT][4], d[2] = {};
#pragma unroll
        for (int T = 0; T < 4; ++T) {
            bias_of(A.bias + min(nb, A.NB - 1) * SBLOCK, T, h, acc[0][T]);
#pragma unroll
            for (int m = 1; m < MT; ++m) acc[m][T] = acc[0][T];
        }
        v4i x[MT][4], w[2][4];
        float s[MT], s_last = 0.0f;                                          // of this stage's rows; of the product still to be added
        auto read_x = [&](int kb, int m) {
            const int r = m0 + m * 32 + j;
#pragma unroll
            for (int c = 0; c < 4; ++c) x[m][c] = xs[kb & 1][r * 8 + ((2 * c + h) ^ (r >> 1 & 7))];
        };
        auto read_w = [&](int kb, int T) {
#pragma unroll
            for (int c = 0; c < 4; ++c) w[T & 1][c] = ws[kb & 1][wn * 1024 + ((2 * T + (j >> 4)) * 2 + (c >> 1)) * 64 + ((2 * c + h) & 3) * 16 + (j & 15)];
        };
        auto add = [&](int p, const v16f& from, float scale, int half) {     // half of product p to its sums
#pragma unroll
            for (int e = 8 * half; e < 8 * half + 8; ++e) acc[p % MT][p / MT][e] = fmaf(from[e], scale, acc[p % MT][p / MT][e]);
        };
        read_w(0, 0);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            read_x(0, m);
            s[m] = scale_of(0, m0 + m * 32 + j);
        }
        auto stage = [&](int kb, auto more) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int T = p / MT, m = p % MT, last = (p + P - 1) % P;
                const float scale = p == 0 ? s_last : s[last % MT];
                if (m == 0 && T < 3) read_w(kb, T + 1);
                if (m == 0 && T == 3 && more) {
                    landed();
                    read_w(kb + 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                d[p & 1] = half_product<0>(w[T & 1], x[m], (v16f){});
                add(last, d[(p & 1) ^ 1], scale, 0);
                __builtin_amdgcn_sched_barrier(0);
                d[p & 1] = half_product<1>(w[T & 1], x[m], d[p & 1]);
                add(last, d[(p & 1) ^ 1], scale, 1);
                __builtin_amdgcn_sched_barrier(0);
                if (T == 3 && m == MT - 1) s_last = s[m];
                if (T == 3 && more) {
                    read_x(kb + 1, m);
                    s[m] = scale_of(kb + 1, m0 + m * 32 + j);
#pragma unroll
                    for (int i = m * XL / MT; i < (m + 1) * XL / MT; ++i) request_x(kb + 2, i);
#pragma unroll
                    for (int i = m * WL / MT; i < (m + 1) * WL / MT; ++i) request_w(kb + 2, i);
                    if (m == 0) request_s(kb + 2);
                }
            }
        };
#pragma unroll 1
        for (int kb = 0; kb < KB - 1; ++kb) stage(kb, std::true_type());
        if (A.K & 15) {                                                      // what stands behind a row's end takes no part
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < 4; ++c) cut(x[m][c], A.K - (KB - 1) * SBLOCK - (2 * c + h) * 16);
        }
        stage(KB - 1, std::false_type());
        add(P - 1, d[(P - 1) & 1], s_last, 0);
        add(P - 1, d[(P - 1) & 1], s_last, 1);
        __syncthreads();                                                     // the last stage has been read
        if (nb >= A.NB) return;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float v[64];
            in_runs(acc[m], v);
            finish<YT, 4, 32>(A, v, nb, row0 + m0 + m * 32, turn, [&](int i) { return run_of(i, h); });
        }
    }
}

// Quantizes x first where it is given as values; behind the checks of the product that follows.
int quantize_first(const LinearArgs& A, const mixaq_rows* values, hipStream_t st)
{
    if (!values) return MIXAQ_OK;
    return launch_quantize(*values, A.M, A.K, 1, {(void*)A.x, A.ldx, MIXAQ_E4M3, (float*)A.sx, A.ldsx}, st);
}

template <int YT, int MT, int WM, int WN>
int launch_tiles(const LinearArgs& A, const mixaq_rows* values, hipStream_t st)
{
    constexpr int TM = 32 * MT * WM;
    const int tiles_m = (int)(((long long)A.M + TM - 1) / TM), tiles_n = (A.NB + WN - 1) / WN;
    const long long blocks = ((long long)tiles_m * tiles_n + 7) / 8 * 8;
    if (blocks * WM * WN * 64 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", A.M, A.N);
    const int rc = quantize_first(A, values, st);
    if (rc) return rc;
    hipLaunchKernelGGL((tile_kernel<YT, MT, WM, WN>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0, st, A, tiles_m, tiles_n, FastDiv(GROUP_M * tiles_n));
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

template <int XT, int YT, int MR, int NR, int NW>
int launch_split(const LinearArgs& A, const mixaq_rows* values, hipStream_t st)
{
    const long long row_tiles = ((long long)A.M + 16 * MR - 1) / (16 * MR), groups = row_tiles * (A.NB * 8 / NR);
    const long long blocks = (groups + 7) / 8 * 8;
    if (blocks * NW * 64 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", A.M, A.N);
    const int rc = quantize_first(A, values, st);
    if (rc) return rc;
    hipLaunchKernelGGL((split_kernel<XT, YT, MR, NR, NW>), dim3((unsigned)blocks), dim3(NW * 64), 0, st, A, (int)row_tiles, FastDiv((int)row_tiles), (int)groups);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

template <int XT, int YT>
int launch_few(const LinearArgs& A, const mixaq_rows* values, hipStream_t st)
{
    if constexpr (YT == MIXAQ_E4M3) return launch_split<XT, YT, 1, 8, 8>(A, values, st);
    else return launch_split<XT, YT, 1, 1, 8>(A, values, st);
}
template <int YT>
int launch_linear(const LinearArgs& A, ScaledForm form, int x_type, const mixaq_rows* values, hipStream_t st)
{
    switch (form) {
    case SCALED_FEW:
        if (x_type == MIXAQ_F32) return launch_few<MIXAQ_F32, YT>(A, values, st);
        if (x_type == MIXAQ_F16) return launch_few<MIXAQ_F16, YT>(A, values, st);
        if (x_type == MIXAQ_BF16) return launch_few<MIXAQ_BF16, YT>(A, values, st);
        return launch_few<MIXAQ_E4M3, YT>(A, values, st);
    case SCALED_MID:
        if constexpr (YT == MIXAQ_E4M3) return launch_split<MIXAQ_E4M3, YT, 1, 8, 8>(A, values, st);
        else return launch_split<MIXAQ_E4M3, YT, 2, 2, 8>(A, values, st);
    case SCALED_SPLIT:
        if constexpr (YT == MIXAQ_E4M3) return launch_split<MIXAQ_E4M3, YT, 2, 8, 4>(A, values, st);
        else return launch_split<MIXAQ_E4M3, YT, 4, 4, 4>(A, values, st);
    case SCALED_TILE: return launch_tiles<YT, 1, 4, 1>(A, values, st);
    default:
        if constexpr (exact_sums(YT)) return launch_tiles<YT, 1, 8, 1>(A, values, st);
        else return launch_tiles<YT, 2, 4, 2>(A, values, st);
    }
}

int round_up16(int v) { return (v + 15) / 16 * 16; }
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// the workspace: codes and scales of x, where it is given as values and not quantized on its way into the product
size_t workspace_of(const mixaq_scaled_linear* h, int32_t rows, int32_t x_type)
{
    if (x_type == MIXAQ_E4M3 || rows == 0 || quantized_inside(rows, h->KB, h->NB)) return 0;
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
    if (rows < 0 || rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 (got %d)", rows);
    for (int t : {x_type, y_type})
        if (t < MIXAQ_F32 || t > MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "unknown type %d", t);
    *bytes = workspace_of(h, rows, x_type);
    return MIXAQ_OK;
}

int mixaq_scaled_linear_forward(const mixaq_scaled_linear* h, const mixaq_rows* x, int32_t rows, const mixaq_rows* y, void* workspace,
                                size_t workspace_bytes, void* stream)
{
    if (!h) return fail(MIXAQ_E_NULL, "layer is NULL");
    if (rows < 0 || rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 (got %d)", rows);
    if (rows == 0) return MIXAQ_OK;
    const int K = h->d.K, N = h->d.N;
    int rc = check_rows(x, "x", K, true, rows);
    if (!rc) rc = check_rows(y, "y", N, true, rows);
    if (rc) return rc;
    const Extent in[2] = {extent_of(*x, rows, K), scales_of(*x, rows, K)}, out[2] = {extent_of(*y, rows, N), scales_of(*y, rows, N)};
    for (const Extent& o : out)
        for (const Extent& i : in)
            if (overlap(o, i)) return fail(MIXAQ_E_SHAPE, "x and y overlap");
    if (overlap(out[0], out[1])) return fail(MIXAQ_E_SHAPE, "codes and scales of y overlap");
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
        const Extent ws = {(uintptr_t)workspace, 0, 1, (long long)need};
        if (overlap(ws, in[0]) || overlap(ws, out[0]) || overlap(ws, out[1])) return fail(MIXAQ_E_SHAPE, "the workspace overlaps x or y");
        codes = {workspace, round_up16(K), MIXAQ_E4M3, (float*)((char*)workspace + align256((size_t)rows * round_up16(K))), rows};
    }
    LinearArgs A;
    A.x = (const uint8_t*)codes.data; A.ldx = codes.stride;
    A.sx = codes.scales; A.ldsx = codes.scale_stride;
    A.w = h->packed; A.sw = h->scales; A.bias = h->bias;
    A.y = y->data; A.ldy = y->stride;
    A.sy = y->scales; A.ldsy = y->scale_stride;
    A.M = rows; A.N = N; A.K = K; A.KB = h->KB; A.NB = h->NB;
    A.gelu = h->d.activation == 1;
    const ScaledForm form = scaled_form(rows, h->KB, h->NB, A.gelu, exact_sums(y->type), A.ldx);
    const mixaq_rows* const values = need ? x : nullptr;
    const int x_type = codes.type;
    switch (y->type) {
    case MIXAQ_F32: return launch_linear<MIXAQ_F32>(A, form, x_type, values, st);
    case MIXAQ_F16: return launch_linear<MIXAQ_F16>(A, form, x_type, values, st);
    case MIXAQ_BF16: return launch_linear<MIXAQ_BF16>(A, form, x_type, values, st);
    default: return launch_linear<MIXAQ_E4M3>(A, form, x_type, values, st);
    }
}

}  // extern "C"
