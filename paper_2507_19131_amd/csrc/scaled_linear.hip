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

// The 32 outputs of one row that a lane holds, 16 from `col` on and 16 from col + 64 on.
__device__ __forceinline__ void finish(const LinearArgs& A, float (&v)[32], int nb, int g, int row)
{
    const int col = nb * SBLOCK + g * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            v[h * 16 + e] += A.bias[col + h * 64 + e];
            if (A.gelu) v[h * 16 + e] = gelu(v[h * 16 + e]);
        }
    if (A.y_type == MIXAQ_E4M3) {
        unsigned m = 0;                                   // outputs beyond N are gelu(0) = 0 (or NaN where the whole row is)
#pragma unroll
        for (int e = 0; e < 32; ++e) m = max(m, magnitude(v[e]));
        m = max(m, (unsigned)__shfl_xor((int)m, 16, 64));
        m = max(m, (unsigned)__shfl_xor((int)m, 32, 64));
        const BlockScale s = block_scale(m);
        if (row >= A.M) return;
        if (g == 0) A.sy[nb * A.ldsy + row] = s.scale;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = A.N - col - h * 64;
            uint8_t* p = (uint8_t*)A.y + row * A.ldy + col + h * 64;
            store_codes8(p, n, v + h * 16, s.inv);
            store_codes8(p + 8, n - 8, v + h * 16 + 8, s.inv);
        }
        return;
    }
    if (row >= A.M) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int n = A.N - col - h * 64;
        const long long at = row * A.ldy + col + h * 64;
        if (A.y_type == MIXAQ_F32) store16((float*)A.y + at, n, v + h * 16);
        else if (A.y_type == MIXAQ_F16) store16((_Float16*)A.y + at, n, v + h * 16);
        else store16((__bf16*)A.y + at, n, v + h * 16);
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
    finish(A, v, nb, g, row);
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
    if (y->type == MIXAQ_F32 || y->type == MIXAQ_E4M3) hipLaunchKernelGGL(linear_kernel<true>, dim3(A.tiles), dim3(256), 0, st, A);
    else hipLaunchKernelGGL(linear_kernel<false>, dim3(A.tiles), dim3(256), 0, st, A);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

}  // extern "C"
