// Linear layers on int8 codes with a scale per token and channel: y = act(x w^T + bias), the products on the int8 matrix instructions of gfx950,
// the sums exact; for one matrix, or for rows sorted by expert and a matrix for each.
#include "token.h"

#include <algorithm>
#include <new>

using namespace mixaq;

struct mixaq_token_linear {
    mixaq_token_linear_desc d;
    int KB, NB, device;               // blocks of 128 inputs and outputs
    uint8_t* packed = nullptr;        // [experts][NB][KB][8 tiles][2 halves][64 lanes] x 16 bytes, zero beyond K and N
    float* scales = nullptr;          // [experts][NB * 128], zeros beyond N
    float* bias = nullptr;            // the same, zeros without a bias
    void* memory = nullptr;
    ~mixaq_token_linear() { if (memory) (void)hipFree(memory); }
};

namespace {

struct TokenArgs {
    const void* x;                    // codes (token_few_kernel: or values)
    const float* sx;
    const uint8_t* w;
    const float *sw, *bias;
    void* y;
    const int *offsets, *gather;      // of rows sorted by expert
    const float* weights;
    long long ldx, ldy;
    int M, x_rows, N, K, KB, NB, act, experts;
};

// ---- layouts --------------------------------------------------------------------------------------------------------
// Weights are the row operand, activations the column operand, so that a lane's results are outputs of ONE row of x: its scale is a
// value of the lane.  The instruction takes of lane l row (or column) l % 16 and 16 bytes of k, chunk l / 16 of 64.  Its result r of lane l is
// row 4 * (l / 16) + r.  The rows of the 8 tiles of a block of 128 outputs are dealt so that a lane ends up with two runs of 16
// neighbouring outputs.  Beyond K the packed weights are zero, and since every code is a number, what stands there in x adds nothing.
constexpr int TILE_BYTES = 2048;                  // of packed weights: 16 outputs x 128 inputs
__device__ __forceinline__ int output_of(int tile, int row) { return (tile >> 2) * 64 + (row >> 2) * 16 + (tile & 3) * 4 + (row & 3); }

__global__ __launch_bounds__(256) void token_pack_kernel(const int8_t* w, long long ldw, int N, int K, int KB, int NB, v4i* packed, long long total)
{
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {     // one 16-byte piece
        const int lane = (int)i & 63, half = (int)(i >> 6) & 1, tile = (int)(i >> 7) & 7;
        const long long block = i >> 10, kb = block % KB, nb = block / KB % NB, e = block / KB / NB;
        const int n = (int)nb * SBLOCK + output_of(tile, lane & 15), k = (int)kb * SBLOCK + half * 64 + (lane >> 4) * 16;
        int8_t b[16] = {};
        if (n < N)
            for (int j = 0; j < 16; ++j)
                if (k + j < K) b[j] = w[(e * N + n) * ldw + k + j];
        v4i v;
        __builtin_memcpy(&v, b, 16);
        packed[i] = v;
    }
}
__global__ __launch_bounds__(256) void token_pack_vectors_kernel(const float* s, const float* bias, int N, int padded, long long total, float* scales, float* out)
{
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {
        const long long e = i / padded;
        const int n = (int)(i - e * padded);
        scales[i] = n < N ? s[e * N + n] : 0.0f;
        out[i] = bias && n < N ? bias[e * N + n] : 0.0f;
    }
}

// The rows of an expert, whatever the offsets say within 0 .. M.
__device__ __forceinline__ void rows_of(const TokenArgs& A, int e, int& first, int& end)
{
    first = min(max(A.offsets[e], 0), A.M);
    end = min(max(A.offsets[e + 1], first), A.M);
}
// The row of x that row r reads, or -1: then r is left as it was.
__device__ __forceinline__ int source_of(const TokenArgs& A, int r)
{
    if (!A.gather) return r;
    const int s = A.gather[r];
    return s >= 0 && s < A.x_rows ? s : -1;
}

// ---- operands straight from memory, K split over the waves --------------------------------------------------------------------
// A workgroup of NW waves computes 16 MR rows times NR tiles of 16 outputs, wave w the blocks w, w + NW, .. of K; the waves' sums meet in LDS.
// x may be given as values: the waves look for the rows' maxima first, each in its blocks, and quantize what they multiply.  SORTED: a workgroup takes
// all rows of its expert, one tile after the other.
template <int XT>
__device__ __forceinline__ void values_of(const void* row, int k0, int K, float (&v)[32])     // 16 from k0 on, 16 from k0 + 64 on
{
    using T = typename TypeOf<XT>::T;
    const T* const from = (const T*)row;
    T t[2][16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int k = k0 + h * 64;
        if (k + 16 <= K) __builtin_memcpy(t[h], from + k, sizeof(t[h]));
        else
#pragma unroll
            for (int e = 0; e < 16; ++e) t[h][e] = k + e < K ? from[k + e] : (T)0.0f;
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = (float)t[e >> 4][e & 15];
}

template <int XT, int YT, int MR, int NR, int NW, bool SORTED>
__global__ __launch_bounds__(NW * 64) void token_few_kernel(TokenArgs A, int per, FastDiv by_per, int groups)
{
    constexpr int FR = MR * NR;                                              // 16 x 16 results of the workgroup
    constexpr bool FROM_CODES = XT == MIXAQ_I8;
    using X = typename std::conditional<FROM_CODES, TypeOf<MIXAQ_E4M3>, TypeOf<XT>>::type::T;
    __shared__ v4i part[NW][FR][64];
    __shared__ unsigned top[NW][16 * MR];
    __shared__ float scale_of[16 * MR];
    __shared__ int source[16 * MR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // a run of workgroups per XCD; the row tiles of one run of weights beside one another
    const int per_xcd = (groups + 7) / 8, t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || t >= groups) return;            // the whole workgroup
    const int q = by_per(t), in = t - q * per, nt = SORTED ? in : q, nb = nt * NR / 8, tile0 = nt * NR % 8;
    if (nb * SBLOCK + output_of(tile0, 0) >= A.N) return;                    // (the tiles of the last block may all lie beyond)
    int first = in * 16 * MR, end = A.M;
    if (SORTED) rows_of(A, q, first, end);
    const long long layer = SORTED ? (long long)q * A.NB : 0;                // blocks of 128 outputs before this expert's
    const v4i* const w0 = (const v4i*)(A.w + ((layer + nb) * A.KB * 8 + tile0) * TILE_BYTES) + lane;
    for (int r0 = first; r0 < (SORTED ? end : first + 1); r0 += 16 * MR) {
        const X* from[MR];
        int src[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            const int r = min(r0 + m * 16 + c, end - 1);
            src[m] = SORTED ? source_of(A, r) : r;
            from[m] = (const X*)A.x + (long long)max(src[m], 0) * A.ldx;
        }
        RowScale s[MR];
        if constexpr (FROM_CODES) {
#pragma unroll
            for (int m = 0; m < MR; ++m) s[m].scale = A.sx[max(src[m], 0)];
        } else {
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                unsigned largest = 0;
                for (int kb = wave; kb < A.KB; kb += NW) {
                    float v[32];
                    values_of<XT>(from[m], kb * SBLOCK + g * 16, A.K, v);
#pragma unroll
                    for (int e = 0; e < 32; ++e) largest = max(largest, magnitude(v[e]));
                }
                largest = over4rows(largest, MaxOf());
                if (g == 0) top[wave][m * 16 + c] = largest;
            }
            __syncthreads();
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                unsigned largest = 0;
#pragma unroll
                for (int w = 0; w < NW; ++w) largest = max(largest, top[w][m * 16 + c]);
                s[m] = row_scale(largest);
            }
        }
        v4i acc[MR][NR] = {};
        for (int kb = wave; kb < A.KB; kb += NW) {
            v4i w[NR][2], x[MR][2];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                w[n][0] = w0[(kb * 8 + n) * 128];
                w[n][1] = w0[(kb * 8 + n) * 128 + 64];
            }
            const int k0 = kb * SBLOCK + g * 16;
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                if constexpr (FROM_CODES) {
                    x[m][0] = *(const v4i*)(from[m] + (k0 < A.K ? k0 : 0));
                    x[m][1] = *(const v4i*)(from[m] + (k0 + 64 < A.K ? k0 + 64 : 0));
                } else {
                    float v[32];
                    values_of<XT>(from[m], k0, A.K, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[m][i >> 2][i & 3] = int_codes4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], s[m].inv);
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int m = 0; m < MR; ++m) {
                    acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[n][0], x[m][0], acc[m][n], 0, 0, 0);
                    acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[n][1], x[m][1], acc[m][n], 0, 0, 0);
                }
        }
#pragma unroll
        for (int m = 0; m < MR; ++m) {
#pragma unroll
            for (int n = 0; n < NR; ++n) part[wave][m * NR + n][lane] = acc[m][n];
            if (wave == 0 && g == 0) {
                scale_of[m * 16 + c] = s[m].scale;
                source[m * 16 + c] = r0 + m * 16 + c < end ? src[m] : -1;
            }
        }
        __syncthreads();
        using T = typename TypeOf<YT>::T;
        const int used = min(NW, A.KB);
#pragma unroll
        for (int i = 0; i < (FR + NW - 1) / NW; ++i) {                       // results that a wave sums and finishes
            const int f = wave + i * NW;
            if (f >= FR) break;
            v4i sum = part[0][f][lane];
            for (int w = 1; w < used; ++w) sum += part[w][f][lane];
            const int own = f / NR * 16 + c, r = r0 + own, n0 = nb * SBLOCK + output_of(tile0 + f % NR, 4 * g);
            const float sx = scale_of[own];
            v4f sw, b;
            __builtin_memcpy(&sw, A.sw + layer * SBLOCK + n0, 16);
            __builtin_memcpy(&b, A.bias + layer * SBLOCK + n0, 16);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf((float)sum[e], sx * sw[e], b[e]);
            activate(v, A.act);
            if (source[own] < 0) continue;
            T out[4];
            const float weight = SORTED && A.weights ? A.weights[r] : 1.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = (T)(weight * v[e]);
            T* const to = (T*)A.y + (long long)r * A.ldy + n0;
            if (n0 + 4 <= A.N) __builtin_memcpy(to, out, sizeof(out));
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n0 + e < A.N) to[e] = out[e];
        }
        if (SORTED) __syncthreads();                                         // before the next tile's sums
    }
}

// Quantizes x first where it is given as values; behind the checks of the product that follows.
int quantize_first(const TokenArgs& A, const mixaq_rows* values, hipStream_t st)
{
    if (!values) return MIXAQ_OK;
    return launch_token_quantize(*values, A.x_rows, A.K, {(void*)A.x, A.ldx, MIXAQ_I8, (float*)A.sx, 0}, st);
}

template <int XT, int YT, int MR, int NR, int NW, bool SORTED>
int launch_few(const TokenArgs& A, const mixaq_rows* values, hipStream_t st)
{
    const long long columns = A.NB * 8 / NR, rows = ((long long)A.M + 16 * MR - 1) / (16 * MR), groups = SORTED ? A.experts * columns : rows * columns;
    const long long blocks = (groups + 7) / 8 * 8;
    if (blocks * NW * 64 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", A.M, A.N);
    const int rc = quantize_first(A, values, st);
    if (rc) return rc;
    const int per = (int)(SORTED ? columns : rows);
    hipLaunchKernelGGL((token_few_kernel<XT, YT, MR, NR, NW, SORTED>), dim3((unsigned)blocks), dim3(NW * 64), 0, st, A, per, FastDiv(per), (int)groups);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

template <int YT, bool SORTED>
int launch_linear(const TokenArgs& A, int x_type, const mixaq_rows* values, hipStream_t st)
{
    if (x_type == MIXAQ_F32) return launch_few<MIXAQ_F32, YT, 1, 1, 8, SORTED>(A, values, st);
    if (x_type == MIXAQ_F16) return launch_few<MIXAQ_F16, YT, 1, 1, 8, SORTED>(A, values, st);
    if (x_type == MIXAQ_BF16) return launch_few<MIXAQ_BF16, YT, 1, 1, 8, SORTED>(A, values, st);
    return launch_few<MIXAQ_I8, YT, 1, 1, 8, SORTED>(A, values, st);
}

// Whether values are quantized on their way into the product
bool quantized_inside(int x_rows) { return x_rows <= 16; }

// the workspace: codes and scales of x, where it is given as values and not quantized on its way into the product
size_t workspace_of(const mixaq_token_linear* h, int32_t x_rows, int32_t x_type)
{
    if (x_type == MIXAQ_I8 || x_rows == 0 || quantized_inside(x_rows)) return 0;
    return align256((size_t)x_rows * round_up16(h->d.K)) + align256((size_t)x_rows * 4);
}

int create(const mixaq_token_linear_desc* desc, const mixaq_token_linear_params* p, hipStream_t st, mixaq_token_linear** out)
{
    if (!out) return fail(MIXAQ_E_NULL, "out is NULL");
    *out = nullptr;
    if (!desc) return fail(MIXAQ_E_NULL, "descriptor is NULL");
    if (!p) return fail(MIXAQ_E_NULL, "params is NULL");
    const int K = desc->K, N = desc->N;
    if (K < 1 || K > 65536 || N < 1 || N > 65536) return fail(MIXAQ_E_SHAPE, "K=%d, N=%d outside 1..65536", K, N);
    if (desc->experts < 1 || desc->experts > 4096 || (long long)desc->experts * N > (1 << 24))
        return fail(MIXAQ_E_SHAPE, "experts=%d outside 1..4096 or over 2^24 rows of weights in all", desc->experts);
    if (desc->activation < ACT_NONE || desc->activation > ACT_RELU) return fail(MIXAQ_E_SHAPE, "unknown activation %d", desc->activation);
    int rc = check_token_rows(&p->w, "w", K, CODES);
    if (rc) return rc;
    mixaq_token_linear* h = new (std::nothrow) mixaq_token_linear();
    if (!h) return fail(MIXAQ_E_HIP, "out of host memory");
    struct Owner {                       // frees a half-built layer on every early return
        mixaq_token_linear* h;
        ~Owner() { delete h; }
    } owner{h};
    h->d = *desc;
    h->KB = blocks_of(K);
    h->NB = blocks_of(N);
    HIP_TRY(hipGetDevice(&h->device));
    const size_t codes = (size_t)desc->experts * h->NB * h->KB * 8 * TILE_BYTES, vectors = (size_t)desc->experts * h->NB * SBLOCK;
    HIP_TRY(hipMalloc(&h->memory, codes + 2 * vectors * 4));
    h->packed = (uint8_t*)h->memory;
    h->scales = (float*)(h->packed + codes);
    h->bias = h->scales + vectors;
    const long long pieces = (long long)(codes / 16);
    hipLaunchKernelGGL(token_pack_kernel, dim3((unsigned)std::min((pieces + 255) / 256, 1LL << 20)), dim3(256), 0, st, (const int8_t*)p->w.data,
                       (long long)p->w.stride, N, K, h->KB, h->NB, (v4i*)h->packed, pieces);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(token_pack_vectors_kernel, dim3((unsigned)std::min((vectors + 255) / 256, (size_t)1 << 14)), dim3(256), 0, st, p->w.scales, p->bias, N,
                       h->NB * SBLOCK, (long long)vectors, h->scales, h->bias);
    HIP_TRY(hipGetLastError());
    HIP_TRY(hipStreamSynchronize(st));
    owner.h = nullptr;
    *out = h;
    return MIXAQ_OK;
}

struct Sorted {
    const int32_t *offsets, *gather;
    const float* weights;
};

int forward(const mixaq_token_linear* h, const mixaq_rows* x, int32_t x_rows, const Sorted* sorted, const mixaq_rows* y, int32_t rows, void* workspace,
            size_t workspace_bytes, hipStream_t st)
{
    const int K = h->d.K, N = h->d.N;
    int rc = check_token_rows(x, "x", K, VALUES | CODES);
    if (!rc) rc = check_token_rows(y, "y", N, VALUES);
    if (rc) return rc;
    const Extent out = extent_of(*y, rows, N), in[2] = {extent_of(*x, x_rows, K), token_scales_of(*x, x_rows)};
    for (const Extent& i : in)
        if (overlap(out, i)) return fail(MIXAQ_E_SHAPE, "x and y overlap");
    const long long lists[3] = {h->d.experts * 4LL + 4, rows * 4LL, rows * 4LL};
    const void* const at[3] = {sorted ? sorted->offsets : nullptr, sorted ? sorted->gather : nullptr, sorted ? sorted->weights : nullptr};
    const char* const names[3] = {"offsets", "gather", "row_weights"};
    for (int i = 0; i < 3; ++i) {
        if ((uintptr_t)at[i] % 4) return fail(MIXAQ_E_SHAPE, "%s is not aligned", names[i]);
        if (overlap(out, memory_of(at[i], lists[i]))) return fail(MIXAQ_E_SHAPE, "y and %s overlap", names[i]);
    }
    int device = -1;
    HIP_TRY(hipGetDevice(&device));
    if (device != h->device) return fail(MIXAQ_E_SHAPE, "the layer was created on device %d, device %d is current", h->device, device);
    mixaq_rows codes = *x;
    const size_t need = workspace_of(h, x_rows, x->type);
    if (need) {
        if (!workspace) return fail(MIXAQ_E_NULL, "workspace is NULL (%zu bytes needed)", need);
        if (workspace_bytes < need) return fail(MIXAQ_E_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
        if ((uintptr_t)workspace & 255) return fail(MIXAQ_E_WORKSPACE, "workspace must be 256-byte aligned");
        const Extent ws = memory_of(workspace, (long long)need);
        if (overlap(ws, in[0]) || overlap(ws, out)) return fail(MIXAQ_E_SHAPE, "the workspace overlaps x or y");
        for (int i = 0; i < 3; ++i)
            if (overlap(ws, memory_of(at[i], lists[i]))) return fail(MIXAQ_E_SHAPE, "the workspace and %s overlap", names[i]);
        codes = {workspace, round_up16(K), MIXAQ_I8, (float*)((char*)workspace + align256((size_t)x_rows * round_up16(K))), 0};
    }
    TokenArgs A = {};
    A.x = codes.data; A.ldx = codes.stride;
    A.sx = codes.scales;
    A.w = h->packed; A.sw = h->scales; A.bias = h->bias;
    A.y = y->data; A.ldy = y->stride;
    A.M = rows; A.x_rows = x_rows; A.N = N; A.K = K; A.KB = h->KB; A.NB = h->NB;
    A.act = h->d.activation; A.experts = h->d.experts;
    const mixaq_rows* const values = need ? x : nullptr;
    if (sorted) {
        A.offsets = sorted->offsets; A.gather = sorted->gather; A.weights = sorted->weights;
        if (y->type == MIXAQ_F32) return launch_linear<MIXAQ_F32, true>(A, codes.type, values, st);
        if (y->type == MIXAQ_F16) return launch_linear<MIXAQ_F16, true>(A, codes.type, values, st);
        return launch_linear<MIXAQ_BF16, true>(A, codes.type, values, st);
    }
    if (y->type == MIXAQ_F32) return launch_linear<MIXAQ_F32, false>(A, codes.type, values, st);
    if (y->type == MIXAQ_F16) return launch_linear<MIXAQ_F16, false>(A, codes.type, values, st);
    return launch_linear<MIXAQ_BF16, false>(A, codes.type, values, st);
}

}  // namespace

extern "C" {

int mixaq_token_linear_create(const mixaq_token_linear_desc* desc, const mixaq_token_linear_params* params, void* stream, mixaq_token_linear** out)
{
    return create(desc, params, (hipStream_t)stream, out);
}

int mixaq_token_linear_destroy(mixaq_token_linear* h)
{
    delete h;
    return MIXAQ_OK;
}

int mixaq_token_linear_workspace_bytes(const mixaq_token_linear* h, int32_t x_rows, int32_t x_type, size_t* bytes)
{
    if (!h || !bytes) return fail(MIXAQ_E_NULL, "layer or bytes is NULL");
    if (x_rows < 0 || x_rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= x_rows <= 2^30 (got %d)", x_rows);
    if (x_type < MIXAQ_F32 || x_type > MIXAQ_I8 || x_type == MIXAQ_E4M3) return fail(MIXAQ_E_SHAPE, "unknown type %d", x_type);
    *bytes = workspace_of(h, x_rows, x_type);
    return MIXAQ_OK;
}

int mixaq_token_linear_forward(const mixaq_token_linear* h, const mixaq_rows* x, int32_t rows, const mixaq_rows* y, void* workspace, size_t workspace_bytes,
                               void* stream)
{
    if (!h) return fail(MIXAQ_E_NULL, "layer is NULL");
    if (rows < 0 || rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 (got %d)", rows);
    if (h->d.experts != 1) return fail(MIXAQ_E_SHAPE, "a layer of %d experts takes rows sorted by expert", h->d.experts);
    if (rows == 0) return MIXAQ_OK;
    return forward(h, x, rows, nullptr, y, rows, workspace, workspace_bytes, (hipStream_t)stream);
}

int mixaq_token_linear_forward_grouped(const mixaq_token_linear* h, const mixaq_rows* x, int32_t x_rows, const int32_t* offsets, const int32_t* gather,
                                       const float* row_weights, const mixaq_rows* y, int32_t rows, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!h) return fail(MIXAQ_E_NULL, "layer is NULL");
    if (rows < 0 || rows > MOST_ROWS || x_rows < 0 || x_rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows, x_rows <= 2^30 (got %d, %d)", rows, x_rows);
    if (!gather && x_rows < rows) return fail(MIXAQ_E_SHAPE, "%d rows of x for %d of y without a list", x_rows, rows);
    if (rows == 0 || x_rows == 0) return MIXAQ_OK;
    if (!offsets) return fail(MIXAQ_E_NULL, "offsets is NULL");
    const Sorted sorted = {offsets, gather, row_weights};
    return forward(h, x, x_rows, &sorted, y, rows, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
