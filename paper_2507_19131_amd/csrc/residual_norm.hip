// y = residual_scale * x + gate * post_norm(branch), out = pre_norm(y): what stands between two layers of a residual stream, in one
// pass over x and branch.
#include "scaled.h"

#include <algorithm>
#include <cmath>

using namespace mixaq;

namespace {

#define HIP_TRY(expr)                                                                                   \
    do {                                                                                                \
        hipError_t e_ = (expr);                                                                         \
        if (e_ != hipSuccess) return fail(MIXAQ_E_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

enum { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };

struct NormArgs {
    const void *x, *branch;
    void *y, *out;
    float* scales;
    long long ldx, ldb, ldy, ldo, lds;
    int rows, C, post, pre, out_type, rows_per_gate;
    float post_eps, pre_eps, residual_scale, inv_C;
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta, *gate;
};

// Sum over the G lanes of a row; with more than a wave, through LDS (`part`: a float per wave, free again after the call).
template <int G>
__device__ __forceinline__ float row_sum(float v, float* part)
{
#pragma unroll
    for (int d = (G < 64 ? G : 64) / 2; d; d >>= 1) v += __shfl_xor(v, d, 64);
    if constexpr (G > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) v += part[w];
    }
    return v;
}

// One norm of a row whose values lie in registers, V times eight a lane: mean first, then the squares of what is left, so that
// a large mean costs no digits.  Sums in binary32.
template <int G, int V>
__device__ __forceinline__ void norm_row(float (&v)[V][8], int kind, float eps, const float* gamma, const float* beta, const NormArgs& A,
                                         int l, float* part)
{
    float mean = 0.0f;
    if (kind == NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[j][e];
        mean = row_sum<G>(s, part) * A.inv_C;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int n = A.C - (j * G + l) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[j][e] = e < n ? v[j][e] - mean : 0.0f;
            q = fmaf(v[j][e], v[j][e], q);
        }
    }
    const float r = 1.0f / sqrtf(row_sum<G>(q, part) * A.inv_C + eps);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int col = (j * G + l) * 8, n = A.C - col;
        float g[8], b[8];
        if (gamma) load8(gamma + col, n, g);
        if (beta) load8(beta + col, n, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[j][e] *= r;
            if (gamma) v[j][e] *= g[e];
            if (beta) v[j][e] += b[e];
        }
    }
}

template <int TX, int TB, int G, int V>
__global__ __launch_bounds__(256) void residual_norm_kernel(NormArgs A)
{
    using X = typename TypeOf<TX>::T;
    using B = typename TypeOf<TB>::T;
    __shared__ float part[4];
    const int l = threadIdx.x % G, rows_at_once = 256 / G;
    for (long long r0 = (long long)blockIdx.x * rows_at_once; r0 < A.rows; r0 += (long long)gridDim.x * rows_at_once) {
        const long long row = r0 + threadIdx.x / G;
        const long long at = row < A.rows ? row : A.rows - 1;        // spare lanes take the last row along and store nothing
        float y[V][8];
        if (A.branch) {
#pragma unroll
            for (int j = 0; j < V; ++j) load8((const B*)A.branch + at * A.ldb + (j * G + l) * 8, A.C - (j * G + l) * 8, y[j]);
            if (A.post) norm_row<G, V>(y, A.post, A.post_eps, A.post_gamma, A.post_beta, A, l, part);
        }
        const float* gate = A.gate ? A.gate + (long long)((int)at / A.rows_per_gate) * A.C : nullptr;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int col = (j * G + l) * 8, n = A.C - col;
            float x[8], g[8];
            load8((const X*)A.x + at * A.ldx + col, n, x);
            if (gate) load8(gate + col, n, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float b = A.branch ? (gate ? y[j][e] * g[e] : y[j][e]) : 0.0f;
                y[j][e] = fmaf(A.residual_scale, x[e], b);
            }
            if (A.y && row < A.rows && n > 0) store8((X*)A.y + row * A.ldy + col, n, y[j]);
        }
        if (!A.out) continue;
        if (A.pre) norm_row<G, V>(y, A.pre, A.pre_eps, A.pre_gamma, A.pre_beta, A, l, part);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int col = (j * G + l) * 8, n = A.C - col;
            if (A.out_type == MIXAQ_E4M3) {
                const BlockScale s = block_scale(max16(max_magnitude(y[j])));
                if (row < A.rows && n > 0) {
                    store_codes8((uint8_t*)A.out + row * A.ldo + col, n, y[j], s.inv);
                    if ((l & 15) == 0) A.scales[(long long)(col / SBLOCK) * A.lds + row] = s.scale;
                }
            } else if (row < A.rows && n > 0) {
                if (A.out_type == MIXAQ_F32) store8((float*)A.out + row * A.ldo + col, n, y[j]);
                else if (A.out_type == MIXAQ_F16) store8((_Float16*)A.out + row * A.ldo + col, n, y[j]);
                else store8((__bf16*)A.out + row * A.ldo + col, n, y[j]);
            }
        }
    }
}

template <int TX, int TB, int G, int V>
void launch(const NormArgs& A, hipStream_t st)
{
    const long long groups = ((long long)A.rows + 256 / G - 1) / (256 / G);
    hipLaunchKernelGGL((residual_norm_kernel<TX, TB, G, V>), dim3((unsigned)std::min(groups, 1LL << 23)), dim3(256), 0, st, A);
}
// The lanes of a row: 16 as long as three vectors of eight hold their share, then a wave, then a workgroup.
template <int TX, int TB>
void launch_types(const NormArgs& A, hipStream_t st)
{
    if (A.C <= 128) launch<TX, TB, 16, 1>(A, st);
    else if (A.C <= 256) launch<TX, TB, 16, 2>(A, st);
    else if (A.C <= 384) launch<TX, TB, 16, 3>(A, st);
    else if (A.C <= 512) launch<TX, TB, 64, 1>(A, st);
    else if (A.C <= 1024) launch<TX, TB, 64, 2>(A, st);
    else if (A.C <= 2048) launch<TX, TB, 64, 4>(A, st);
    else if (A.C <= 4096) launch<TX, TB, 256, 2>(A, st);
    else if (A.C <= 8192) launch<TX, TB, 256, 4>(A, st);
    else launch<TX, TB, 256, 8>(A, st);
}
template <int TX>
void launch_branch(const NormArgs& A, int tb, hipStream_t st)
{
    if (tb == MIXAQ_F32) launch_types<TX, MIXAQ_F32>(A, st);
    else if (tb == MIXAQ_F16) launch_types<TX, MIXAQ_F16>(A, st);
    else launch_types<TX, MIXAQ_BF16>(A, st);
}

// written in place: every value is read by the lane that writes it, and before
bool same_place(const mixaq_rows& a, const mixaq_rows& b) { return a.data == b.data && a.stride == b.stride && a.type == b.type; }

int check_norm(int kind, float eps, const char* name)
{
    if (kind < NORM_NONE || kind > NORM_RMS) return fail(MIXAQ_E_SHAPE, "%s: unknown norm %d", name, kind);
    if (kind != NORM_NONE && (!(eps > 0.0f) || !std::isfinite(eps))) return fail(MIXAQ_E_SHAPE, "%s: eps must be positive", name);
    return MIXAQ_OK;
}

}  // namespace

extern "C" int mixaq_residual_norm(const mixaq_residual_norm_desc* desc, const mixaq_residual_norm_params* params, const mixaq_rows* x,
                                   const mixaq_rows* branch, const mixaq_rows* y, const mixaq_rows* out, int32_t rows, void* stream)
{
    if (!desc) return fail(MIXAQ_E_NULL, "descriptor is NULL");
    if (!params) return fail(MIXAQ_E_NULL, "params is NULL");
    const mixaq_residual_norm_desc& d = *desc;
    if (d.C < 1 || d.C > 16384) return fail(MIXAQ_E_SHAPE, "C=%d outside 1..16384", d.C);
    if (rows < 0) return fail(MIXAQ_E_SHAPE, "rows must not be negative (got %d)", rows);
    int rc = check_norm(d.post_norm, d.post_eps, "post_norm");
    if (!rc) rc = check_norm(d.pre_norm, d.pre_eps, "pre_norm");
    if (rc) return rc;
    if (!y && !out) return fail(MIXAQ_E_NULL, "y and out are both NULL");
    if (!out && d.pre_norm) return fail(MIXAQ_E_NULL, "pre_norm without out");
    if (!branch && (d.post_norm || params->gate)) return fail(MIXAQ_E_NULL, "post_norm or gate without branch");
    if (params->gate && d.rows_per_gate < 1) return fail(MIXAQ_E_SHAPE, "rows_per_gate must be positive (got %d)", d.rows_per_gate);
    if (rows == 0) return MIXAQ_OK;
    rc = check_rows(x, "x", d.C, false, 0);
    if (!rc && branch) rc = check_rows(branch, "branch", d.C, false, 0);
    if (!rc && y) rc = check_rows(y, "y", d.C, false, 0);
    if (!rc && out) rc = check_rows(out, "out", d.C, true, rows);
    if (rc) return rc;
    if (y && y->type != x->type) return fail(MIXAQ_E_SHAPE, "y must have the type of x");
    const mixaq_rows* outputs[2] = {y, out};
    const char* names[2] = {"y", "out"};
    for (int i = 0; i < 2; ++i) {
        if (!outputs[i]) continue;
        if (!same_place(*outputs[i], *x) && rows_overlap(*outputs[i], rows, d.C, *x, rows, d.C))
            return fail(MIXAQ_E_SHAPE, "%s and x overlap", names[i]);
        if (branch && !same_place(*outputs[i], *branch) && rows_overlap(*outputs[i], rows, d.C, *branch, rows, d.C))
            return fail(MIXAQ_E_SHAPE, "%s and branch overlap", names[i]);
    }
    if (y && out && rows_overlap(*y, rows, d.C, *out, rows, d.C)) return fail(MIXAQ_E_SHAPE, "y and out overlap");

    NormArgs A = {};
    A.x = x->data; A.ldx = x->stride;
    if (branch) { A.branch = branch->data; A.ldb = branch->stride; }
    if (y) { A.y = y->data; A.ldy = y->stride; }
    if (out) { A.out = out->data; A.ldo = out->stride; A.out_type = out->type; A.scales = out->scales; A.lds = out->scale_stride; }
    A.rows = rows; A.C = d.C; A.post = d.post_norm; A.pre = d.pre_norm;
    A.rows_per_gate = std::max(d.rows_per_gate, 1);
    A.post_eps = d.post_eps; A.pre_eps = d.pre_eps; A.residual_scale = d.residual_scale;
    A.inv_C = 1.0f / (float)d.C;
    A.post_gamma = params->post_gamma; A.post_beta = params->post_beta;
    A.pre_gamma = params->pre_gamma; A.pre_beta = params->pre_beta;
    A.gate = params->gate;
    const int tb = branch ? branch->type : x->type;
    if (x->type == MIXAQ_F32) launch_branch<MIXAQ_F32>(A, tb, (hipStream_t)stream);
    else if (x->type == MIXAQ_F16) launch_branch<MIXAQ_F16>(A, tb, (hipStream_t)stream);
    else launch_branch<MIXAQ_BF16>(A, tb, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}
