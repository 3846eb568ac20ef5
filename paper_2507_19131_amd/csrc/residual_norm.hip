// y = residual_scale * x + gate * post_norm(branch), out = pre_norm(y): what stands between two layers of a residual stream, in one
// pass over x and branch.
#include "scaled.h"

#include <algorithm>
#include <cmath>

using namespace mixaq;

namespace {

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

// Sums over the G lanes of a row, of N values a lane.  With more than a wave, through LDS (`part`: a place per wave, twice, used in turn, so that one
// barrier is enough: who writes a half again has passed the barrier of the other one, behind which nobody reads it any more): a lane reads one
// wave's sums, and its neighbours add them up.
struct Sums { float v[2]; };
template <int G> using Part = Sums[G < 64 ? 1 : G / 64];
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], Part<G>* part, int& turn)
{
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __uint_as_float(G == 16 ? over16(__float_as_uint(v[n]), SumOf()) : over64(__float_as_uint(v[n]), SumOf()));
    if constexpr (G > 64) {
        Sums* const p = part[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) p[threadIdx.x >> 6].v[n] = v[n];
        }
        __syncthreads();
        const Sums& mine = p[threadIdx.x % (G / 64)];
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = __uint_as_float(over_few<G / 64>(__float_as_uint(mine.v[n]), SumOf()));
    }
}

// A vector of parameters: a lane's values of it.
template <int V> struct Vector { float v[V][8]; };
template <int G, int V, bool TINY>
__device__ __forceinline__ void load_vector(Vector<V>& to, const float* from, const Eight (&c)[V], int C, float otherwise)
{
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (from) load8f<TINY>(from, c[j], C, to.v[j]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) to.v[j][e] = otherwise;
    }
}

// One norm of a row whose values lie in registers, V times eight a lane: mean first, then the squares of what is left.  Beside the squares what is left
// is summed as well: that is what the roundings of the first sum and of 1 / C have kept out of the mean (1000 equal values of 1000 gave -0.019
// instead of 0, of -77777.7 0.93), and it comes off the mean square and the values.  So a large mean costs no digits but the values' own.  An addition a value and a
// second value in the exchange: us of two LayerNorms, without it / with it, 68208 x 96 of f32 to codes 19.2 / 19.5, of bf16 14.4 / 15.6, 17000 x 768 28.1 / 29.2,
// 8190 x 4096 58.0 / 59.6.  Sums in binary32.
template <int G, int V, bool TINY>
__device__ __forceinline__ void norm_row(float (&v)[V][8], int kind, float eps, const Vector<V>& gamma, const Vector<V>& beta, const Eight (&c)[V],
                                         const NormArgs& A, Part<G>* part, int& turn)
{
    float mean = 0.0f;
    if (kind == NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += own8<TINY>(c[j], e, A.C) ? v[j][e] : 0.0f;
        row_sums<G>(s, part, turn);
        mean = s[0] * A.inv_C;
    }
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[j][e] -= mean;
            const float o = own8<TINY>(c[j], e, A.C) ? v[j][e] : 0.0f;
            q[0] += o;
            q[1] = fmaf(o, o, q[1]);
        }
    // An RMS norm has no use for q[0], but an exchange of its own costs registers, which rows of more than a wave and of two times eight values a lane lack:
    // 2000 x 16384 95 us with it, 89 without (8190 x 4096 of RMS norms, which have them, 55 and 57).
    if (kind == NORM_LAYER || (V == 2 && G != 256)) {
        row_sums<G>(q, part, turn);
    } else {
        float only[1] = {q[1]};
        row_sums<G>(only, part, turn);
        q[1] = only[0];
    }
    const float rest = kind == NORM_LAYER ? q[0] * A.inv_C : 0.0f;
    float square = fmaf(-rest, rest, q[1] * A.inv_C);
    square = square < 0.0f ? 0.0f : square;                           // (a NaN stays one)
    const float r = 1.0f / sqrtf(square + eps), off = -rest * r;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = fmaf(fmaf(v[j][e], r, off), gamma.v[j][e], beta.v[j][e]);
}

// A workgroup's next row is on its way while this one is worked on: with about three workgroups a CU, whose rows would otherwise be
// requested, reduced and stored in turn, memory is seldom without requests (of 16-bit values three waves a SIMD are asked for, which 129 to 256 and 513 to
// 1024 columns would miss by few registers: 17000 x 768 29 us instead of 39).  KEEP: the vectors of both norms and the gate stay in registers
// from row to row; else they come anew (from the caches) for every row, where four of them would not fit beside it.
// What bounds it is memory: 8190 x 4096 of bf16 with two outputs 4.4 TB/s, a copy of that size 5.1.  Rows that start anywhere (an
// odd width) cost a third more: every vector access of a wave then touches a line more.
template <int TX, int TB, int G, int V, bool TINY>
__global__ __launch_bounds__(G < 256 ? 256 : G, G <= 256 && sizeof(typename TypeOf<TX>::T) + sizeof(typename TypeOf<TB>::T) == 4 ? 3 : 1) void residual_norm_kernel(NormArgs A)
{
    using X = typename TypeOf<TX>::T;
    using B = typename TypeOf<TB>::T;
    constexpr bool KEEP = G <= 256 || V == 1;
    constexpr int ROWS = G < 256 ? 256 / G : 1;                       // at one time
    __shared__ Part<G> part[2];
    int turn = 0;
    const int l = threadIdx.x % G;
    Eight c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = place8<TINY>((j * G + l) * 8, A.C);
    Vector<V> post_gamma, post_beta, pre_gamma, pre_beta, gate;
    auto load_post = [&] {
        load_vector<G, V, TINY>(post_gamma, A.post_gamma, c, A.C, 1.0f);
        load_vector<G, V, TINY>(post_beta, A.post_beta, c, A.C, 0.0f);
    };
    auto load_pre = [&] {
        load_vector<G, V, TINY>(pre_gamma, A.pre_gamma, c, A.C, 1.0f);
        load_vector<G, V, TINY>(pre_beta, A.pre_beta, c, A.C, 0.0f);
    };
    const long long step = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + threadIdx.x / G;
    X tx[V][8];
    B tb[V][8];
    auto request = [&](long long r) {
        const long long at = min(r, (long long)A.rows - 1);          // spare lanes take the last row along and store nothing
#pragma unroll
        for (int j = 0; j < V; ++j) load8<TINY>((const X*)A.x + at * A.ldx, c[j], A.C, tx[j]);
        if (A.branch) {
#pragma unroll
            for (int j = 0; j < V; ++j) load8<TINY>((const B*)A.branch + at * A.ldb, c[j], A.C, tb[j]);
        }
    };
    request(row);
    if (KEEP && A.post) load_post();
    if (KEEP && A.pre) load_pre();
    int gate_row = -1;
    for (long long r0 = row - threadIdx.x / G; r0 < A.rows; r0 += step, row += step) {
        const bool real = row < A.rows;
        float x[V][8], y[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[j][e] = (float)tx[j][e];
                y[j][e] = A.branch ? (float)tb[j][e] : 0.0f;
            }
        // (of rows written in place too: another turn's row is another row, and what spare lanes read nobody uses)
        if (r0 + step < A.rows) request(row + step);
        if (A.gate) {
            const int g = (int)min(row, (long long)A.rows - 1) / A.rows_per_gate;
            if (!KEEP || g != gate_row) load_vector<G, V, TINY>(gate, A.gate + (long long)g * A.C, c, A.C, 1.0f);
            gate_row = g;
        }
        if (A.post) {
            if (!KEEP) load_post();
            norm_row<G, V, TINY>(y, A.post, A.post_eps, post_gamma, post_beta, c, A, part, turn);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (A.gate) y[j][e] *= gate.v[j][e];
                y[j][e] = A.branch ? fmaf(A.residual_scale, x[j][e], y[j][e]) : A.residual_scale * x[j][e];
            }
            if (A.y && real) store8<TINY>((X*)A.y + row * A.ldy, c[j], A.C, y[j]);
        }
        if (!A.out) continue;
        if (A.pre) {
            if (!KEEP) load_pre();
            norm_row<G, V, TINY>(y, A.pre, A.pre_eps, pre_gamma, pre_beta, c, A, part, turn);
        }
        if (A.out_type == MIXAQ_E4M3) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const BlockScale s = block_scale(max16(max_magnitude<TINY>(c[j], A.C, y[j])));
                const int col = (j * G + l) * 8;
                if (real && col < A.C) {
                    store_codes8<TINY>((uint8_t*)A.out + row * A.ldo, c[j], A.C, y[j], s.inv);
                    if ((l & 15) == 0) A.scales[(long long)(col / SBLOCK) * A.lds + row] = s.scale;
                }
            }
        } else if (real) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (A.out_type == MIXAQ_F32) store8<TINY>((float*)A.out + row * A.ldo, c[j], A.C, y[j]);
                else if (A.out_type == MIXAQ_F16) store8<TINY>((_Float16*)A.out + row * A.ldo, c[j], A.C, y[j]);
                else store8<TINY>((__bf16*)A.out + row * A.ldo, c[j], A.C, y[j]);
            }
        }
    }
}

template <int TX, int TB, int G, int V, bool TINY = false>
void launch(const NormArgs& A, hipStream_t st)
{
    // Three workgroups a CU, each on every 768th group of rows: neighbouring rows are on their way at one time.  8190 x 4096 values of bf16 with
    // gates, us: 512 workgroups 68, 768 61, 1024 73, 2048 67, 4096 71; a run of neighbouring rows for each of 1024 73.  Up to 64 values, which are few
    // bytes a turn, 2048: 200000 x 64 38 instead of 43, 260000 x 128 68 instead of 60.
    constexpr int ROWS = G < 256 ? 256 / G : 1;
    const long long groups = ((long long)A.rows + ROWS - 1) / ROWS;
    hipLaunchKernelGGL((residual_norm_kernel<TX, TB, G, V, TINY>), dim3((unsigned)std::min(groups, A.C <= 64 ? 2048LL : 768LL)), dim3(G < 256 ? 256 : G), 0, st, A);
}
// The lanes of a row: 16, a wave, then a workgroup of four or sixteen, with one or two times eight values each.  (us, bf16, with gates:  C = 256
// in 16 lanes of two 60, in 64 of one 88;  1024 in 64 of two 61, in 256 of one 105;  4096 in 256 of two 60, in 512 of one 71;  8192 in 512 of
// two 92, in 1024 of one, which can keep the vectors, 82.)
template <int TX, int TB>
void launch_types(const NormArgs& A, hipStream_t st)
{
    if (A.C < 8) launch<TX, TB, 16, 1, true>(A, st);
    else if (A.C <= 128) launch<TX, TB, 16, 1>(A, st);
    else if (A.C <= 256) launch<TX, TB, 16, 2>(A, st);
    else if (A.C <= 512) launch<TX, TB, 64, 1>(A, st);
    else if (A.C <= 1024) launch<TX, TB, 64, 2>(A, st);
    else if (A.C <= 2048) launch<TX, TB, 256, 1>(A, st);
    else if (A.C <= 4096) launch<TX, TB, 256, 2>(A, st);
    else if (A.C <= 8192) launch<TX, TB, 1024, 1>(A, st);
    else launch<TX, TB, 1024, 2>(A, st);
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
    if (rows < 0 || rows > MOST_ROWS) return fail(MIXAQ_E_SHAPE, "need 0 <= rows <= 2^30 (got %d)", rows);
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
        const Extent o = extent_of(*outputs[i], rows, d.C), os = scales_of(*outputs[i], rows, d.C);
        for (const mixaq_rows* in : {x, branch}) {
            if (!in) continue;
            const Extent e = extent_of(*in, rows, d.C);
            if ((!same_place(*outputs[i], *in) && overlap(o, e)) || overlap(os, e)) return fail(MIXAQ_E_SHAPE, "%s and %s overlap", names[i], in == x ? "x" : "branch");
        }
        const float* const vectors[5] = {params->post_gamma, params->post_beta, params->pre_gamma, params->pre_beta, params->gate};
        const char* const of[5] = {"post_gamma", "post_beta", "pre_gamma", "pre_beta", "gate"};
        for (int v = 0; v < 5; ++v) {
            const long long count = v < 4 ? 1 : (rows - 1LL) / std::max(d.rows_per_gate, 1) + 1;
            const Extent e = {(uintptr_t)vectors[v], d.C * 4LL, vectors[v] ? count : 0, d.C * 4LL};
            if (overlap(o, e) || overlap(os, e)) return fail(MIXAQ_E_SHAPE, "%s and %s overlap", names[i], of[v]);
        }
        if (overlap(o, os)) return fail(MIXAQ_E_SHAPE, "codes and scales of %s overlap", names[i]);
    }
    if (y && out && (overlap(extent_of(*y, rows, d.C), extent_of(*out, rows, d.C)) || overlap(extent_of(*y, rows, d.C), scales_of(*out, rows, d.C))))
        return fail(MIXAQ_E_SHAPE, "y and out overlap");

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
