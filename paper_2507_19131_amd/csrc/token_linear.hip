// Linear layers on int8 codes with a scale per token and channel: y = act(x w^T + bias), the products on the int8 matrix instructions of gfx950,
// the sums exact; for one matrix, or for rows sorted by expert and a matrix for each.
#include "token.h"
#include "token_forms.h"

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
    bool aligned;                     // rows of y start at multiples of 16 bytes
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
// x may be given as values (8 .. INSIDE_K a row): the workgroup quantizes its 16 rows into LDS first, 32 lanes a row, a row in registers between its maximum
// and its codes.  SORTED: a workgroup takes all rows of its expert, one tile after the other, so that weights come once.  Weights, rows, scales and bias are asked
// for as soon as their places are known.
// What bounds it: a launch and round trips to memory (1 x 1024 x 4096 from codes 3.1 us of a graph replay, 4.2 MB of weights would take 0.8; from values 4.3; 16 rows of
// 32 experts, 2048 x 1024 each, 5.6 us where the 27 MB of the experts they hit take 5.4; from values 7.7: a row comes after its offsets and its place in the list,
// and the weights behind it, in whose place they would be waited for first), with more rows the operands' way through the caches, each workgroup
// for itself (256 x 1024 x 1024 in 32 x 32 4.2 us, 1024 x 4096 x 1024 in 64 x 64 14.7).
constexpr int INSIDE_K = 1024;                    // the most inputs of values that are quantized here

template <int XT, int YT, int MR, int NR, int NW, bool SORTED>
__global__ __launch_bounds__(NW * 64, MR == 1 ? 4 : 1) void token_few_kernel(TokenArgs A, int per, FastDiv by_per, int groups)
{
    constexpr int FR = MR * NR;                                              // 16 x 16 results of the workgroup
    constexpr bool FROM_CODES = XT == MIXAQ_I8;
    using X = typename std::conditional<FROM_CODES, TypeOf<MIXAQ_E4M3>, TypeOf<XT>>::type::T;
    __shared__ v4i part[NW][FR][64];
    constexpr int CODED = FROM_CODES ? 16 : INSIDE_K + 16;                   // bytes of a row of codes: 16 lanes of a chunk in different banks
    __shared__ v4i coded[16][CODED / 16];
    static_assert(FROM_CODES || (MR == 1 && NW * 64 == 16 * 32 && NW * SBLOCK >= INSIDE_K), "16 rows, a block of K for each wave");
    __shared__ float scale_of[16 * MR];
    __shared__ int source[16 * MR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // a run of workgroups per XCD, the row tiles of one run of weights beside one another; of rows sorted by expert every XCD has a share of each expert, of
    // which some may have no rows
    const int per_xcd = (groups + 7) / 8, t = SORTED ? (int)blockIdx.x : (int)((blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3));
    if ((!SORTED && (int)(blockIdx.x >> 3) >= per_xcd) || t >= groups) return;           // the whole workgroup
    const int q = by_per(t), in = t - q * per, nt = SORTED ? in : q, nb = nt * NR / 8, tile0 = nt * NR % 8;
    if (nb * SBLOCK + output_of(tile0, 0) >= A.N) return;                    // (the tiles of the last block may all lie beyond)
    int first = in * 16 * MR, end = A.M;
    if (SORTED) rows_of(A, q, first, end);
    const long long layer = SORTED ? (long long)q * A.NB : 0;                // blocks of 128 outputs before this expert's
    const v4i* const w0 = (const v4i*)(A.w + ((layer + nb) * A.KB * 8 + tile0) * TILE_BYTES) + lane;
    constexpr int MINE = (FR + NW - 1) / NW;                                 // results that a wave sums and finishes
    v4f sw[MINE], bias[MINE];
    if (!SORTED || first < end) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const long long n0 = (layer + nb) * SBLOCK + output_of(tile0 + min(wave + i * NW, FR - 1) % NR, 4 * g);
            __builtin_memcpy(&sw[i], A.sw + n0, 16);
            __builtin_memcpy(&bias[i], A.bias + n0, 16);
        }
    }
    struct Operands { v4i w[NR][2], x[MR][2]; };
    for (int r0 = first; r0 < (SORTED ? end : first + 1); r0 += 16 * MR) {
        auto load_w = [&](int kb, Operands& o) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                o.w[n][0] = w0[(kb * 8 + n) * 128];
                o.w[n][1] = w0[(kb * 8 + n) * 128 + 64];
            }
        };
        Operands now;
        const bool works = wave < A.KB;
        if (FROM_CODES && works) load_w(wave, now);                          // on their way while the rows are looked up
        const X* from[MR];
        auto load_x = [&](int kb, Operands& o) {                             // (behind a row's end the row's first codes: the weights there are zero)
            const int k0 = kb * SBLOCK + g * 16;
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                o.x[m][0] = *(const v4i*)(from[m] + (k0 < A.K ? k0 : 0));
                o.x[m][1] = *(const v4i*)(from[m] + (k0 + 64 < A.K ? k0 + 64 : 0));
            }
        };
        if constexpr (FROM_CODES) {
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                const int r = r0 + m * 16 + c, at = min(r, end - 1), src = SORTED ? source_of(A, at) : at;
                from[m] = (const X*)A.x + (long long)max(src, 0) * A.ldx;
                if (wave == 0 && g == 0) {
                    scale_of[m * 16 + c] = A.sx[max(src, 0)];
                    source[m * 16 + c] = r < end ? src : -1;
                }
            }
            if (works) load_x(wave, now);
        } else {
            const int row = threadIdx.x >> 5, l = threadIdx.x & 31, r = r0 + row, at = min(r, end - 1), src = SORTED ? source_of(A, at) : at;
            const X* const values = (const X*)A.x + (long long)max(src, 0) * A.ldx;
            Eight place[INSIDE_K / 256];
            float v[INSIDE_K / 256][8];
            unsigned largest = 0;
#pragma unroll
            for (int j = 0; j < INSIDE_K / 256; ++j) {
                place[j] = place8<false>((j * 32 + l) * 8, A.K);
                load8f<false>(values, place[j], A.K, v[j]);
            }
            if (works) load_w(wave, now);                                    // (behind the values: loads come back in order)
#pragma unroll
            for (int j = 0; j < INSIDE_K / 256; ++j) largest = max(largest, max_magnitude<false>(place[j], A.K, v[j]));
            largest = max16(largest);
            const RowScale s = row_scale(max(largest, (unsigned)__shfl_xor((int)largest, 16, 64)));
#pragma unroll
            for (int j = 0; j < INSIDE_K / 256; ++j) store_int_codes8<false>((int8_t*)coded[row], place[j], A.K, v[j], s.inv);
            if (l == 0) {
                scale_of[row] = s.scale;
                source[row] = r < end ? src : -1;
            }
            __syncthreads();
            if (works) {                                                     // (what stands behind a row's end: the weights there are zero)
                now.x[0][0] = coded[c][wave * 8 + g];
                now.x[0][1] = coded[c][wave * 8 + g + 4];
            }
        }
        v4i acc[MR][NR] = {};
        auto multiply = [&](const Operands& o) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int m = 0; m < MR; ++m) {
                    acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o.w[n][0], o.x[m][0], acc[m][n], 0, 0, 0);
                    acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o.w[n][1], o.x[m][1], acc[m][n], 0, 0, 0);
                }
        };
        if (works) {                                                         // one block's operands travel under the products of the last one
            for (int kb = wave + NW; FROM_CODES && kb < A.KB; kb += NW) {
                Operands next;
                load_w(kb, next);
                load_x(kb, next);
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
        using T = typename TypeOf<YT>::T;
        const int used = min(NW, A.KB);
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int f = wave + i * NW;
            if (f >= FR) break;
            v4i sum = part[0][f][lane];
            for (int w = 1; w < used; ++w) sum += part[w][f][lane];
            const int own = f / NR * 16 + c, r = r0 + own, n0 = nb * SBLOCK + output_of(tile0 + f % NR, 4 * g);
            const float sx = scale_of[own];
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf((float)sum[e], sx * sw[i][e], bias[i][e]);
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

// ---- both operands through LDS ------------------------------------------------------------------------------------------
// A workgroup of four waves computes 128 rows times 128 outputs, a wave 32 rows times the outputs.  K goes in stages of 64 through a
// ring of four LDS buffers filled by direct loads, three stages ahead of the products.  For products whose tiles are few or whose stages are: 4704 x 384 x 1536 with a
// GELU 11.6 us (444 tiles, two a CU, of six stages: the first loads, the GELU, 14 MB of results), 4704 x 1536 x 384 11.7 (111 tiles: a stage takes 0.35 us, a
// round trip, however little there is to multiply).
// Rows of x lie in LDS as 4 chunks of 16 bytes whose places are turned by a fourth of the row's number, so that the 16 lanes that are served
// together (16 rows, one chunk) meet all 64 banks.
// The direct loads are asm: as a builtin every LDS read behind them waits for all of them.  They do nothing for stages from `end` on, which the asm finds out: a
// branch around it would be one in the middle of a stage.
// Two pieces one behind the other in LDS.
__device__ __forceinline__ void request2(const uint8_t* uniform_src, unsigned first, unsigned second, unsigned lds_dst, int stage, int end)
{
    int m0;                                                                  // given back: the compiler does not let an asm statement change it
    asm volatile("s_cmp_ge_i32 %5, %6\n\ts_cbranch_scc1 .Lskip%=\n\ts_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0\n.Lskip%=:"
                 : "=&s"(m0) : "v"(first), "v"(second), "s"(uniform_src), "s"(lds_dst), "s"(stage), "s"(end) : "memory", "scc");
}
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(size_t)(const __attribute__((address_space(3))) char*)p; }

// Of instructions of 32 x 32 x 32 the packed tiles 2 T and 2 T + 1 are rows 0 .. 31 of the T-th, lane half h takes the 16-byte chunk 2 c + h of a row's 128 bytes in
// step c.  Result e is row 8 (e / 4) + 4 h + e % 4: of the outputs, by output_of, number 4 (2 (T % 2) + e / 8) + e % 4 of
// run 2 (e / 4 % 2) + h of 16, in half T / 2 of the block.
__device__ __forceinline__ int run_of(int i, int h) { return (i >> 1) * 64 + (2 * (i & 1) + h) * 16; }
// of number q of run i (0 .. 3: the two of a half, then the other half's): which T, which result
__device__ __forceinline__ constexpr int tile_of_run(int i, int q) { return (i >> 1) * 2 + (q >> 3); }
__device__ __forceinline__ constexpr int result_of_run(int i, int q) { return (q >> 2 & 1) * 8 + (i & 1) * 4 + (q & 3); }

// Inclusive sums over the lanes of a wave, in the vector unit: within rows of 16, then the last lane of a row to the next one's, of the first half to the second.
template <int CTRL, int ROWS> __device__ __forceinline__ int from_before(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int scan64(int v)
{
    v += from_before<0x111, 0xf>(v);
    v += from_before<0x112, 0xf>(v);
    v += from_before<0x114, 0xf>(v);
    v += from_before<0x118, 0xf>(v);
    v += from_before<0x142, 0xa>(v);
    return v + from_before<0x143, 0xc>(v);
}
// Row tiles of TM rows, expert after expert: how many there are in all, and of the t-th its expert and its rows.  By every wave for itself.
template <int TM>
struct SortedTiles {
    int total = 0, kept = 0;                                                 // kept: of the last 64 experts looked at
    __device__ int tiles(const TokenArgs& A, int e)
    {
        if (e >= A.experts) return 0;
        int first, end;
        rows_of(A, e, first, end);
        return (end - first + TM - 1) / TM;
    }
    __device__ void count(const TokenArgs& A, int most)                      // at most `most`, whatever the offsets
    {
        for (int e0 = 0; e0 < A.experts; e0 += 64) {
            kept = scan64(tiles(A, e0 + (threadIdx.x & 63)));
            total = min(total + __builtin_amdgcn_readlane(kept, 63), most);
        }
    }
    __device__ void find(const TokenArgs& A, int t, int& e, int& first, int& end)
    {
        int before = 0;
        first = end = 0;
        for (int e0 = 0; e0 < A.experts; e0 += 64) {                         // (t < total: some expert has it)
            if (A.experts > 64) kept = scan64(tiles(A, e0 + (threadIdx.x & 63)));
            const unsigned long long behind = __ballot(before + kept > t);
            if (behind) {
                const int l = __ffsll((long long)behind) - 1;
                e = __builtin_amdgcn_readfirstlane(e0 + l);
                const int skipped = before + (l ? __builtin_amdgcn_readlane(kept, l - 1) : 0);
                rows_of(A, e, first, end);
                first += (t - skipped) * TM;
                end = min(end, first + TM);
                return;
            }
            before += __builtin_amdgcn_readlane(kept, 63);
        }
    }
};

constexpr int GROUP_M = 4;                        // row tiles that run beside one another

// The tile of this workgroup: TM rows from `first` to before `end`, of an expert, and its outputs' place tn; false where there is none.  A run of tiles
// per XCD, so that what its CUs read at one time meets in its L2: in groups of GROUP_M row tiles with all their outputs, or row tile by row tile.
template <int TM, bool SORTED>
__device__ __forceinline__ bool tile_of(const TokenArgs& A, int tiles_m, int tiles_n, FastDiv by, int& tn, int& first, int& end, int& expert)
{
    SortedTiles<TM> sorted;
    if (SORTED) sorted.count(A, tiles_m);
    const int tiles = (SORTED ? sorted.total : tiles_m) * tiles_n, per_xcd = (tiles + 7) / 8;
    const int t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || t >= tiles) return false;
    expert = 0;
    if (SORTED) {
        const int rt = by(t);
        tn = t - rt * tiles_n;
        sorted.find(A, rt, expert, first, end);
    } else {
        const int group = by(t), in = t - group * GROUP_M * tiles_n, gm = min(GROUP_M, tiles_m - group * GROUP_M);
        tn = in / gm;
        first = (group * GROUP_M + in - tn * gm) * TM;
        end = min(A.M, first + TM);
    }
    return true;
}

// The sums of a wave's 32 MT rows from row0 on and of its 64 H outputs from n0 on, to results.  A lane holds those of one row in every 32, in 2 H runs of 16 neighbouring
// ones, the lanes l and l + 32 the whole row.  Through LDS (`turn`: 32 rows x 256 bytes of the wave's own, of which 64 outputs of 16 bits take half), so that a
// store covers whole lines; its 16-byte pieces are turned by the row, so that neither side meets a bank twice.  Whole pieces go past the caches, which x and the
// weights are in (4704 x 384 x 1536 with a GELU 13.3 us -> 11.6, with the layers before and after it 36.8 -> 35.0).
template <int YT, int MT, int H, bool SORTED>
__device__ __forceinline__ void finish(const TokenArgs& A, const v16i (&acc)[MT][2 * H], int expert, int n0, int row0, int end, v4i* turn)
{
    using T = typename TypeOf<YT>::T;
    constexpr int ES = sizeof(T), ROW_BYTES = 64 * H * ES < 256 ? 64 * H * ES : 256, PASSES = 64 * H * ES / ROW_BYTES, PIECES = ROW_BYTES / 16, RUNS = 2 * H / PASSES;
    const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
    const long long layer = (long long)expert * A.NB * SBLOCK + n0;
    float s[2 * H][16], b[2 * H][16];
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) {
        __builtin_memcpy(s[i], A.sw + layer + run_of(i, h), 64);
        __builtin_memcpy(b[i], A.bias + layer + run_of(i, h), 64);
    }
    auto place = [](int r, int p) { return r * PIECES + (PIECES == 16 ? p ^ (r & 15) : p ^ (r >> 1 & 7)); };
    auto in_order = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };           // among the lanes of the wave, which runs in step
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r0 = row0 + m * 32, at = min(r0 + j, end - 1), src = SORTED ? source_of(A, at) : at;
        const float sx = A.sx[max(src, 0)], weight = SORTED && A.weights ? A.weights[at] : 1.0f;
        const unsigned kept = (unsigned)__ballot(r0 + j < end && src >= 0);              // a bit for each row that is stored
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
#pragma unroll
            for (int i = pass * RUNS; i < (pass + 1) * RUNS; ++i) {
                float v[16];
                T t[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = fmaf((float)acc[m][tile_of_run(i, e)][result_of_run(i, e)], sx * s[i][e], b[i][e]);
                activate(v, A.act);
#pragma unroll
                for (int e = 0; e < 16; ++e) t[e] = (T)(SORTED ? weight * v[e] : v[e]);
                const int p = run_of(i, h) * ES % ROW_BYTES / 16;
#pragma unroll
                for (int q = 0; q < ES; ++q) __builtin_memcpy(&turn[place(j, p + q)], (const uint8_t*)t + q * 16, 16);
            }
            in_order();
#pragma unroll
            for (int k = 0; k < PIECES / 2; ++k) {
                const int r = (k * 64 + lane) / PIECES, p = lane % PIECES, n = n0 + (pass * ROW_BYTES + p * 16) / ES;
                const v4i piece = turn[place(r, p)];
                if (!(kept >> r & 1)) continue;
                T* const to = (T*)A.y + (long long)(r0 + r) * A.ldy + n;
                if (A.aligned && n + 16 / ES <= A.N) __builtin_nontemporal_store(piece, (v4i*)to);
                else if (n + 16 / ES <= A.N) __builtin_memcpy(to, &piece, 16);
                else {
                    T u[16 / ES];
                    __builtin_memcpy(u, &piece, 16);
#pragma unroll
                    for (int e = 0; e < 16 / ES; ++e)
                        if (n + e < A.N) to[e] = u[e];
                }
            }
            in_order();
        }
    }
}

// Waits until of the stages that this wave has requested, R loads each, at most min(CAP, left) are on their way.
template <int R, int CAP>
__device__ __forceinline__ void wait_stages(int left)
{
    static_assert(CAP == 2 || CAP == 3, "");
    if constexpr (CAP == 3)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_cmp_lt_i32 %0, 1\n\ts_cbranch_scc1 .Lnone%=\n\ts_cmp_lt_i32 %0, 2\n\ts_cbranch_scc1 .Lone%=\n\ts_cmp_lt_i32 %0, 3\n\t"
                     "s_cbranch_scc1 .Ltwo%=\n\ts_waitcnt vmcnt(%3)\n\ts_branch .Ldone%=\n.Ltwo%=:\n\ts_waitcnt vmcnt(%2)\n\ts_branch .Ldone%=\n.Lone%=:\n\t"
                     "s_waitcnt vmcnt(%1)\n\ts_branch .Ldone%=\n.Lnone%=:\n\ts_waitcnt vmcnt(0)\n.Ldone%=:" :: "s"(left), "n"(R), "n"(2 * R), "n"(3 * R) : "memory", "scc");
    else
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_cmp_lt_i32 %0, 1\n\ts_cbranch_scc1 .Lnone%=\n\ts_cmp_lt_i32 %0, 2\n\ts_cbranch_scc1 .Lone%=\n\ts_waitcnt vmcnt(%2)\n\t"
                     "s_branch .Ldone%=\n.Lone%=:\n\ts_waitcnt vmcnt(%1)\n\ts_branch .Ldone%=\n.Lnone%=:\n\ts_waitcnt vmcnt(0)\n.Ldone%=:"
                     :: "s"(left), "n"(R), "n"(2 * R) : "memory", "scc");
}

constexpr int DEPTH = 64, RING = 4;               // bytes of K in a stage, stages in LDS

template <int YT, bool SORTED>
__global__ __launch_bounds__(256, 2) void token_tile_kernel(TokenArgs A, int tiles_m, int tiles_n, FastDiv by)
{
    constexpr int TM = 128, PIECES = 8, OWN = 2, R = 2 * OWN;                // 1 KB pieces of a stage, of x and as many of w, and a wave's
    __shared__ v4i xs[RING][PIECES * 64], ws[RING][PIECES * 64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, h = lane >> 5;
    const int KB = A.KB, stages = (A.K + DEPTH - 1) / DEPTH;
    int nb, first, end, expert;
    if (!tile_of<TM, SORTED>(A, tiles_m, tiles_n, by, nb, first, end, expert)) return;       // the whole workgroup

    // what this wave requests: rows (2 wave + i) 16 + lane / 4 of x, whose lanes take the chunk that belongs in their place, and pieces 2 wave + i of w
    const int chunk = ((lane & 3) ^ (lane >> 4)) * 16, last_chunk = (A.K - 1) & ~15;      // (what stands behind a row's end is the last chunk again, the weights there are zero)
    const uint8_t* const xb = (const uint8_t*)A.x + (SORTED ? 0 : (long long)first * A.ldx);
    unsigned from[OWN], piece[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int r = min(first + (wave * OWN + i) * 16 + (lane >> 2), end - 1);
        from[i] = (unsigned)(SORTED ? max(source_of(A, r), 0) : r - first) * (unsigned)A.ldx;
        piece[i] = i * TILE_BYTES + lane * 16;
    }
    const uint8_t* const wb = A.w + ((long long)expert * A.NB + nb) * KB * (8 * TILE_BYTES) + wave * OWN * TILE_BYTES;
    const unsigned lx = lds_address(xs), lw = lds_address(ws);
    const unsigned own = wave * OWN * 1024;
    auto request_x = [&](int ks) {
        const unsigned k = min(ks * DEPTH + chunk, last_chunk);
        request2(xb, from[0] + k, from[1] + k, lx + ks % RING * (PIECES * 1024) + own, ks, stages);
    };
    auto request_w = [&](int ks) {
        request2(wb + (long long)(ks >> 1) * (8 * TILE_BYTES) + (ks & 1) * 1024, piece[0], piece[1], lw + ks % RING * (PIECES * 1024) + own, ks, stages);
    };
    auto meet = [] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll
    for (int ks = 0; ks < RING; ++ks) {
        request_x(ks);
        request_w(ks);
    }
    const int m0 = wave * 32;
    v16i acc[1][4] = {};
    v4i x[2], w[2][4];
    const v4i* const xr[2] = {&xs[0][(m0 + j) * 4 + (h ^ (j >> 2 & 3))], &xs[0][(m0 + j) * 4 + (h ^ 2 ^ (j >> 2 & 3))]};
    const v4i* const wr = &ws[0][(j >> 4) * 64 + h * 16 + (j & 15)];
    auto read_x = [&](int ks, int c) { x[c] = xr[c][ks % RING * (PIECES * 64)]; };
    auto read_w = [&](int ks, int c, int T) { w[c][T] = wr[ks % RING * (PIECES * 64) + T * 128 + c * 32]; };
    wait_stages<R, 3>(stages - 1);
    meet();
    read_x(0, 0);
#pragma unroll
    for (int T = 0; T < 4; ++T) read_w(0, 0, T);
    // Of each stage two steps of 32.  What a step's products need is read under those of the step before; behind the last read of a stage the waves
    // meet, and its buffer is requested anew.  The last stage reads on like the others, for nobody.
#pragma unroll 1
    for (int ks = 0; ks < stages; ++ks) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (c == 1) {
                wait_stages<R, 2>(stages - 2 - ks);
                meet();
            }
            const int next = c == 1 ? ks + 1 : ks;
#pragma unroll
            for (int T = 0; T < 4; ++T) {
                __builtin_amdgcn_sched_barrier(0);
                acc[0][T] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[c][T], x[c], acc[0][T], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (T == 0) {
                    read_x(next, c ^ 1);
                    read_w(next, c ^ 1, 0);
                    if (c == 1) request_x(ks + RING);
                } else if (T == 1) {
                    read_w(next, c ^ 1, 1);
                    read_w(next, c ^ 1, 2);
                } else if (T == 2) {
                    read_w(next, c ^ 1, 3);
                    if (c == 1) request_w(ks + RING);
                }
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");              // (and the last reads for nobody)
    meet();
    static_assert(RING * PIECES * 64 >= 4 * 512, "room for a wave's 32 rows of 256 bytes");
    finish<YT, 1, 2, SORTED>(A, acc, expert, nb * SBLOCK, first + m0, end, &xs[0][0] + wave * 512);
}

// ---- weights straight from memory, x through LDS ------------------------------------------------------------------------------
// Four waves side by side, all 128 rows and 64 outputs each.  Packed weights lie as the instruction takes them, so a wave loads its own into registers, four
// steps ahead, and no weight comes twice; x goes through two LDS buffers of 128.  With both operands in LDS its reads and the direct loads' writes took as long as the
// products: 16384 x 4096 x 3840 261 us in 256 x 256 by two times two waves, 254 with the weights in registers, 239 so, where a second workgroup on the CU runs beside
// a tile's start and end (a library product 278; 8192^3 470, 458, 463, library 453).  What bounds it: the matrix instructions are busy in 59 % of the clocks, and
// the clock is 1.65 to 1.75 GHz under this load; of 32768 rows of 64 experts x 2048 x 1024 (97 us, unsorted 72) a third as well, 1150 tiles in rounds of 512, which end
// unevenly.
template <int YT, bool SORTED>
__global__ __launch_bounds__(256, 2) void token_wide_kernel(TokenArgs A, int tiles_m, int tiles_n, FastDiv by)
{
    constexpr int MT = 4, TM = 32 * MT, XP = TM / 8, XL = XP / 4;                    // 1 KB pieces of a stage, a wave's
    __shared__ v4i xs[2][XP * 64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, h = lane >> 5, KB = A.KB;
    int tn, first, end, expert;
    if (!tile_of<TM, SORTED>(A, tiles_m, tiles_n, by, tn, first, end, expert)) return;       // the whole workgroup
    const int n0 = tn * 256 + wave * 64, nb = min(n0 / SBLOCK, A.NB - 1);    // (a wave without outputs computes others' and stores none)

    // rows (wave XL + i) 8 + lane / 8 of x, whose lanes take the chunk that belongs in their place
    const int chunk[2] = {((lane & 7) ^ (lane >> 4)) * 16, ((lane & 7) ^ (lane >> 4) ^ 4) * 16}, last_chunk = (A.K - 1) & ~15;      // of even and of odd pieces
    const uint8_t* const xb = (const uint8_t*)A.x + (SORTED ? 0 : (long long)first * A.ldx);
    unsigned from[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = min(first + (wave * XL + i) * 8 + (lane >> 3), end - 1);
        from[i] = (unsigned)(SORTED ? max(source_of(A, r), 0) : r - first) * (unsigned)A.ldx;
    }
    const unsigned lx = lds_address(xs);
    auto request = [&](int kb, int i) {                                      // two pieces; behind a row's end the last chunk again, the weights there are zero
        request2(xb, from[i] + min(kb * SBLOCK + chunk[0], last_chunk), from[i + 1] + min(kb * SBLOCK + chunk[1], last_chunk),
                 lx + ((kb & 1) * XP + wave * XL + i) * 1024, kb, KB);
    };
    auto meet = [] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const v4i* const wb = (const v4i*)(A.w + (((long long)expert * A.NB + nb) * KB * 8 + (n0 % SBLOCK ? 4 : 0)) * TILE_BYTES) + (j >> 4) * 128 + h * 16 + (j & 15);
    v16i acc[MT][2] = {};
    v4i x[2][MT], w[4][2];
    auto load = [&](int kb, int c, int T) { w[c][T] = wb[(long long)min(kb, KB - 1) * 1024 + T * 256 + (c >> 1) * 64 + (c & 1) * 32]; };
    const v4i* const xr = &xs[0][j * 8];
    auto read = [&](int kb, int c, int i) { x[c & 1][i] = xr[(kb & 1) * (XP * 64) + i * 256 + ((2 * c + h) ^ (j >> 1 & 7))]; };
#pragma unroll
    for (int i = 0; i < XL; i += 2) request(0, i);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int T = 0; T < 2; ++T) load(0, c, T);
#pragma unroll
    for (int i = 0; i < XL; i += 2) request(1, i);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    meet();
#pragma unroll
    for (int i = 0; i < MT; ++i) read(0, 0, i);
    // Of each stage four steps of 32.  What a step's products need of x is read under those of the step before; behind the last read of a stage the waves
    // meet, and its buffer is requested anew.  The last stage reads on like the others, for nobody.
#pragma unroll 1
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c == 3) {                                                    // behind the last requests there are this stage's six loads of weights
                asm volatile("s_waitcnt lgkmcnt(0) vmcnt(6)" ::: "memory");
                meet();
            }
#pragma unroll
            for (int p = 0; p < 2 * MT; ++p) {
                const int T = p / MT, m = p % MT;
                __builtin_amdgcn_sched_barrier(0);
                acc[m][T] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[c][T], x[c & 1][m], acc[m][T], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (m == MT - 1) load(kb + 1, c, T);
                if (p < MT) read(c == 3 ? kb + 1 : kb, (c + 1) & 3, p);
                if (c == 3 && p % 2 == 1 && p < XL) request(kb + 2, p - 1);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");              // (and the last reads for nobody)
    meet();
    if (n0 >= A.N) return;
    finish<YT, MT, 1, SORTED>(A, acc, expert, n0, first, end, &xs[0][0] + wave * 512);
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

template <int YT, int TM, int TN, bool SORTED>
int launch_tiles(const TokenArgs& A, const mixaq_rows* values, hipStream_t st)
{
    const int tiles_n = (A.NB + TN / SBLOCK - 1) / (TN / SBLOCK);
    const long long tiles_m = ((long long)A.M + TM - 1) / TM + (SORTED ? std::min(A.experts, A.M) : 0);      // (every expert's last tile may be cut)
    const long long blocks = (tiles_m * tiles_n + 7) / 8 * 8;
    if (blocks * 256 >= MOST_THREADS) return fail(MIXAQ_E_SHAPE, "%d rows of %d outputs are too many for one call", A.M, A.N);
    const int rc = quantize_first(A, values, st);
    if (rc) return rc;
    const FastDiv by(SORTED ? tiles_n : GROUP_M * tiles_n);
    if constexpr (TN == 256) hipLaunchKernelGGL((token_wide_kernel<YT, SORTED>), dim3((unsigned)blocks), dim3(256), 0, st, A, (int)tiles_m, tiles_n, by);
    else hipLaunchKernelGGL((token_tile_kernel<YT, SORTED>), dim3((unsigned)blocks), dim3(256), 0, st, A, (int)tiles_m, tiles_n, by);
    HIP_TRY(hipGetLastError());
    return MIXAQ_OK;
}

template <int YT, bool SORTED>
int launch_linear(const TokenArgs& A, TokenForm form, int x_type, const mixaq_rows* values, hipStream_t st)
{
    switch (form) {
    case TOKEN_TILE: return launch_tiles<YT, 128, 128, SORTED>(A, values, st);
    case TOKEN_WIDE: return launch_tiles<YT, 128, 256, SORTED>(A, values, st);
    case TOKEN_MID:
        if constexpr (!SORTED) return launch_few<MIXAQ_I8, YT, 2, 2, 8, SORTED>(A, values, st);
    case TOKEN_SPLIT: return launch_few<MIXAQ_I8, YT, 4, 4, 4, SORTED>(A, values, st);
    case TOKEN_FEW: break;
    }
    constexpr int NR = SORTED ? 4 : 1;                                       // of values
    if (x_type == MIXAQ_F32) return launch_few<MIXAQ_F32, YT, 1, NR, 8, SORTED>(A, nullptr, st);
    if (x_type == MIXAQ_F16) return launch_few<MIXAQ_F16, YT, 1, NR, 8, SORTED>(A, nullptr, st);
    if (x_type == MIXAQ_BF16) return launch_few<MIXAQ_BF16, YT, 1, NR, 8, SORTED>(A, nullptr, st);
    // 16 outputs a workgroup, or 64 where those would be more than run at one time
    if ((SORTED ? A.experts : (A.M + 15LL) / 16) * A.NB * 8 > 1024) return launch_few<MIXAQ_I8, YT, 1, 4, 8, SORTED>(A, values, st);
    return launch_few<MIXAQ_I8, YT, 1, 1, 8, SORTED>(A, values, st);
}

// the workspace: codes and scales of x, where it is given as values
size_t workspace_of(const mixaq_token_linear* h, int32_t x_rows, int32_t x_type)
{
    if (x_type == MIXAQ_I8 || x_rows == 0) return 0;
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
    const size_t need = token_quantized_inside(rows, K, h->NB, h->d.experts, sorted != nullptr) ? 0 : workspace_of(h, x_rows, x->type);
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
    A.aligned = (uintptr_t)y->data % 16 == 0 && y->stride * size_of(y->type) % 16 == 0;
    A.M = rows; A.x_rows = x_rows; A.N = N; A.K = K; A.KB = h->KB; A.NB = h->NB;
    A.act = h->d.activation; A.experts = h->d.experts;
    const mixaq_rows* const values = need ? x : nullptr;
    const TokenForm form = codes.type != MIXAQ_I8 ? TOKEN_FEW : token_form(rows, A.KB, A.NB, h->d.experts, sorted != nullptr, (sorted ? x_rows : 128LL) * A.ldx);
    if (sorted) {
        A.offsets = sorted->offsets; A.gather = sorted->gather; A.weights = sorted->weights;
        if (y->type == MIXAQ_F32) return launch_linear<MIXAQ_F32, true>(A, form, codes.type, values, st);
        if (y->type == MIXAQ_F16) return launch_linear<MIXAQ_F16, true>(A, form, codes.type, values, st);
        return launch_linear<MIXAQ_BF16, true>(A, form, codes.type, values, st);
    }
    if (y->type == MIXAQ_F32) return launch_linear<MIXAQ_F32, false>(A, form, codes.type, values, st);
    if (y->type == MIXAQ_F16) return launch_linear<MIXAQ_F16, false>(A, form, codes.type, values, st);
    return launch_linear<MIXAQ_BF16, false>(A, form, codes.type, values, st);
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
