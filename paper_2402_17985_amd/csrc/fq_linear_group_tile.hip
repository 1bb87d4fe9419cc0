// fq_linear_group_i4 for more rows than the kernel of single tokens takes: tiles of X shared by the waves of a workgroup through LDS.
//
// A wave multiplies 16 MT rows by 16 NT columns; WN waves lie side by side and WK waves take turns along the reduction, a step of 128 columns each, so that few
// columns of output still give every CU work.  X goes through registers into one of two buffers in LDS while the other is multiplied; weights go from
// memory into the registers of the one wave that needs them, a step ahead, and are widened there, once for all its rows.
// Codes stay whole numbers up to the end of a group, whose sum takes the scale in fp32: nothing is rounded to 16 bits on the way.
#include <algorithm>
#include <atomic>

#include "fq_internal.h"
#include "fq_linear_group.h"

namespace fq {
namespace {

template <int XT, int MT, int NT, int WN, int WK, int GROUP, bool OFFSET>
__global__ __launch_bounds__(64 * WN * WK, 2) void linear_group_tile_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int THREADS = 64 * WN * WK, PER = 128 / GROUP, EACH = 4 / PER;
    constexpr bool TURN = GROUP != 128;                          // product j takes columns 32 j .. 32 j + 31, of one group
    constexpr int ROWS = 16 * MT, PITCH = 256 * WK, BUFFER = ROWS * PITCH, PIECES = ROWS * WK * 16 / THREADS;
    static_assert(ROWS * WK * 16 % THREADS == 0, "whole pieces a thread");
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave % WN, wk = wave / WN;
    int tile_m, tile_n;
    group_tile(blockIdx.x, a.tiles / a.tiles_n, a.tiles_n, tile_m, tile_n);
    const int m0 = tile_m * ROWS, n0 = (tile_n * WN + wn) * 16 * NT;
    const int steps = (a.K + 127) / 128, stages = (steps + WK - 1) / WK;

    // ---- what a thread loads for a stage: pieces of X, codes and scales of its wave's columns ----
    const uint8_t* x_base = static_cast<const uint8_t*>(a.X);
    size_t x_row[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) x_row[i] = (size_t)min(m0 + (tid + i * THREADS) / (16 * WK), a.M - 1) * a.ldx * 2;
    const int x_piece = tid % (16 * WK);                         // the same for all of them: THREADS is a multiple of a row's pieces
    static_assert(THREADS % (16 * WK) == 0, "");
    const uint8_t* w_row[NT];
    size_t g_row[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = min(n0 + 16 * j + lane / 4, a.N - 1);
        w_row[j] = a.Wq + (size_t)n * (a.K / 2);
        g_row[j] = (size_t)n * a.groups;
    }
    v4u x_next[PIECES], w_next[NT];
    uint32_t s_next[NT], b_next[NT];
    auto load = [&](int stage) {
        const int col = stage * 128 * WK + 8 * x_piece, k = stage * WK + wk;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x_next[i] = *reinterpret_cast<const v4u*>(x_base + x_row[i] + 2 * min(col, a.K - 8));
        if (col >= a.K) {                                        // zeros behind a row's end; the codes there do not matter then
#pragma unroll
            for (int i = 0; i < PIECES; ++i) x_next[i] = v4u{0, 0, 0, 0};
        }
        const int group = min(k * PER + lane % 4, a.groups - 1);      // lane l: scale l % 4 of the step, of column l / 4
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w_next[j] = *reinterpret_cast<const v4u*>(w_row[j] + min(64 * k + 16 * (lane % 4), a.K / 2 - 16));
            s_next[j] = a.one_scale(a.S, g_row[j] + group);
            if (OFFSET) b_next[j] = a.one_scale(a.B, g_row[j] + group);
        }
    };
    auto store_x = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int row = (tid + i * THREADS) / (16 * WK);
            *reinterpret_cast<v4u*>(lds + buffer * BUFFER + row * PITCH + 16 * (x_piece ^ (row & 15))) = x_next[i];
        }
    };

    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    load(0);
    store_x(0);
    __syncthreads();
    for (int stage = 0; stage < stages; ++stage) {
        v8 wf[NT][4];
        float s[NT][PER], b[NT][PER];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            v4u codes;
#pragma unroll
            for (int q = 0; q < 4; ++q) codes[q] = __shfl(w_next[j][q], 4 * r + c, 64);
            if (TURN) transpose_quarters(codes);
#pragma unroll
            for (int q = 0; q < 4; ++q) wf[j][q] = M_::widen(codes[q]);
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                s[j][g] = a.value(__shfl(s_next[j], 4 * r + g, 64));
                b[j][g] = OFFSET ? a.value(__shfl(b_next[j], 4 * r + g, 64)) : 0.0f;
            }
        }
        if (stage + 1 < stages) load(stage + 1);
        const uint8_t* x_at = lds + (stage & 1) * BUFFER + r * PITCH;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            v8 xf[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) xf[q] = *reinterpret_cast<const v8*>(x_at + 16 * i * PITCH + 16 * ((16 * wk + (TURN ? 4 * q + c : 4 * c + q)) ^ r));
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                v4f p[NT], less = {0.0f, 0.0f, 0.0f, 0.0f}, sum = less;
#pragma unroll
                for (int q = EACH * g; q < EACH * (g + 1); ++q) {
                    if (M_::SURPLUS) less = M_::mul(xf[q], M_::all(true), less);
                    if (OFFSET) sum = M_::mul(xf[q], M_::all(false), sum);
                }
#pragma unroll
                for (int q = EACH * g; q < EACH * (g + 1); ++q)
#pragma unroll
                    for (int j = 0; j < NT; ++j) p[j] = M_::mul(xf[q], wf[j][q], q == EACH * g ? less : p[j]);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[i][j][e] = __builtin_fmaf(s[j][g], p[j][e], acc[i][j][e]);
                        if (OFFSET) acc[i][j][e] = __builtin_fmaf(b[j][g], sum[e], acc[i][j][e]);
                    }
            }
        }
        if (stage + 1 < stages) store_x((stage + 1) & 1);        // read last in the stage before this one
        __syncthreads();
    }

    // ---- the waves' sums meet in LDS; rows leave four columns a thread ----
    constexpr int COLS = 16 * NT * WN;
    float* sums = reinterpret_cast<float*>(lds);                 // [WK][ROWS][COLS + 4]
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(wk * ROWS + 16 * i + 4 * c + e) * (COLS + 4) + (wn * NT + j) * 16 + r] = acc[i][j][e];
    __syncthreads();
    for (int at = tid; at < ROWS * COLS / 4; at += THREADS) {
        const int row = at / (COLS / 4), col = at % (COLS / 4) * 4, m = m0 + row, n = tile_n * COLS + col;
        if (m >= a.M || n >= a.N) continue;
        v4f v = *reinterpret_cast<const v4f*>(sums + row * (COLS + 4) + col);
#pragma unroll
        for (int k = 1; k < WK; ++k) v += *reinterpret_cast<const v4f*>(sums + (k * ROWS + row) * (COLS + 4) + col);
        a.store4(v, m, n);
    }
}

template <int XT, int MT, int NT, int WN, int WK> int launch(GroupProduct a, int group, hipStream_t stream)
{
    auto kern = a.B ? (group == 32 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, true> : group == 64 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 64, true> : linear_group_tile_kernel<XT, MT, NT, WN, WK, 128, true>)
                    : (group == 32 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, false> : group == 64 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 64, false> : linear_group_tile_kernel<XT, MT, NT, WN, WK, 128, false>);
    constexpr int SMEM = std::max(2 * 16 * MT * 256 * WK, WK * 16 * MT * (16 * NT * WN + 4) * 4);
    static std::atomic<unsigned long long> attr_set[6];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), SMEM, attr_set[(group == 32 ? 0 : group == 64 ? 1 : 2) + (a.B ? 3 : 0)])) return rc;
    a.tiles_n = (a.N + 16 * NT * WN - 1) / (16 * NT * WN);
    a.tiles = a.tiles_n * ((a.M + 16 * MT - 1) / (16 * MT));
    kern<<<(unsigned)a.tiles, 64 * WN * WK, SMEM, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group-scaled layer launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

}  // namespace

template <int XT> int launch_group_tile(const GroupProduct& a, int group, hipStream_t stream)
{
    const long long cus = compute_units(), rows64 = (a.M + 63) / 64;
    if (rows64 * ((a.N + 255) / 256) >= cus) return launch<XT, 4, 4, 4, 1>(a, group, stream);
    if (a.M > 32 && rows64 * ((a.N + 63) / 64) >= cus) return launch<XT, 4, 2, 2, 2>(a, group, stream);
    if (a.M <= 16) return launch<XT, 1, 1, 1, 4>(a, group, stream);
    if (a.M <= 32) return launch<XT, 2, 1, 1, 4>(a, group, stream);
    if (a.M <= 48) return launch<XT, 3, 1, 1, 4>(a, group, stream);
    return launch<XT, 4, 1, 1, 4>(a, group, stream);
}
#if FQ_GROUP_TYPE == 1
template int launch_group_tile<FQ_F16>(const GroupProduct&, int, hipStream_t);
#else
template int launch_group_tile<FQ_BF16>(const GroupProduct&, int, hipStream_t);
#endif

}  // namespace fq
