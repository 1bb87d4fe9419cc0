// fq_linear_group_i4 for more rows than the kernel of single tokens takes: tiles of X shared by the waves of a workgroup through LDS.
//
// A wave multiplies 16 MT rows by 16 NT columns; WN waves lie side by side and WK waves take turns along the reduction, a step of 128 columns each, so that few
// columns of output still give every CU work.  X is copied straight into one of two buffers in LDS while the other is multiplied; weights go from
// memory into the registers of the one wave that needs them, a step ahead, and are widened there, once for all its rows.
// Codes stay whole numbers up to the end of a group, whose sum takes the scale in fp32: nothing is rounded to 16 bits on the way.
#include <algorithm>
#include <atomic>

#include "fq_gemm_common.h"
#include "fq_linear_group.h"

namespace fq {
namespace {

// GROUP = 32 serves groups of any size: every product of 32 columns takes its scale.
template <int XT, int MT, int NT, int WN, int WK, int GROUP, bool OFFSET>
__global__ __launch_bounds__(64 * WN * WK) void linear_group_tile_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int THREADS = 64 * WN * WK, PER = 128 / GROUP, EACH = 4 / PER;
    constexpr bool TURN = GROUP != 128;                          // product j takes columns 32 j .. 32 j + 31, of one group
    constexpr int ROWS = 16 * MT, PITCH = 256 * WK, BUFFER = ROWS * PITCH, COPIES = BUFFER / 1024 / (WN * WK);
    static_assert(BUFFER % (1024 * WN * WK) == 0, "whole copies a wave");
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave % WN, wk = wave / WN;
    int tile_m, tile_n;
    tile_of_workgroup(blockIdx.x, a.tiles, a.tiles / a.tiles_n, a.tiles_n, tile_m, tile_n);
    const int m0 = tile_m * ROWS, n0 = (tile_n * WN + wn) * 16 * NT;
    const int steps = (a.K + 127) / 128, stages = (steps + WK - 1) / WK;

    // ---- copies of X: 1 KiB each; piece p of row m of a buffer lies at place p ^ (m % 16), for the banks ----
    const uint8_t* x_tile = static_cast<const uint8_t*>(a.X) + (size_t)m0 * a.ldx * 2;
    uint32_t x_from[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int at = (wave * COPIES + i) * 64 + lane, row = at / (16 * WK);
        x_from[i] = (uint32_t)min(row, a.M - 1 - m0) * (uint32_t)(a.ldx * 2) + 16 * (at % (16 * WK) ^ (row & 15));
    }
    const uint32_t x_lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)FQ_LDS_PTR(lds)) + wave * COPIES * 1024;
    auto copy = [&](int stage) {
        const uint8_t* from = x_tile + (size_t)stage * PITCH;
        const uint32_t to = x_lds + (stage & 1) * BUFFER;
        if ((stage + 1) * WK * 128 <= a.K) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) dma16(from, x_from[i], to + i * 1024);
        } else {                                                 // zeros behind a row's end; the codes there do not matter then
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int at = (wave * COPIES + i) * 64 + lane, piece = at % (16 * WK) ^ (at / (16 * WK) & 15);
                dma16_addr(stage * WK * 128 + 8 * piece < a.K ? from + x_from[i] : reinterpret_cast<const uint8_t*>(g_zero_chunk), to + i * 1024);
            }
        }
    };
    // ---- codes and scales of the wave's columns: lane l has piece l % 4 of the step of column l / 4, and scale l % 4 ----
    const uint8_t* w_tile = a.Wq + (size_t)min(n0, a.N - 1) * (a.K / 2);
    uint32_t w_row[NT], g_row[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = max(min(16 * j + lane / 4, a.N - 1 - n0), 0);
        w_row[j] = (uint32_t)n * (a.K / 2);
        g_row[j] = (uint32_t)n * a.groups;
    }
    const size_t g_tile = (size_t)min(n0, a.N - 1) * a.groups;
    v4u w_next[NT];
    uint32_t s_next[NT], b_next[NT];
    auto load = [&](int stage) {
        const int k = stage * WK + wk;
        const uint32_t w_at = min(64 * k + 16 * (lane % 4), a.K / 2 - 16);
        const uint32_t group = min(GROUP == 32 ? (128 * k + 32 * (lane % 4)) >> a.group_shift : k * PER + lane % 4, a.groups - 1);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w_next[j] = *reinterpret_cast<const v4u*>(w_tile + (w_row[j] + w_at));
            s_next[j] = a.one_scale(a.S, g_tile + (g_row[j] + group));
            if (OFFSET) b_next[j] = a.one_scale(a.B, g_tile + (g_row[j] + group));
        }
    };

    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    load(0);
    copy(0);
    for (int stage = 0; stage < stages; ++stage) {
        // this stage's copies have landed, and the other buffer is read no more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
        if (stage + 1 < stages) {
            load(stage + 1);
            copy(stage + 1);
        }
        const uint8_t* x_at = lds + (stage & 1) * BUFFER + r * PITCH;
        auto operands = [&](int i, v8 (&xf)[4]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) xf[q] = *reinterpret_cast<const v8*>(x_at + 16 * i * PITCH + 16 * ((16 * wk + (TURN ? 4 * q + c : 4 * c + q)) ^ r));
        };
        v8 x[2][4];
        operands(0, x[0]);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (i + 1 < MT) operands(i + 1, x[(i + 1) % 2]);
            const v8 (&xf)[4] = x[i % 2];
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
            __builtin_amdgcn_sched_barrier(0);       // operands of two blocks of rows are enough in registers
        }
    }
    __syncthreads();

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

template <int XT, int MT, int NT, int WN, int WK, bool ANY> int launch(GroupProduct a, int group, hipStream_t stream)
{
    void (*kern)(GroupProduct);
    if constexpr (ANY) kern = a.B ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, true> : linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, false>;
    else
        kern = a.B ? (group == 32 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, true> : group == 64 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 64, true> : linear_group_tile_kernel<XT, MT, NT, WN, WK, 128, true>)
                   : (group == 32 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 32, false> : group == 64 ? linear_group_tile_kernel<XT, MT, NT, WN, WK, 64, false> : linear_group_tile_kernel<XT, MT, NT, WN, WK, 128, false>);
    constexpr int SMEM = std::max(2 * 16 * MT * 256 * WK, WK * 16 * MT * (16 * NT * WN + 4) * 4);
    static std::atomic<unsigned long long> attr_set[6];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), SMEM, attr_set[(group == 32 ? 0 : group == 64 ? 1 : 2) + (a.B ? 3 : 0)])) return rc;
    a.group_shift = group == 32 ? 5 : group == 64 ? 6 : 7;
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
    if (rows64 * ((a.N + 255) / 256) >= cus) return launch<XT, 4, 4, 4, 1, false>(a, group, stream);
    const bool wide = rows64 * ((a.N + 31) / 32) >= cus;
    if (a.M <= 16) return wide ? launch<XT, 1, 2, 1, 8, true>(a, group, stream) : launch<XT, 1, 1, 1, 8, true>(a, group, stream);
    if (a.M <= 32) return wide ? launch<XT, 2, 2, 1, 4, true>(a, group, stream) : launch<XT, 2, 1, 1, 4, true>(a, group, stream);
    if (a.M <= 48) return wide ? launch<XT, 3, 2, 1, 4, true>(a, group, stream) : launch<XT, 3, 1, 1, 4, true>(a, group, stream);
    return wide ? launch<XT, 4, 2, 1, 4, true>(a, group, stream) : launch<XT, 4, 1, 1, 4, true>(a, group, stream);
}
#if FQ_GROUP_TYPE == 1
template int launch_group_tile<FQ_F16>(const GroupProduct&, int, hipStream_t);
#else
template int launch_group_tile<FQ_BF16>(const GroupProduct&, int, hipStream_t);
#endif

}  // namespace fq
