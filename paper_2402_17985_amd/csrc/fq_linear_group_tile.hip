// fq_linear_group_i4 for more rows than the kernel of single tokens takes: tiles of X shared by the waves of a workgroup through LDS.
//
// A wave multiplies 16 MT rows by 16 NT columns; WN waves lie side by side and WK waves take turns along the reduction, a step of 128 columns each, so that few
// columns of output still give every CU work.  Everything is copied straight into a ring of S stages in LDS, S - 1 of them on their way: X for all waves, codes
// and scales for the one wave that needs them, which widens codes in registers once for all its rows.
// Codes stay whole numbers up to the end of a group, whose sum takes the scale in fp32: nothing is rounded to 16 bits on the way.
#include <algorithm>
#include <atomic>

#include "fq_gemm_common.h"
#include "fq_linear_group.h"
#include "fq_rules.h"

namespace fq {
namespace {

// s_waitcnt immediate: at most `vm` copies on their way, and no LDS operation
constexpr int wait_imm(int vm) { return (vm & 0xf) | ((vm >> 4) << 14) | 0x0070; }

// Copies of 2 or 4 bytes a lane into 4 bytes of LDS each, as dma16
__device__ __forceinline__ void dma2(const uint8_t* uniform_base, uint32_t lane_offset, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %0" : : "s"(uniform_base), "v"(lane_offset), "s"(lds_base) : "memory");
}
__device__ __forceinline__ void dma4(const uint8_t* uniform_base, uint32_t lane_offset, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, %0" : : "s"(uniform_base), "v"(lane_offset), "s"(lds_base) : "memory");
}

// Bytes of LDS: a wave's codes and scales of a stage; a stage; the whole
constexpr int own_bytes(int NT, int PER, bool offset) { return NT * 1024 + (NT * PER + 3) / 4 * 256 * (offset ? 2 : 1); }
constexpr int stage_bytes(int MT, int NT, int WN, int WK, int PER, bool offset) { return 16 * MT * 256 * WK + WN * WK * own_bytes(NT, PER, offset); }
constexpr int sums_bytes(int MT, int NT, int WN, int WK) { return WK * 16 * MT * (16 * NT * WN + 4) * 4; }

// GROUP = 32 serves groups of any size: every product of 32 columns takes its scale.  (NT * PER < 4: the copies of scales bring some of the columns behind, too.)
template <int XT, int MT, int NT, int WN, int WK, int S, int GROUP, bool OFFSET>
__global__ __launch_bounds__(64 * WN * WK) void linear_group_tile_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int THREADS = 64 * WN * WK, PER = 128 / GROUP, EACH = 4 / PER;
    constexpr bool SURPLUS = OFFSET || M_::SURPLUS;              // codes as q + 24 (2048 rows, 11008 x 4096, fp16 with offsets: 251 us, as q 261)
    constexpr bool TURN = GROUP != 128;                          // product j takes columns 32 j .. 32 j + 31, of one group
    constexpr int ROWS = 16 * MT, PITCH = 256 * WK, X_BYTES = ROWS * PITCH, COPIES = X_BYTES / 1024 / (WN * WK);
    constexpr int SCALES = (NT * PER + 3) / 4, OWN = own_bytes(NT, PER, OFFSET), STAGE = stage_bytes(MT, NT, WN, WK, PER, OFFSET);
    constexpr int IN_STAGE = COPIES + NT + SCALES * (OFFSET ? 2 : 1);      // copies of a wave
    static_assert(X_BYTES % (1024 * WN * WK) == 0, "whole copies a wave");
    static_assert((S - 2) * IN_STAGE < 64, "copies are counted in six bits");
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave % WN, wk = wave / WN;
    int tile_m, tile_n;
    tile_of_workgroup(blockIdx.x, a.tiles, a.tiles / a.tiles_n, a.tiles_n, tile_m, tile_n);
    const int m0 = tile_m * ROWS, n0 = (tile_n * WN + wn) * 16 * NT;
    const int steps = (a.K + 127) / 128, stages = (steps + WK - 1) / WK;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)FQ_LDS_PTR(lds));

    // ---- X: copies of 1 KiB; piece p of row m of a stage lies at place p ^ (m % 16), for the banks ----
    const uint8_t* x_tile = static_cast<const uint8_t*>(a.X) + (size_t)m0 * a.ldx * 2;
    uint32_t x_from[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int at = (wave * COPIES + i) * 64 + lane, row = at / (16 * WK);
        x_from[i] = (uint32_t)min(row, a.M - 1 - m0) * (uint32_t)(a.ldx * 2) + 16 * (at % (16 * WK) ^ (row & 15));
    }
    // ---- codes: lane l copies a piece of column l / 4, pieces turned by column / 4; scales: 64 (column, group of the step) to a copy ----
    const int n_first = min(n0, a.N - 1), n_last = a.N - 1 - n_first;
    const uint8_t* w_tile = a.Wq + (size_t)n_first * (a.K / 2);
    uint32_t w_from[NT], g_from[SCALES];
    const int piece = (lane & 3) ^ (lane >> 4);
#pragma unroll
    for (int j = 0; j < NT; ++j) w_from[j] = (uint32_t)min(16 * j + lane / 4, n_last) * (a.K / 2);
#pragma unroll
    for (int j = 0; j < SCALES; ++j) g_from[j] = (uint32_t)min((64 * j + lane) / PER, n_last) * a.groups;
    const int g_size = a.s_dtype == FQ_F32 ? 4 : 2;
    const uint8_t* s_tile = static_cast<const uint8_t*>(a.S) + (size_t)n_first * a.groups * g_size;
    const uint8_t* b_tile = static_cast<const uint8_t*>(a.B) + (size_t)n_first * a.groups * g_size;
    auto copy = [&](int stage, int buffer) {
        const uint32_t to = lds0 + buffer * STAGE, mine = to + X_BYTES + wave * OWN;
        const int k = stage * WK + wk;
        const uint32_t w_at = min(64 * k + 16 * piece, a.K / 2 - 16);      // what lies behind a row's end is read from its end
#pragma unroll
        for (int j = 0; j < NT; ++j) dma16(w_tile, w_from[j] + w_at, mine + j * 1024);
        const uint32_t group = min(GROUP == 32 ? (128 * k + 32 * (lane % 4)) >> a.group_shift : k * PER + lane % PER, a.groups - 1);
#pragma unroll
        for (int j = 0; j < SCALES; ++j) {
            const uint32_t at = mine + NT * 1024 + j * 256;
            if (g_size == 4) {
                dma4(s_tile, (g_from[j] + group) * 4, at);
                if (OFFSET) dma4(b_tile, (g_from[j] + group) * 4, at + SCALES * 256);
            } else {
                dma2(s_tile, (g_from[j] + group) * 2, at);
                if (OFFSET) dma2(b_tile, (g_from[j] + group) * 2, at + SCALES * 256);
            }
        }
        const uint8_t* from = x_tile + (size_t)stage * PITCH;
        if ((stage + 1) * WK * 128 <= a.K) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) dma16(from, x_from[i], to + (wave * COPIES + i) * 1024);
        } else {                                                 // zeros behind a row's end; the codes there do not matter then
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int at = (wave * COPIES + i) * 64 + lane, x_piece = at % (16 * WK) ^ (at / (16 * WK) & 15);
                dma16_addr(stage * WK * 128 + 8 * x_piece < a.K ? from + x_from[i] : reinterpret_cast<const uint8_t*>(g_zero_chunk),
                           to + (wave * COPIES + i) * 1024);
            }
        }
    };

    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
        if (i < stages) copy(i, i);
    for (int stage = 0, buffer = 0; stage < stages; ++stage) {
        // this stage's copies have landed, and the stage before it is read no more: its place is free
        if (stage + S - 1 <= stages) __builtin_amdgcn_s_waitcnt(wait_imm((S - 2) * IN_STAGE));
        else __builtin_amdgcn_s_waitcnt(wait_imm(0));
        asm volatile("s_barrier" ::: "memory");
        if (stage + S - 1 < stages) copy(stage + S - 1, buffer == 0 ? S - 1 : buffer - 1);
        const uint8_t* here = lds + buffer * STAGE;
        const uint8_t* own = here + X_BYTES + wave * OWN;
        buffer = buffer + 1 == S ? 0 : buffer + 1;
        v8 wf[NT][4];
        float s[NT][PER], b[NT][PER];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            v4u codes = *reinterpret_cast<const v4u*>(own + j * 1024 + 64 * r + 16 * (c ^ (r >> 2)));
            if (TURN) transpose_quarters(codes);
#pragma unroll
            for (int q = 0; q < 4; ++q) wf[j][q] = SURPLUS ? M_::widen24(codes[q]) : M_::widen(codes[q]);
            const uint32_t* scales = reinterpret_cast<const uint32_t*>(own + NT * 1024) + (16 * j + r) * PER;
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                s[j][g] = a.value(scales[g]);
                // An offset takes the surplus out as well, without a product of its own (2048 rows, 11008 x 4096 with groups of 128 245 us instead of 261)
                b[j][g] = OFFSET ? a.value(scales[SCALES * 64 + g]) : 0.0f;
                if (OFFSET) b[j][g] = __builtin_fmaf(-24.0f, s[j][g], b[j][g]);
            }
        }
        const uint8_t* x_at = here + r * PITCH;
        auto operands = [&](int i, v8 (&xf)[4]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) xf[q] = *reinterpret_cast<const v8*>(x_at + 16 * i * PITCH + 16 * ((16 * wk + (TURN ? 4 * q + c : 4 * c + q)) ^ r));
        };
        v8 x[2][4];
        operands(0, x[0]);
        // Where a CU has several workgroups, one that multiplies goes before one that widens codes, so that they fall out of step: 2048 rows, 11008 x 4096 with
        // groups of 128 / 64 / 32 224 / 271 / 341 us instead of 237 / 291 / 348 (matrix instructions alone before the others: 235 / 283 / 344).
        if (WK == 1) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (i + 1 < MT) operands(i + 1, x[(i + 1) % 2]);
            const v8 (&xf)[4] = x[i % 2];
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                v4f p[NT], less = {0.0f, 0.0f, 0.0f, 0.0f}, sum = less;
#pragma unroll
                for (int q = EACH * g; q < EACH * (g + 1); ++q) {
                    if (SURPLUS && !OFFSET) less = M_::mul(xf[q], M_::all(true), less);
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
            if (MT * NT > 8) __builtin_amdgcn_sched_barrier(0);      // large tiles: operands of two blocks of rows are enough in registers
        }
        if (WK == 1) __builtin_amdgcn_s_setprio(0);
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

template <int XT, int MT, int NT, int WN, int WK, int S, int GROUP, bool OFFSET> int launch_one(GroupProduct a, hipStream_t stream)
{
    constexpr int SMEM = std::max(S * stage_bytes(MT, NT, WN, WK, 128 / GROUP, OFFSET), sums_bytes(MT, NT, WN, WK));
    static_assert(SMEM <= 160 * 1024, "LDS of a CU");
    auto kern = linear_group_tile_kernel<XT, MT, NT, WN, WK, S, GROUP, OFFSET>;
    const long long tiles_n = ((long long)a.N + 16 * NT * WN - 1) / (16 * NT * WN), tiles = tiles_n * (((long long)a.M + 16 * MT - 1) / (16 * MT));
    if (!launch_holds(tiles, 64 * WN * WK)) return fail(FQ_ERR_RANGE, "%d x %d outputs are more than one launch holds", a.M, a.N);
    a.tiles_n = (int)tiles_n;
    a.tiles = (int)tiles;
    static std::atomic<unsigned long long> attr_set;
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), SMEM, attr_set)) return rc;
    kern<<<(unsigned)a.tiles, 64 * WN * WK, SMEM, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group-scaled layer launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}
template <int XT, int MT, int NT, int WN, int WK, int S, int GROUP = 32> int launch(const GroupProduct& a, hipStream_t stream)
{
    return a.B ? launch_one<XT, MT, NT, WN, WK, S, GROUP, true>(a, stream) : launch_one<XT, MT, NT, WN, WK, S, GROUP, false>(a, stream);
}

}  // namespace

// Tiles by how many there are: the smallest of which each CU gets one at most, as a workgroup's time goes by its stages more than by what is in them
// (32 x 32, 512 or 768 columns a stage: 1.0 or 1.35 us; without the copies of X 15 % less, without those of the scales 4 %).
// us (bf16, groups of 128 or as given), the taken one first:
//   16 x 16    16 rows, 4096 x 11008: 11; 16 x 32 15
//   16 x 32    16 rows, 22016 x 8192: 39; 16 x 16 50.  As for groups of 32 whatever their size: with groups of 128 for themselves 44
//   32 x 16    24 rows, 4096 x 11008: 16; 32 x 32 19.  64 rows, 1024 x 4096: 6.4; 32 x 32 8.7
//   32 x 32    64 rows, 4096 x 4096: 9.6; 32 x 64 13.  512 columns a stage with groups of 128, three stages; else 768, two: the last, and the other one, over 4096 x
//              11008 with groups of 32 24 and 28, 64 22 and 25, 128 20 and 22, but 128 over 4096 x 4096 10.7 and 9.9, 8192 x 8192 (32 rows) 17.7 and 16.5
//   32 x 64    128 rows, 4096 x 4096: 13; 32 x 128 16
//   48 x 64    48 rows, 11008 x 4096: 15.5; 32 x 128 16.4.  22016 x 8192: 65; 32 x 128 71
//   32 x 128   256 rows, 4096 x 4096: 17; 64 x 128 21; 32 x 64 26.  128 rows, 11008 x 4096: 31; 64 x 128 38.  512 rows, 4096 x 4096: 33; 64 x 128 31
// Groups of 64 and 128 columns have kernels of their own: 64 rows, 4096 x 4096, groups of 128: 9.6; as for groups of 32 12.
template <int XT, int GROUP> int launch_small(const GroupProduct& a, long long cus, hipStream_t stream)
{
    const long long M = a.M, N = a.N;
    auto tiles = [&](int rows, int cols) { return ((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
    if (M <= 16) return tiles(16, 16) <= cus ? launch<XT, 1, 1, 1, 8, 3, GROUP>(a, stream) : launch<XT, 1, 1, 2, 8, 2, 32>(a, stream);
    if (tiles(32, 16) <= cus) return launch<XT, 2, 1, 1, 8, 2, GROUP>(a, stream);
    if (tiles(32, 32) <= cus) return GROUP == 128 ? launch<XT, 2, 1, 2, 4, 3, 128>(a, stream) : launch<XT, 2, 1, 2, 6, 2, GROUP>(a, stream);
    if (tiles(32, 64) <= cus) return launch<XT, 2, 1, 4, 4, 2, GROUP>(a, stream);
    if (M > 32 && M <= 48) return launch<XT, 3, 1, 4, 4, 2, GROUP>(a, stream);
    return launch<XT, 2, 2, 4, 4, 2, GROUP>(a, stream);
}
// Large tiles where the smaller ones would take turns on the CUs: us, 64 x 256 with two waves along the reduction / with one / 32 x 128:
// 256 rows, 11008 x 4096 45 / 57 / 47; 1024 rows, 4096 x 4096 46 / 58 / 69; 512 rows, 11008 x 4096 87 / 75 / 91; 2048 rows, 11008 x 4096 255 / 232 / 329.
// With groups of 32 columns there is a scale to apply after every matrix product, and large tiles of 128 columns are best (2048 rows, 11008 x 4096: 345; 256 columns
// 512), from more of them on: 64 x 128 / 32 x 128, 256 rows, 11008 x 4096 75 / 68, 384 rows 105 / 112, 512 rows 102 / 133.
template <int XT> int launch_group_tile(const GroupProduct& product, int group, hipStream_t stream)
{
    GroupProduct a = product;
    a.group_shift = group == 32 ? 5 : group == 64 ? 6 : 7;
    const long long cus = compute_units(), M = a.M, N = a.N;
    const long long large = (M + 63) / 64 * ((N + 127) / 128);
    if (M <= 48 || 2 * large <= (group == 32 ? 3 : 2) * cus)
        return group == 32 ? launch_small<XT, 32>(a, cus, stream) : group == 64 ? launch_small<XT, 64>(a, cus, stream) : launch_small<XT, 128>(a, cus, stream);
    if (group == 32) return launch<XT, 4, 2, 4, 1, 2>(a, stream);
    if ((M + 63) / 64 * ((N + 255) / 256) <= cus) return group == 64 ? launch<XT, 4, 4, 4, 2, 2, 64>(a, stream) : launch<XT, 4, 4, 4, 2, 2, 128>(a, stream);
    return group == 64 ? launch<XT, 4, 4, 4, 1, 2, 64>(a, stream) : launch<XT, 4, 4, 4, 1, 2, 128>(a, stream);
}
#if FQ_GROUP_TYPE == 1
template int launch_group_tile<FQ_F16>(const GroupProduct&, int, hipStream_t);
#else
template int launch_group_tile<FQ_BF16>(const GroupProduct&, int, hipStream_t);
#endif

}  // namespace fq
