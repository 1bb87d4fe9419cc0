// fq_linear_group_i4: 16-bit activations times 4-bit weights with group scales, few rows.
//
// Y[i,n] = sum over groups of s (sum x q) + b (sum x).  A code enters the matrix product as the 16-bit number 16 + u (u = q + 8, four
// bits ORed below the exponent of 16): exact, and made in one shift and one three-operand logic instruction for two weights.  bf16
// products therefore carry 24 (sum x) too much, which leaves with the offset: s P + (b - 24 s) (sum x), sum x being a product with ones.
// fp16 has a packed subtraction: codes are q itself there.
// With few rows the call is the stream of its weights.  A workgroup owns 16 columns and all of the reduction: its eight waves take
// 256 columns of the reduction (one cache line of each of the 16 rows) in turn, straight into registers, some steps ahead, and their sums
// meet in LDS once; no barrier before that.
#include <algorithm>
#include <atomic>

#include "fq_internal.h"
#include "fq_linear_group.h"

namespace fq {
namespace {


// rows of X in LDS
constexpr int x_bytes(int M, int K) { return M * ((K + 127) / 128 * 256 + 16); }

// Workgroup barrier that orders LDS only: loads stay in flight across it.
__device__ __forceinline__ void strip_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// XLDS: all rows of X lie in LDS (the first tile's weights are on their way meanwhile); else they come with the weights, step by step.
template <int XT, int NW, int MT, int GROUP, bool OFFSET, bool XLDS, int D>
__global__ __launch_bounds__(NW * 64) void linear_group_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int THREADS = NW * 64;
    constexpr int PER = 128 / GROUP, EACH = 4 / PER;            // groups in a step of 128 columns, products (32 columns) in a group
    static_assert(4 % D == 0, "the ring divides a chunk");
    extern __shared__ __align__(16) uint8_t lds[];
    v4f* red = reinterpret_cast<v4f*>(lds);                     // two of [NW][MT][64]
    uint8_t* x_lds = lds + 2 * NW * MT * 1024;
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // ---- steps of 128 columns: a wave has a stretch of them, chunks of four ----
    const int whole = a.K / 128, steps = (a.K + 127) / 128;
    const int each = ((steps + NW - 1) / NW + 1) & ~1;          // even: two steps are a cache line of a row
    const int first = min(wave * each, steps), last = min(first + each, steps);
    // a lane's columns of a step in product d: 8 from x_col + x_next * d on
    constexpr bool TURN = GROUP != 128;                         // product d takes columns 32 d .. 32 d + 31, of one group
    constexpr int x_next = TURN ? 32 : 8;
    const int x_col = TURN ? 8 * c : 32 * c;

    // what is loaded next: a chunk of a tile
    const uint8_t* w_row;
    size_t g_row;
    const uint16_t* x_row[MT][4];
    // Loads are laid out so that neighbouring lanes read neighbouring pieces (a wave's load is worked on lane by lane else, four times as long): lane l
    // reads 16 bytes l % 4 of the step of row l / 4 of the weights; lanes() brings them where the matrix instruction wants them.
    auto column = [&](int tile) { return min(tile % a.tiles_n * 16 + lane / 4, a.N - 1); };
    auto begin_scales = [&](int tile) { g_row = (size_t)column(tile) * a.groups; };
    auto begin_rows = [&](int tile) {
        const int m0 = tile / a.tiles_n * 16 * MT;
        w_row = a.Wq + (size_t)column(tile) * (a.K / 2);
        if (XLDS) return;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) x_row[i][q] = static_cast<const uint16_t*>(a.X) + (size_t)min(m0 + 16 * i + 4 * q + c, a.M - 1) * a.ldx;
    };
    v4u w[D], x[D][MT][4];
    StepScales<PER> s_next, b_next = {};
    // lane l has the scales of row l / 4 in step l % 4 of a chunk
    auto load_scales = [&](int k) {
        s_next = a.step_scales<PER>(a.S, g_row, (k + lane % 4) * PER);
        if (OFFSET) b_next = a.step_scales<PER>(a.B, g_row, (k + lane % 4) * PER);
    };
    // No branches around loads: where paths meet, the compiler has to wait as if the later ones had not been issued.  What lies behind a row's end is
    // read from its end, and not used.
    auto load = [&](int d, int k) {
        w[d] = *reinterpret_cast<const v4u*>(w_row + min(64 * k + 16 * (lane % 4), a.K / 2 - 16));
        if (XLDS) return;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) x[d][i][q] = *reinterpret_cast<const v4u*>(x_row[i][q] + min(128 * k + 8 * r, a.K - 8));      // 256 bytes of four rows
    };
    begin_scales(blockIdx.x);
    begin_rows(blockIdx.x);
    load_scales(first);
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, first + d);
    // rows of X 16 bytes further than whole steps, so that 16 rows are read from all banks; zeros behind the columns
    const int pitch = steps * 256 + 16;
    const uint8_t* x_at = x_lds + (r < a.M ? r : 0) * pitch + 2 * x_col;
    // else 16 rows of a step pass through a wave's own 4 KiB; piece p of row m lies at place p ^ m, again for the banks
    uint8_t* turn = x_lds + wave * 4096;
    if (XLDS) {
        const int pieces = steps * 16;
        for (int i = threadIdx.x; i < a.M * pieces; i += THREADS) {
            const int m = i / pieces, p = i % pieces;
            v4u v = {0, 0, 0, 0};
            if (8 * p < a.K) v = *reinterpret_cast<const v4u*>(static_cast<const uint16_t*>(a.X) + (size_t)m * a.ldx + 8 * p);
            *reinterpret_cast<v4u*>(x_lds + m * pitch + 16 * p) = v;
        }
        strip_barrier();
    }

    v4f acc[MT];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    };
    // Products of a step; `products` of its four (32 columns each) lie in the row.  Scalar conditions: the matrix instruction ignores the execution mask.
    auto compute = [&](int d, int k, int products, const float (&s)[PER], const float (&b)[PER]) {
        v4u codes;
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[j] = __shfl(w[d][j], 4 * r + c, 64);
        if (TURN) transpose_quarters(codes);
        const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (!XLDS) {
#pragma unroll
                for (int q = 0; q < 4; ++q) *reinterpret_cast<v4u*>(turn + (4 * q + c) * 256 + 16 * (r ^ (4 * q + c))) = x[d][i][q];
            }
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                if (EACH * g >= products) continue;
                v4f p = zero, sum = zero;
#pragma unroll
                for (int q = 0; q < EACH; ++q) {
                    const int j = EACH * g + q;
                    v8 xf;
                    if (XLDS) xf = *reinterpret_cast<const v8*>(x_at + 256 * k + 2 * x_next * j);
                    else xf = *reinterpret_cast<const v8*>(turn + r * 256 + 16 * ((TURN ? 4 * j + c : 4 * c + j) ^ r));
                    if (!XLDS && !TURN && 32 * c + 8 * j >= 32 * products) xf = M_::none();      // behind the row's end
                    if (TURN && j >= products) continue;
                    p = M_::mul(xf, M_::widen(codes[j]), p);
                    if (M_::SURPLUS) p = M_::mul(xf, M_::all(true), p);
                    if (OFFSET) sum = M_::mul(xf, M_::all(false), sum);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[i][e] = __builtin_fmaf(s[g], p[e], acc[i][e]);
                    if (OFFSET) acc[i][e] = __builtin_fmaf(b[g], sum[e], acc[i][e]);
                }
            }
        }
    };
    // a chunk: its four steps, and the loads of the one after it: in the same tile, at the beginning of the tile `after`, or none
    enum { SAME, AFTER, NO_MORE };
    auto chunk = [&](int k, int after, auto more) {
        constexpr int MORE = decltype(more)::value;
        const int next = MORE == SAME ? k + 4 : first;
        float s[4][PER], b[4][PER];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                s[t][g] = a.scale_at(g, [&](int i) { return __shfl(s_next.v[i], 4 * r + t, 64); });
                b[t][g] = OFFSET ? a.scale_at(g, [&](int i) { return __shfl(b_next.v[i], 4 * r + t, 64); }) : 0.0f;
            }
        if (MORE == AFTER) begin_scales(after);
        if (MORE != NO_MORE) load_scales(next);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (k + t < min(last, whole)) compute(t % D, k + t, 4, s[t], b[t]);
            else if (k + t < last) compute(t % D, k + t, (a.K - 128 * (k + t)) / 32, s[t], b[t]);
            __builtin_amdgcn_sched_barrier(0);      // a step's registers are loaded again when it is done, not before
            if (MORE == AFTER && t + D == 4) begin_rows(after);
            if (t + D < 4) load(t % D, k + t + D);
            else if (MORE != NO_MORE) load(t % D, next + t + D - 4);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int half = 0;
    auto finish = [&](int tile) {
        v4f* mine = red + half * (NW * MT * 64);
#pragma unroll
        for (int i = 0; i < MT; ++i) mine[(wave * MT + i) * 64 + lane] = acc[i];
        strip_barrier();
        const float* sums = reinterpret_cast<const float*>(mine);
        const int n0 = tile % a.tiles_n * 16, m0 = tile / a.tiles_n * 16 * MT;
        for (int e = threadIdx.x; e < MT * 256; e += THREADS) {
            const int m = m0 + e / 16, col = n0 + e % 16;
            if (m >= a.M || col >= a.N) continue;
            const int at = (e / 256 * 64 + e / 16 % 16 / 4 * 16 + e % 16) * 4 + e / 16 % 4;
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < NW; ++i) v += sums[i * MT * 256 + at];
            if (a.bias) v += a.bias[col];
            a.store(v, (size_t)m * a.ldy + col);
        }
        half ^= 1;      // these sums are read while the next tile's are written; its barrier comes before they are written again
    };
    for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        clear();
        const int after = tile + gridDim.x;
        int k = first;
        for (; k + 4 < last; k += 4) chunk(k, 0, std::integral_constant<int, SAME>{});
        if (k < last) {
            if (after < a.tiles) chunk(k, after, std::integral_constant<int, AFTER>{});
            else chunk(k, 0, std::integral_constant<int, NO_MORE>{});
        }
        finish(tile);
    }
}

template <int XT, int NW, int MT, bool XLDS, int D> int launch(GroupProduct a, int group, int wgs, hipStream_t stream)
{
    auto kern = a.B ? (group == 32 ? linear_group_kernel<XT, NW, MT, 32, true, XLDS, D> : group == 64 ? linear_group_kernel<XT, NW, MT, 64, true, XLDS, D> : linear_group_kernel<XT, NW, MT, 128, true, XLDS, D>)
                    : (group == 32 ? linear_group_kernel<XT, NW, MT, 32, false, XLDS, D> : group == 64 ? linear_group_kernel<XT, NW, MT, 64, false, XLDS, D> : linear_group_kernel<XT, NW, MT, 128, false, XLDS, D>);
    const int smem = 2 * NW * MT * 1024 + (XLDS ? x_bytes(a.M, a.K) : NW * 4096);
    static std::atomic<unsigned long long> attr_set[6];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), 160 * 1024, attr_set[(group == 32 ? 0 : group == 64 ? 1 : 2) + (a.B ? 3 : 0)])) return rc;
    a.tiles_n = (a.N + 15) / 16;
    a.tiles = a.tiles_n * ((a.M + 16 * MT - 1) / (16 * MT));
    kern<<<(unsigned)std::min(a.tiles, wgs), NW * 64, smem, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group-scaled layer launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

}  // namespace

int launch_linear_group(const void* X, int x_dtype, int M, int K, int ldx, const void* Wq, const void* S, const void* B, int s_dtype, int group, int N,
                        const float* bias, void* Y, int y_dtype, int ldy, hipStream_t stream)
{
    GroupProduct a = {};
    a.X = X; a.Wq = static_cast<const uint8_t*>(Wq); a.S = S; a.B = B; a.bias = bias; a.Y = Y;
    a.M = M; a.N = N; a.K = K; a.groups = (K + group - 1) / group; a.s_dtype = s_dtype; a.y_dtype = y_dtype;
    a.ldx = ldx; a.ldy = ldy;
    const int cus = compute_units();
    auto with = [&](auto xt) -> int {
        constexpr int XT = decltype(xt)::value;
        if (M <= 16 && x_bytes(M, K) <= 64 * 1024) return launch<XT, 8, 1, true, 4>(a, group, 2 * cus, stream);
        if (M <= 16 && x_bytes(M, K) <= 128 * 1024) return launch<XT, 16, 1, true, 4>(a, group, cus, stream);
        return launch_group_tile<XT>(a, group, stream);
    };
    return x_dtype == FQ_F16 ? with(std::integral_constant<int, FQ_F16>{}) : with(std::integral_constant<int, FQ_BF16>{});
}

}  // namespace fq
