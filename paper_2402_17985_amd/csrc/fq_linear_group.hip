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

#include "fq_internal.h"
#include "fq_linear_group.h"

namespace fq {
namespace {

constexpr int NW = 8, THREADS = NW * 64;

template <int XT, int MT, int GROUP, bool OFFSET, int D>
__global__ __launch_bounds__(THREADS) void linear_group_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int PER = 128 / GROUP;                            // groups in a step of 128 columns
    constexpr bool SUMS = OFFSET || XT == FQ_BF16;              // sum x is wanted
    __shared__ v4f red[NW][MT][64];
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile_n = blockIdx.x % a.tiles_n, tile_m = blockIdx.x / a.tiles_n;
    const int n0 = tile_n * 16, m0 = tile_m * 16 * MT, n = min(n0 + r, a.N - 1);
    const uint8_t* w_row = a.Wq + (size_t)n * (a.K / 2) + 16 * c;
    const size_t g_row = (size_t)n * a.groups;
    const uint16_t* x_row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x_row[i] = static_cast<const uint16_t*>(a.X) + (size_t)min(m0 + 16 * i + r, a.M - 1) * a.ldx;
    // a lane's columns of a step in product d: 8 from x_col + x_next * d on
    constexpr int x_next = GROUP == 128 ? 8 : 32;
    const int x_col = GROUP == 128 ? 32 * c : 8 * c;

    // ---- steps: 128 columns; the wave takes pairs of them in turn with the others ----
    const int whole = a.K / 128, steps = (a.K + 127) / 128;
    const int pairs = (steps + 1) / 2, my_pairs = (pairs - wave + NW - 1) / NW;
    // the last pair may have one step only
    const int mine = __builtin_amdgcn_readfirstlane(wave < pairs ? 2 * my_pairs - (steps % 2 != 0 && (pairs - 1) % NW == wave ? 1 : 0) : 0);
    auto step_of = [&](int t) -> int { return 2 * (wave + NW * (t >> 1)) + (t & 1); };
    v4u w[D], x[D][MT][4];
    float s[D][PER], b[D][PER];
    auto scales = [&](int d, int k) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const size_t at = g_row + min(k * PER + j, a.groups - 1);
            s[d][j] = a.scale(a.S, at);
            b[d][j] = OFFSET ? a.scale(a.B, at) : 0.0f;
        }
    };
    auto load = [&](int d, int t) {
        const int k = step_of(t);
        w[d] = *reinterpret_cast<const v4u*>(w_row + (size_t)k * 64);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[d][i][j] = *reinterpret_cast<const v4u*>(x_row[i] + 128 * k + x_col + x_next * j);
        scales(d, k);
    };
    // a step that may go beyond the row's end: activations there are zeros, whatever the codes are
    auto load_last = [&](int d, int t) {
        const int k = step_of(t);
        if (k < whole) {
            load(d, t);
            return;
        }
        w[d] = v4u{0, 0, 0, 0};
        if (64 * k + 16 * c < a.K / 2) w[d] = *reinterpret_cast<const v4u*>(w_row + (size_t)k * 64);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = 128 * k + x_col + x_next * j;
                x[d][i][j] = v4u{0, 0, 0, 0};
                if (col < a.K) x[d][i][j] = *reinterpret_cast<const v4u*>(x_row[i] + col);
            }
        scales(d, k);
    };
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto compute = [&](int d) {
        v4u codes = w[d];
        if (GROUP != 128) transpose_quarters(codes);
        v4f p[MT], q[MT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool first = j % (4 / PER) == 0, last = (j + 1) % (4 / PER) == 0;
            const v8 wf = M_::widen(codes[j]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const v8 xf = M_::activations(x[d][i][j]);
                const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
                p[i] = M_::mul(xf, wf, first ? zero : p[i]);
                if (SUMS) q[i] = M_::mul(xf, M_::ones(), first ? zero : q[i]);
                if (last) {
                    const float sc = s[d][j / (4 / PER)], of = b[d][j / (4 / PER)] - (XT == FQ_BF16 ? 24.0f * sc : 0.0f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[i][e] = __builtin_fmaf(sc, p[i][e], acc[i][e]);
                        if (SUMS) acc[i][e] = __builtin_fmaf(of, q[i][e], acc[i][e]);
                    }
                }
            }
        }
    };
    // rounds of D steps, then the rest with scalar conditions: the matrix instruction ignores the execution mask
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < mine) load_last(d, d);
    int t = 0;
    for (; t + 2 * D < mine; t += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            compute(d);
            load(d, t + D + d);
        }
    }
    const int left = __builtin_amdgcn_readfirstlane(mine - t);     // at most 2 D, the first D of them loaded
#pragma unroll
    for (int d = 0; d < D; ++d) {
        if (d < left) compute(d);
        if (D + d < left) load_last(d, t + D + d);
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (D + d < left) compute(d);

#pragma unroll
    for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
    __syncthreads();
    const float* sums = reinterpret_cast<const float*>(red);
    for (int e = threadIdx.x; e < MT * 256; e += THREADS) {
        const int m = m0 + e / 16, col = n0 + e % 16;
        if (m >= a.M || col >= a.N) continue;
        const int row = e / 16 % 16, at = (e / 256 * 64 + row / 4 * 16 + e % 16) * 4 + row % 4;
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < NW; ++i) v += sums[i * MT * 256 + at];
        if (a.bias) v += a.bias[col];
        a.store(v, (size_t)m * a.ldy + col);
    }
}

template <int XT, int MT, int D> void launch(const GroupProduct& a, int group, hipStream_t stream)
{
    auto kern = a.B ? (group == 32 ? linear_group_kernel<XT, MT, 32, true, D> : group == 64 ? linear_group_kernel<XT, MT, 64, true, D> : linear_group_kernel<XT, MT, 128, true, D>)
                    : (group == 32 ? linear_group_kernel<XT, MT, 32, false, D> : group == 64 ? linear_group_kernel<XT, MT, 64, false, D> : linear_group_kernel<XT, MT, 128, false, D>);
    kern<<<(unsigned)(a.tiles_n * ((a.M + 16 * MT - 1) / (16 * MT))), THREADS, 0, stream>>>(a);
}

}  // namespace

int launch_linear_group(const void* X, int x_dtype, int M, int K, int ldx, const void* Wq, const void* S, const void* B, int s_dtype, int group, int N,
                        const float* bias, void* Y, int y_dtype, int ldy, hipStream_t stream)
{
    GroupProduct a = {};
    a.X = X; a.Wq = static_cast<const uint8_t*>(Wq); a.S = S; a.B = B; a.bias = bias; a.Y = Y;
    a.M = M; a.N = N; a.K = K; a.groups = (K + group - 1) / group; a.s_dtype = s_dtype; a.y_dtype = y_dtype;
    a.ldx = ldx; a.ldy = ldy; a.tiles_n = (N + 15) / 16;
    auto with = [&](auto xt) {
        constexpr int XT = decltype(xt)::value;
        if (M <= 16) launch<XT, 1, 4>(a, group, stream);
        else if (M <= 32) launch<XT, 2, 2>(a, group, stream);
        else launch<XT, 4, 2>(a, group, stream);
    };
    if (x_dtype == FQ_F16) with(std::integral_constant<int, FQ_F16>{});
    else with(std::integral_constant<int, FQ_BF16>{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group-scaled layer launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

}  // namespace fq
