// fq_linear_group_i4: 16-bit activations times 4-bit weights with group scales; up to 16 rows whose activations fit into LDS.
//
// Y[i,n] = sum over groups of s (sum x q) + b (sum x).  Codes enter the matrix product as 16-bit whole numbers (fq_linear_group.h), their sums stay in fp32
// and take the group's scale there.
// The call is the stream of its weights.  A workgroup goes through tiles of 16 columns; of each its waves have a stretch of the reduction, and their sums
// meet in LDS.  A wave takes steps of 128 columns, four ahead in registers, across the end of a tile: the next tile's weights travel while sums
// meet.  X lies in LDS, staged once for all tiles while the first weights are on their way.
// us (TB/s of weights and scales): one token bf16 4096 x 4096 4.2 (replayed from a graph, one launch 1.5 of them), 11008 x 4096 7.8 (2.9), 22016 x 8192
// 21 (4.4), 5 tokens fp16 with offsets 22016 x 8192 34 (3.0).  The vector pipe is busy for 50 % of the last one's cycles (some 80 instructions a step, 32 of them codes
// to numbers), the matrix pipe for 16 %; the rest is the waves' own chains, the last of 2.7 (5.4) rounds of tiles and the way to the first weights.
// Loads go by lane order: neighbouring lanes read neighbouring pieces, and lanes exchange them afterwards.  In the order that the matrix
// instruction wants, a load of 64 lanes is worked on lane by lane: the address unit was busy for 57 % of 18 us (16 rows, 11008 x 4096).
#include <algorithm>
#include <atomic>

#include "fq_internal.h"
#include "fq_linear_group.h"

namespace fq {
namespace {

// Steps in registers, a chunk.  Two chunks ahead are slower, as the loop that keeps two sets of registers apart is longer: 22016 x 8192, one row 23 us
// (21), 8 rows 29 (25), 5 of fp16 with offsets 40 (35).
constexpr int AHEAD = 4;

// Rows of X in LDS: 16 bytes more than whole steps, so that 16 rows are read from all banks
constexpr int x_pitch(int K) { return (K + 127) / 128 * 256 + 16; }
// Tiles' sums at once: with 16 waves one is what LDS has room for, and takes another barrier
constexpr int sums_of(int NW) { return NW == 8 ? 2 : 1; }

// Workgroup barrier that orders LDS only: loads stay in flight across it.
__device__ __forceinline__ void strip_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int XT, int NW, int GROUP, bool OFFSET>
__global__ __launch_bounds__(NW * 64) void linear_group_kernel(GroupProduct a)
{
    typedef GroupMma<XT> M_;
    typedef typename M_::v8 v8;
    constexpr int THREADS = NW * 64, SUMS = sums_of(NW);
    constexpr int PER = 128 / GROUP, EACH = 4 / PER;            // groups in a step of 128 columns, products (32 columns) in a group
    constexpr bool SURPLUS = OFFSET || M_::SURPLUS;             // codes as q + 24, which costs less where the activations' sum is there anyway
    extern __shared__ __align__(16) uint8_t lds[];
    v4f* red = reinterpret_cast<v4f*>(lds);                     // SUMS times [NW][64]
    uint8_t* x_lds = lds + SUMS * NW * 1024;
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // ---- a wave's stretch of steps ----
    const int steps = (a.K + 127) / 128;
    const int each = ((steps + NW - 1) / NW + 1) & ~1;          // even: two steps are a cache line of a row
    const int first = min(wave * each, steps), last = min(first + each, steps);
    // a lane's columns of a step in product j: 8 from x_col + x_next * j on
    constexpr bool TURN = GROUP != 128;                         // product j takes columns 32 j .. 32 j + 31, of one group
    constexpr int x_next = TURN ? 32 : 8;
    const int x_col = TURN ? 8 * c : 32 * c;

    // ---- what is loaded: lane l has piece l % 4 of the step of row l / 4 of a tile, and that row's scales of step l % 4 of a chunk ----
    const uint8_t* w_tile;
    uint32_t w_row;
    size_t g_row;
    auto begin_tile = [&](int tile) {
        const int row = min(lane / 4, a.N - 1 - 16 * tile);
        w_tile = a.Wq + (size_t)tile * 16 * (a.K / 2);
        w_row = (uint32_t)row * (a.K / 2);
        g_row = (size_t)(16 * tile + row) * a.groups;
    };
    v4u w[AHEAD];
    StepScales<PER> s_next, b_next = {};
    auto load_scales = [&](int k) {
        s_next = a.step_scales<PER>(a.S, g_row, (k + lane % 4) * PER);
        if (OFFSET) b_next = a.step_scales<PER>(a.B, g_row, (k + lane % 4) * PER);
    };
    // No branches around loads: where paths meet, the compiler has to wait as if the later ones had not been issued.  What lies behind a row's end is
    // read from its end; the activations there are zeros.
    auto load = [&](int d, int k) { w[d] = *reinterpret_cast<const v4u*>(w_tile + (w_row + min(64 * k + 16 * (lane % 4), a.K / 2 - 16))); };
    begin_tile(blockIdx.x);
    load_scales(first);
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(d, first + d);
    const int pitch = x_pitch(a.K), pieces = steps * 16;
    for (int i = threadIdx.x; i < a.M * pieces; i += THREADS) {
        const int m = i / pieces, p = i % pieces;
        v4u v = {0, 0, 0, 0};
        if (8 * p < a.K) v = *reinterpret_cast<const v4u*>(static_cast<const uint16_t*>(a.X) + (size_t)m * a.ldx + 8 * p);
        *reinterpret_cast<v4u*>(x_lds + m * pitch + 16 * p) = v;
    }
    strip_barrier();
    const uint8_t* x_at = x_lds + (r < a.M ? r : 0) * pitch + 2 * x_col;      // rows that there are not are row 0; they are not stored

    v4f acc;
    auto compute = [&](int d, int k, const float (&s)[PER], const float (&b)[PER]) {
        v4u codes;
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[j] = __shfl(w[d][j], 4 * r + c, 64);
        if (TURN) transpose_quarters(codes);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            v4f p = {0.0f, 0.0f, 0.0f, 0.0f}, sum = p;
#pragma unroll
            for (int j = EACH * g; j < EACH * (g + 1); ++j) {
                const v8 xf = *reinterpret_cast<const v8*>(x_at + 256 * k + 2 * x_next * j);
                p = M_::mul(xf, SURPLUS ? M_::widen24(codes[j]) : M_::widen(codes[j]), p);
                if (SURPLUS) sum = M_::mul(xf, M_::all(false), sum);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[e] = __builtin_fmaf(s[g], SURPLUS ? __builtin_fmaf(-24.0f, sum[e], p[e]) : p[e], acc[e]);
                if (OFFSET) acc[e] = __builtin_fmaf(b[g], sum[e], acc[e]);
            }
        }
    };
    // A chunk: its four steps, and the loads of the one after it: in the same tile, at the beginning of another, or none.
    // Scalar conditions: the matrix instruction ignores the execution mask.
    enum { SAME, AFTER, NO_MORE };
    auto chunk = [&](int k, int after, auto more) {
        constexpr int MORE = decltype(more)::value;
        const int next = MORE == SAME ? k + AHEAD : first;
        float s[AHEAD][PER], b[AHEAD][PER];
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                s[t][g] = a.scale_at(g, [&](int i) { return __shfl(s_next.v[i], 4 * r + t, 64); });
                b[t][g] = OFFSET ? a.scale_at(g, [&](int i) { return __shfl(b_next.v[i], 4 * r + t, 64); }) : 0.0f;
            }
        if (MORE == AFTER) begin_tile(after);
        if (MORE != NO_MORE) load_scales(next);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) {
            if (k + t < last) compute(t, k + t, s[t], b[t]);
            if (MORE != NO_MORE) load(t, next + t);
        }
    };
    int half = 0;
    for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int after = tile + gridDim.x;
        acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        int k = first;
        for (; k + AHEAD < last; k += AHEAD) chunk(k, 0, std::integral_constant<int, SAME>{});
        if (k < last) {
            if (after < a.tiles) chunk(k, after, std::integral_constant<int, AFTER>{});
            else chunk(k, 0, std::integral_constant<int, NO_MORE>{});
        }
        v4f* mine = red + half * (NW * 64);
        mine[wave * 64 + lane] = acc;
        strip_barrier();
        const float* sums = reinterpret_cast<const float*>(mine);
        if (threadIdx.x < 256) {
            const int m = threadIdx.x / 16, col = 16 * tile + threadIdx.x % 16;
            if (m < a.M && col < a.N) {
                const int at = (m / 4 * 16 + threadIdx.x % 16) * 4 + m % 4;
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < NW; ++i) v += sums[i * 256 + at];
                if (a.bias) v += a.bias[col];
                a.store(v, (size_t)m * a.ldy + col);
            }
        }
        // with two places these sums are read while the next tile's are written, whose barrier comes before this place is written again
        if (SUMS == 1) strip_barrier();
        else half ^= 1;
    }
}

template <int XT, int NW> int launch(GroupProduct a, int group, int wgs, hipStream_t stream)
{
    auto kern = a.B ? (group == 32 ? linear_group_kernel<XT, NW, 32, true> : group == 64 ? linear_group_kernel<XT, NW, 64, true> : linear_group_kernel<XT, NW, 128, true>)
                    : (group == 32 ? linear_group_kernel<XT, NW, 32, false> : group == 64 ? linear_group_kernel<XT, NW, 64, false> : linear_group_kernel<XT, NW, 128, false>);
    static std::atomic<unsigned long long> attr_set[6];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), 160 * 1024, attr_set[(group == 32 ? 0 : group == 64 ? 1 : 2) + (a.B ? 3 : 0)])) return rc;
    a.tiles_n = a.tiles = (a.N + 15) / 16;
    kern<<<(unsigned)std::min(a.tiles, wgs), NW * 64, sums_of(NW) * NW * 1024 + a.M * x_pitch(a.K), stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group-scaled layer launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

}  // namespace

// Two workgroups of eight waves a CU as long as X leaves them the room, one of sixteen up to nearly all of LDS (8 rows, 22016 x 8192:
// 25 us; the tiles 39 or more); else, and beyond 16 rows, the tiles of fq_linear_group_tile.hip.
int launch_linear_group(const void* X, int x_dtype, int M, int K, int ldx, const void* Wq, const void* S, const void* B, int s_dtype, int group, int N,
                        const float* bias, void* Y, int y_dtype, int ldy, hipStream_t stream)
{
    GroupProduct a = {};
    a.X = X; a.Wq = static_cast<const uint8_t*>(Wq); a.S = S; a.B = B; a.bias = bias; a.Y = Y;
    a.M = M; a.N = N; a.K = K; a.groups = (K + group - 1) / group; a.s_dtype = s_dtype; a.y_dtype = y_dtype;
    a.ldx = ldx; a.ldy = ldy;
    const int cus = compute_units();
    const long long x_bytes = (long long)M * x_pitch(K);
    auto with = [&](auto xt) -> int {
        constexpr int XT = decltype(xt)::value;
        if (M <= 16 && x_bytes <= 64 * 1024) return launch<XT, 8>(a, group, 2 * cus, stream);
        if (M <= 16 && x_bytes <= 144 * 1024) return launch<XT, 16>(a, group, cus, stream);
        return launch_group_tile<XT>(a, group, stream);
    };
    return x_dtype == FQ_F16 ? with(std::integral_constant<int, FQ_F16>{}) : with(std::integral_constant<int, FQ_BF16>{});
}

}  // namespace fq
