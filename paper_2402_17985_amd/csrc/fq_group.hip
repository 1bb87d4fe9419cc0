// 4-bit weights with a scale (and an offset) for each row and group of columns: fq_group_weights_i4 makes them.
//
// w ~ s q + b over 32, 64 or 128 columns.  A lane takes 16 columns, 2 to 8 neighbouring lanes a group; least and largest element
// are exchanged between them, so that the weights are read once and stay in registers.
// Bound by bytes: 4096 x 4096 bf16 9.0 us (4.7 TB/s read and written), 11008 x 4000 fp32 with offsets 38 (5.2).
#include "fq_internal.h"
#include "fq_rows.h"

namespace fq {
namespace {

constexpr int THREADS = 256;

// v >= 0 or any finite v rounded to the type, at most its largest finite value
__device__ __forceinline__ float rounded(float v, int dtype)
{
    if (dtype == FQ_F16) return __builtin_amdgcn_fmed3f((float)(_Float16)v, -65504.0f, 65504.0f);
    if (dtype == FQ_BF16) return __builtin_amdgcn_fmed3f((float)(__bf16)v, -0x1.fep127f, 0x1.fep127f);
    return __builtin_amdgcn_fmed3f(v, -0x1.fffffep127f, 0x1.fffffep127f);
}
__device__ __forceinline__ void store_one(float v, void* base, int dtype, size_t at)
{
    if (dtype == FQ_F32) static_cast<float*>(base)[at] = v;
    else if (dtype == FQ_F16) static_cast<_Float16*>(base)[at] = (_Float16)v;
    else static_cast<__bf16*>(base)[at] = (__bf16)v;
}

// LANES lanes a group; a row has `units` lanes, whole groups
template <int DT, int LANES, bool OFFSET>
__global__ __launch_bounds__(THREADS) void group_weights_kernel(const void* __restrict__ W, unsigned total, int K, size_t ldw, unsigned units,
                                                                uint8_t* __restrict__ Wq, void* __restrict__ S, void* __restrict__ B, int s_dtype)
{
    const unsigned at = blockIdx.x * THREADS + threadIdx.x, row = min(at, total - 1) / units, unit = min(at, total - 1) % units;
    const bool mine = at < total && 16 * (int)unit < K;      // K is a multiple of 32: all 16 columns or none
    float w[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float part[8];
        widen<DT>(mine ? load_raw<DT, false>(row_of(W, ldw, element_bytes<DT>(), row), 2 * unit + h, K) : Raw<DT>{}, part);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[8 * h + i] = part[i];
    }
    float lo = __builtin_inff(), hi = -__builtin_inff();
    if (mine) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            lo = fminf(lo, w[i]);
            hi = fmaxf(hi, w[i]);
        }
    }
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, off, 64));
        hi = fmaxf(hi, __shfl_xor(hi, off, 64));
    }
    float s = rounded(OFFSET ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f, s_dtype);
    if (s < 0x1p-126f) s = 0.0f;
    const float b = OFFSET ? rounded(lo + 8.0f * s, s_dtype) : 0.0f, turn = s > 0.0f ? 1.0f / s : 0.0f;
    if (!mine) return;
    float m[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (OFFSET) w[i] = w[i] - b;
        m[i] = turn;
    }
    store16<4>(quantize16<4>(w, m), Wq + (size_t)row * (K / 2) + 8 * unit);
    if (unit % LANES == 0) {
        const size_t place = (size_t)row * (units / LANES) + unit / LANES;
        store_one(s, S, s_dtype, place);
        if (OFFSET) store_one(b, B, s_dtype, place);
    }
}

}  // namespace

int launch_group_weights(const void* W, int w_dtype, int N, int K, int ldw, int group, void* Wq, void* S, void* B, int s_dtype, hipStream_t stream)
{
    const unsigned units = (unsigned)((K + group - 1) / group * (group / 16)), total = units * (unsigned)N;
    auto go = [&](auto dt, auto lanes) {
        constexpr int DT = decltype(dt)::value, LANES = decltype(lanes)::value;
        auto kern = B ? group_weights_kernel<DT, LANES, true> : group_weights_kernel<DT, LANES, false>;
        kern<<<(total + THREADS - 1) / THREADS, THREADS, 0, stream>>>(W, total, K, (size_t)ldw, units, static_cast<uint8_t*>(Wq), S, B, s_dtype);
    };
    auto with = [&](auto dt) {
        if (group == 32) go(dt, std::integral_constant<int, 2>{});
        else if (group == 64) go(dt, std::integral_constant<int, 4>{});
        else go(dt, std::integral_constant<int, 8>{});
    };
    if (w_dtype == FQ_F32) with(std::integral_constant<int, FQ_F32>{});
    else if (w_dtype == FQ_F16) with(std::integral_constant<int, FQ_F16>{});
    else with(std::integral_constant<int, FQ_BF16>{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "group weights launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

}  // namespace fq
