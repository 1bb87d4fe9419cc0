// fq_rms_norm_quant: residual addition, root-mean-square norm, and the flattened, per-tensor quantized activation.
//
// arXiv 2402.17985 Sec. 4.1 Eq. 3 and Sec. 2.1 Eq. 1 (flatten and quantize), applied to y = fl32(fl32(h t) gamma), t = 1 / rms(h).
// A workgroup takes a row at a time, a thread 16 consecutive channels of it, which stay in registers from the load to the
// codes; sums of squares are formed in float64, so that codes do not go by the order of a sum.  Workgroups stay for many
// rows: gamma, the map and its multipliers are read once, and the next row is on its way while this one is reduced.
// Slots that do not lie at their channel's own place (copies, other maps) read y out of LDS.
// A dynamic scale is a maximum over the whole tensor: a first pass stores h, every row's t and each workgroup's candidate, a
// second one forms y again and quantizes it.
#include <algorithm>
#include <atomic>

#include "fq_internal.h"
#include "fq_rows.h"

namespace fq {
namespace {

enum { ONE_PASS, FIND_SCALE, WITH_SCALE };
constexpr int TABLE = 256;        // multipliers m(n) kept for n < 256
constexpr int MAX_WGS = 1024;     // and candidates

struct Norm {
    const void *X, *R, *gamma;
    void *R_out, *Y;
    size_t ldx, ldr, ldro, ldy;
    int M, K, Kpad, g_dtype, y_dtype, bits, candidates;
    float eps;
    const int32_t *src, *rep;
    const float* absmax;
    uint8_t* out;
    float *s_x, *t, *found;
};

// Where channel j of the row lies in LDS: the four 16-byte pieces of a thread's channels are turned by its number, so that the threads of
// a wave write to all banks.
__device__ __forceinline__ int place(int j) { return (j & ~15) | ((((j >> 2) ^ (j >> 6)) & 3) << 2) | (j & 3); }

__device__ __forceinline__ void store_codes(int bits, const float (&x)[16], const float (&m)[16], uint8_t* out, int Kpad, size_t M, int row, int q)
{
    if (bits == 8) store_group<8>(quantize16<8>(x, m), out, Kpad, M, row, q);
    else if (bits == 4) store_group<4>(quantize16<4>(x, m), out, Kpad / 2, M, row, q);
    else store_group<6>(quantize16<6>(x, m), out, 0, M, row, q);
}

// The sum over the workgroup of a value of each thread; `part`: a place for every wave.  The barrier also ends what the workgroup did in LDS before.
__device__ __forceinline__ double sum_of(double v, double* part)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    const int waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    strip_barrier();
    double s = part[0];
    for (int w = 1; w < waves; ++w) s += part[w];
    return s;
}

// GPT: groups of 16 channels a thread has (channels 16 (tid + k threads) ..)
template <int XT, int RT, int PASS, int GPT>
__global__ __launch_bounds__(1024) void rms_norm_kernel(Norm a)
{
    extern __shared__ __align__(16) uint8_t lds[];
    double* part = reinterpret_cast<double*>(lds);                  // 16 waves
    float* best_of = reinterpret_cast<float*>(part + 16);           // 16 waves
    float* table = best_of + 16;                                    // m(n)
    float* row_y = table + TABLE;                                   // the row; behind it a zero
    const int tid = threadIdx.x, threads = blockDim.x, K = a.K, G = (K + 15) / 16, Q = a.out ? a.Kpad / 16 : 0;
    const int zero_at = 16 * G;

    Raw<XT> x[GPT];
    Raw<RT> r[GPT];
    auto fetch = [&](int row) {
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g < G) {
                x[k] = load_raw<XT>(a.X, (size_t)row * a.ldx, g, K);
                r[k] = load_raw<RT>(a.R, (size_t)row * a.ldr, g, K);
            }
        }
    };
    fetch(blockIdx.x);

    // ---- the bound and the multipliers ----
    float bound = 0.0f;
    if (PASS != FIND_SCALE && Q) {
        if (PASS == ONE_PASS) {
            bound = *a.absmax;
            if (!(bound >= 0.0f) || bound > 3.0e38f) bound = 0.0f;     // negative / NaN / Inf static bound: treated as 0
        } else {
            for (int i = tid; i < a.candidates; i += threads) bound = fmaxf(bound, a.found[i]);
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) bound = fmaxf(bound, __shfl_xor(bound, off, 64));
            if ((tid & 63) == 0) best_of[tid >> 6] = bound;
            __syncthreads();
            bound = best_of[0];
            for (int w = 1; w < threads >> 6; ++w) bound = fmaxf(bound, best_of[w]);
        }
        const double qmax = a.bits == 8 ? 127.0 : 7.0;
        for (int n = tid; n < TABLE; n += threads) table[n] = (n > 0 && bound != 0.0f) ? (float)(qmax / ((double)n * (double)bound)) : 0.0f;
        if (blockIdx.x == 0 && tid == 0) *a.s_x = bound == 0.0f ? 1.0f : (float)((double)bound / qmax);
        __syncthreads();
    }
    auto multiplier = [&](int n) -> float {
        if (n <= 0 || bound == 0.0f) return 0.0f;
        return n < TABLE ? table[n] : (float)((a.bits == 8 ? 127.0 : 7.0) / ((double)n * (double)bound));
    };

    // ---- the map: slots of the thread's own channels, where they lie at their own place, and the others ----
    float gamma[GPT][16], m[GPT][16];
    bool own[GPT];
    int first_other = 0;      // the thread's first group of slots that is not its own
#pragma unroll
    for (int k = 0; k < GPT; ++k) {
        const int g = tid + k * threads;
        own[k] = false;
        if (g < G) {
            load_any(a.gamma, a.g_dtype, g, K, gamma[k]);
            if (g < Q) {
                int s[16], n[16];
                load8(a.src + 16 * g, s);
                load8(a.src + 16 * g + 8, s + 8);
                load8(a.rep + 16 * g, n);
                load8(a.rep + 16 * g + 8, n + 8);
                own[k] = 16 * g + 16 <= K;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    own[k] = own[k] && s[i] == 16 * g + i;
                    m[k][i] = PASS == FIND_SCALE ? (n[i] > 0 ? (float)n[i] : 0.0f) : multiplier(n[i]);
                    if (PASS == FIND_SCALE && n[i] > (1 << 24)) own[k] = false;      // not a whole number in fp32
                }
            }
        }
        if (own[k] && first_other == k) first_other = k + 1;
    }
    // any slot group that is not its thread's own
    bool others = false;
    for (int k = 0, q = tid; q < Q; ++k, q += threads) others = others || k >= GPT || !own[k < GPT ? k : 0];
    const bool gathers = __syncthreads_or(others);
    if (gathers && tid == 0) row_y[zero_at] = 0.0f;

    float most[GPT][16], quotient = 0.0f;
    if (PASS == FIND_SCALE) {
#pragma unroll
        for (int k = 0; k < GPT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) most[k][i] = 0.0f;
    }

    for (int row = blockIdx.x; row < a.M; row += gridDim.x) {
        float y[GPT][16];
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g >= G) continue;
            widen<XT>(x[k], y[k]);
            if constexpr (RT != NONE) {
                float add[16];
                widen<RT>(r[k], add);
#pragma unroll
                for (int i = 0; i < 16; ++i) y[k][i] = y[k][i] + add[i];
                const Raw<RT> h = narrow<RT>(y[k]);
                store_raw<RT>(h, a.R_out, (size_t)row * a.ldro, g, K);
                widen<RT>(h, y[k]);
            }
            if (PASS != WITH_SCALE) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = __builtin_fma((double)y[k][i], (double)y[k][i], sum);
            }
        }
        if (row + (int)gridDim.x < a.M) fetch(row + gridDim.x);
        float t;
        if (PASS == WITH_SCALE) {
            t = a.t[row];
            if (gathers) strip_barrier();          // the row before is read no more
        } else {
            t = (float)(1.0 / sqrt(sum_of(sum, part) / (double)K + (double)a.eps));
            if (PASS == FIND_SCALE && tid == 0) a.t[row] = t;
        }
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g >= G) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) y[k][i] = y[k][i] * t * gamma[k][i];
            if (PASS != FIND_SCALE && a.Y) store_any(y[k], a.Y, a.y_dtype, (size_t)row * a.ldy, g, K);
            if (gathers) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) *reinterpret_cast<v4f*>(row_y + place(16 * g + i)) = v4f{y[k][i], y[k][i + 1], y[k][i + 2], y[k][i + 3]};
            }
            if (own[k]) {
                if (PASS == FIND_SCALE) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) most[k][i] = fmaxf(most[k][i], fabsf(y[k][i]));
                } else {
                    store_codes(a.bits, y[k], m[k], a.out, a.Kpad, a.M, row, g);
                }
            }
        }
        if (!gathers) {
            if (PASS != WITH_SCALE) strip_barrier();      // part is read no more
            continue;
        }
        strip_barrier();
        for (int k = first_other, q = tid + first_other * threads; q < Q; ++k, q += threads) {
            if (k < GPT && own[k < GPT ? k : 0]) continue;
            int s[16], n[16];
            load8(a.src + 16 * q, s);
            load8(a.src + 16 * q + 8, s + 8);
            load8(a.rep + 16 * q, n);
            load8(a.rep + 16 * q + 8, n + 8);
            float v[16], by[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool used = (unsigned)s[i] < (unsigned)K && n[i] > 0;
                v[i] = row_y[used ? place(s[i]) : zero_at];
                if (PASS == FIND_SCALE) quotient = fmaxf(quotient, used ? (n[i] == 1 ? fabsf(v[i]) : (float)((double)fabsf(v[i]) / (double)n[i])) : 0.0f);
                else by[i] = multiplier(n[i]);
            }
            if (PASS != FIND_SCALE) store_codes(a.bits, v, by, a.out, a.Kpad, a.M, row, q);
        }
    }

    if (PASS == FIND_SCALE) {
#pragma unroll
        for (int k = 0; k < GPT; ++k)
            if (own[k]) {
#pragma unroll
                for (int i = 0; i < 16; ++i) quotient = fmaxf(quotient, m[k][i] > 0.0f ? (float)((double)most[k][i] / (double)m[k][i]) : 0.0f);
            }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) quotient = fmaxf(quotient, __shfl_xor(quotient, off, 64));
        __syncthreads();
        if ((tid & 63) == 0) best_of[tid >> 6] = quotient;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < threads >> 6; ++w) quotient = fmaxf(quotient, best_of[w]);
            a.found[blockIdx.x] = quotient;
        }
    }
}

template <int XT, int RT, int PASS> int launch(const Norm& a, int wgs, hipStream_t stream)
{
    const int G = (a.K + 15) / 16, threads = std::min(1024, (G + 63) / 64 * 64);
    const int smem = 16 * 8 + 16 * 4 + TABLE * 4 + (16 * G + 16) * 4;
    auto kern = G <= 1024 ? rms_norm_kernel<XT, RT, PASS, 1> : rms_norm_kernel<XT, RT, PASS, 2>;
    static std::atomic<unsigned long long> attr_set[2];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), 136 * 1024, attr_set[G <= 1024 ? 0 : 1])) return rc;
    kern<<<(unsigned)wgs, threads, smem, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FQ_ERR_HIP, "norm launch failed: %s", hipGetErrorString(e));
    return FQ_OK;
}

template <int PASS> int launch_types(const Norm& a, int x_dtype, int r_dtype, int wgs, hipStream_t stream)
{
    if (PASS == WITH_SCALE) r_dtype = NONE;
    auto with = [&](auto xt) -> int {
        constexpr int XT = decltype(xt)::value;
        if constexpr (PASS != WITH_SCALE) {
            if (r_dtype == FQ_F32) return launch<XT, FQ_F32, PASS>(a, wgs, stream);
            if (r_dtype == FQ_F16) return launch<XT, FQ_F16, PASS>(a, wgs, stream);
            if (r_dtype == FQ_BF16) return launch<XT, FQ_BF16, PASS>(a, wgs, stream);
        }
        return launch<XT, NONE, PASS>(a, wgs, stream);
    };
    switch (x_dtype) {
    case FQ_F32: return with(std::integral_constant<int, FQ_F32>{});
    case FQ_F16: return with(std::integral_constant<int, FQ_F16>{});
    default: return with(std::integral_constant<int, FQ_BF16>{});
    }
}

}  // namespace

// every row's t, and a candidate for the bound from each workgroup
size_t rms_norm_workspace(int M) { return round_up((size_t)M * 4, 16) + MAX_WGS * 4; }

int launch_rms_norm_quant(const void* X, int x_dtype, int M, int K, int ldx, const void* R, int r_dtype, int ldr, void* R_out, int ldro,
                          const void* gamma, int g_dtype, float eps, void* Y, int y_dtype, int ldy, const int32_t* src, const int32_t* rep,
                          int Kpad, int bits, const float* absmax_in, void* Xq_out, float* s_x_out, void* workspace, hipStream_t stream)
{
    Norm a = {};
    a.X = X; a.R = R; a.gamma = gamma; a.R_out = R_out; a.Y = Y;
    a.ldx = ldx; a.ldr = ldr; a.ldro = ldro; a.ldy = ldy;
    a.M = M; a.K = K; a.Kpad = Kpad; a.g_dtype = g_dtype; a.y_dtype = y_dtype; a.bits = bits; a.eps = eps;
    a.src = src; a.rep = rep; a.absmax = absmax_in; a.out = static_cast<uint8_t*>(Xq_out); a.s_x = s_x_out;
    const int wgs = std::min(M, MAX_WGS), rt = R ? r_dtype : NONE;
    if (!Xq_out || absmax_in) return launch_types<ONE_PASS>(a, x_dtype, rt, wgs, stream);
    a.t = static_cast<float*>(workspace);
    a.found = a.t + round_up((size_t)M * 4, 16) / 4;
    a.candidates = wgs;
    if (int rc = launch_types<FIND_SCALE>(a, x_dtype, rt, wgs, stream)) return rc;
    if (R) {        // the second pass reads what the first one stored
        a.X = R_out;
        a.ldx = ldro;
        x_dtype = r_dtype;
    }
    return launch_types<WITH_SCALE>(a, x_dtype, NONE, wgs, stream);
}

}  // namespace fq
