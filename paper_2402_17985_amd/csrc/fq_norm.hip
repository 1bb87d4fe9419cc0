// fq_rms_norm_quant: residual addition, root-mean-square norm, and the flattened, per-tensor quantized activation.
//
// arXiv 2402.17985 Sec. 4.1 Eq. 3 and Sec. 2.1 Eq. 1 (flatten and quantize), applied to y = fl32(fl32(h t) gamma), t = 1 / rms(h).
// A workgroup takes a row at a time, a thread two pieces (four of rows beyond 16384 channels) of eight channels of it, as many pieces apart as there are
// threads, which stay in registers from the load to the codes; sums of squares are formed in float64, so that codes do not go by the order of a sum.  Workgroups stay for many
// rows: gamma, the map and its multipliers are read once, and the next row is on its way while this one is reduced.
// Slots that do not lie at their channel's own place (copies, padding, other maps) are worked on one by one, neighbouring threads neighbouring slots, from
// the row in LDS; their codes meet there by sixteens.
// A dynamic scale is a maximum over the whole tensor: a first pass stores h, every row's t and each workgroup's candidate, a
// second one forms y again and quantizes it.  One workgroup does both for a row or two.
// Bound by bytes: bf16 with a residual, static, 8192 x 4096 55 us (4.4 TB/s read and written), 8192 x 8192 102 (4.8), fp32 8192 x 4096 92 (4.8): the rate of
// a copy.  Dynamic 8192 x 4096: 45 and 32 us in the two kernels, 4.4 and 3.3 TB/s.  4099 x 5003 with an fp32 residual, bf16 out: 98 (2.9 TB/s).
// Nibbles, static and dynamic 8192 x 4096: 51 and 72 us.  E3M2 storage packs codes by sixteens, which no thread has: every slot goes one by one through LDS,
// 105 and 181 us, one row of 4096 20, 48 x 5120 static 11.
// One row of 4096, dynamic: 10 us, 48 x 5120 static 7: latency (the map, the row, two or three reductions over the workgroup).
// Sixteen consecutive channels to a thread, two loads of 32-byte strides, kept the address unit busy lane by lane (dynamic 8192 x 4096, both kernels: 94 us, against 72
// with pieces of eight at that time).
#include <algorithm>
#include <atomic>

#include "fq_internal.h"
#include "fq_rows.h"
#include "fq_rules.h"

namespace fq {
namespace {

enum { ONE_PASS, FIND_SCALE, WITH_SCALE, BOTH };
constexpr int TABLE = 256;        // multipliers m(n) kept for n < 256
constexpr int ALONE = 2;          // rows that one workgroup takes
constexpr int ALONE_PLACES = 4;   // of their t in LDS: what follows begins at a multiple of 16 bytes
static_assert(ALONE <= ALONE_PLACES && (16 + ALONE_PLACES + TABLE) % 4 == 0, "LDS");
constexpr int KEPT = 4;           // slots away from their channel's place that a thread keeps in registers

// floats of LDS for a row of K, and the zero behind it
__host__ __device__ constexpr int row_places(int K) { return (K + 7) / 8 * 8 + 8; }

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

__device__ __forceinline__ float largest_of(float v, float* part)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < (int)blockDim.x >> 6; ++w) v = fmaxf(v, part[w]);
    return v;
}

// 1 / sqrt(v) in float64: the hardware's estimate and two steps of Newton's iteration.  Its few last bits off do not reach fp32 but next to a tie.
__device__ __forceinline__ double inverse_root(double v)
{
    double y = __builtin_amdgcn_rsq(v);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = __builtin_fma(0.5 * y, __builtin_fma(-v * y, y, 1.0), y);
    return y;
}

__device__ __forceinline__ float share(float v, int n) { return n == 1 ? fabsf(v) : (float)((double)fabsf(v) / (double)n); }

// The largest fl32(|v| / n) seen: quotients are compared by cross multiplication in float64 (exact for n < 2^29) and divided once; rounding is monotonic.
struct Largest {
    float value = 0.0f, other = 0.0f;
    int n = 1;
    __device__ __forceinline__ void see(float v, int copies)
    {
        v = fabsf(v);
        if (copies >= (1 << 29)) {
            other = fmaxf(other, share(v, copies));
        } else if ((double)v * (double)n > (double)value * (double)copies) {
            value = v;
            n = copies;
        }
    }
    __device__ __forceinline__ float get() const { return fmaxf(other, share(value, n)); }
};

// 16 codes, one per byte
__device__ __forceinline__ void store_packed(int bits, const v4u& q, uint8_t* out, int Kpad, size_t M, int row, int g)
{
    if (bits == 8) store_group<8>(q, out, Kpad, M, row, g);
    else if (bits == 4) store_group<4>(q, out, Kpad / 2, M, row, g);
    else store_group<6>(v4u{e3m2_codes(q[0]), e3m2_codes(q[1]), e3m2_codes(q[2]), e3m2_codes(q[3])}, out, 0, M, row, g);
}
// 8 elements to INT8 or nibbles at slot 8 g of a row
__device__ __forceinline__ void store_eight(int bits, const float (&y)[8], const float* m, uint8_t* out, int Kpad, int row, int g)
{
    if (bits == 8) {
        *reinterpret_cast<v2u*>(out + (size_t)row * Kpad + (uint32_t)(8 * g)) = v2u{quantize4<8>(y, m), quantize4<8>(y + 4, m + 4)};
    } else {
        const uint32_t a = quantize4<4>(y, m), b = quantize4<4>(y + 4, m + 4);
        const uint32_t c = (a & 0x000f000fu) | ((a >> 4) & 0x00f000f0u), d = (b & 0x000f000fu) | ((b >> 4) & 0x00f000f0u);      // bytes 0 and 2: two values each
        *reinterpret_cast<uint32_t*>(out + (size_t)row * (Kpad / 2) + (uint32_t)(4 * g)) = bytes_of(d, c, 0x06040200u);
    }
}

// A thread has GPT times 8 channels, 8 (tid + k threads) on: neighbouring threads read neighbouring pieces.  KEEP: gamma stays in registers, the multipliers of the
// channels' own slots in LDS (in registers, too, the kernel spilled at the 128 that four waves a SIMD leave it).
template <int XT, int RT, int PASS, int GPT, bool RAGGED>
__global__ __launch_bounds__(1024) void rms_norm_kernel(Norm a)
{
    constexpr bool KEEP = GPT <= 2, FIND = PASS == FIND_SCALE || PASS == BOTH;
    constexpr int HT = RT == NONE ? XT : RT;                        // h as it is stored
    extern __shared__ __align__(16) uint8_t lds[];
    double* part = reinterpret_cast<double*>(lds);                  // 16 waves
    float* best_of = reinterpret_cast<float*>(part + 16);           // 16 waves
    float* few_t = best_of + 16;                                    // t of a few rows
    float* table = few_t + ALONE_PLACES;                         // m(n)
    const int tid = threadIdx.x, threads = blockDim.x, K = a.K, G = (K + 7) / 8, Kpad = a.out ? a.Kpad : 0;
    const int zero_at = 8 * G;
    float* row_y = table + TABLE;                                   // the row; behind it a zero
    uint8_t* row_q = reinterpret_cast<uint8_t*>(row_y + row_places(K));     // codes of 16 slots a thread
    float* row_m = reinterpret_cast<float*>(row_q + 16 * threads);          // KEEP: multipliers of the slots before `base`
    const double per_channel = 1.0 / (double)K;

    Raw<XT> x[GPT];
    Raw<RT> r[GPT];
    auto fetch = [&](int row) {
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g < G) {
                x[k] = load_raw<XT, RAGGED>(row_of(a.X, a.ldx, element_bytes<XT>(), row), g, K);
                r[k] = load_raw<RT, RAGGED>(row_of(a.R, a.ldr, element_bytes<RT>(), row), g, K);
            }
        }
    };
    fetch(blockIdx.x);
    float kept_gamma[KEEP ? GPT : 1][8];
    if constexpr (KEEP) {
#pragma unroll
        for (int k = 0; k < GPT; ++k)
            if (tid + k * threads < G) load_any<RAGGED>(a.gamma, a.g_dtype, tid + k * threads, K, kept_gamma[k]);
    }
    auto normalise = [&](int k, float t, float (&y)[8]) {           // y holds h
        float other[8];
        if constexpr (!KEEP) load_any<RAGGED>(a.gamma, a.g_dtype, tid + k * threads, K, other);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * t * (KEEP ? kept_gamma[KEEP ? k : 0][i] : other[i]);
    };

    // ---- the map: do the first slots lie at their channels' own places?  The slots from `base` on are the others.  (E3M2 codes are packed by sixteens: all.) ----
    const int whole = KEEP && a.bits != FQ_BITS_I4_E3M2 ? min(K & ~15, Kpad) : 0;
    int other_src[KEPT], other_rep[KEPT];      // the first of the others that this thread works on, if they begin at `whole`: on their way while the row is
    auto load_others = [&](int base) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            const int p = base + i * threads + tid;
            other_src[i] = p < Kpad ? a.src[p] : -1;
            other_rep[i] = p < Kpad ? a.rep[p] : 0;
        }
    };
    load_others(whole);
    int own_rep[KEEP ? GPT : 1][8];
    bool apart = false, far = false;     // far: copy counts that the table does not have
    if constexpr (KEEP) {
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int at = 8 * (tid + k * threads);
            if (at < whole) {
                int src[8];
                load8(a.src + at, src);
                load8(a.rep + at, own_rep[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    apart |= src[i] != at + i;
                    far |= own_rep[k][i] >= TABLE;
                }
            }
        }
    }
    const int base = __syncthreads_or(apart) ? 0 : whole;
    if (PASS != FIND_SCALE) far = __syncthreads_or(far);
    if (base != whole) load_others(base);
    const bool others = base < Kpad;
    auto own = [&](int k) { return 8 * (tid + k * threads) < base; };
    // In search of the bound a slot counts nothing that another slot of the same channel, at its own place and with no more copies, has counted.
    bool to_count = false;
    auto used = [&](int src, int rep) { return (unsigned)src < (unsigned)K && rep > 0; };
    if (FIND) {
        auto counts = [&](int j, int n) {
            if (!used(j, n)) return false;
            const int own = j < base ? a.rep[j] : 0;
            return own <= 0 || own > n;
        };
#pragma unroll
        for (int i = 0; i < KEPT; ++i) to_count |= counts(other_src[i], other_rep[i]);
        for (int p = base + KEPT * threads + tid; p < Kpad; p += threads) to_count |= counts(a.src[p], a.rep[p]);
        to_count = __syncthreads_or(to_count);
    }
    if (tid == 0) row_y[zero_at] = 0.0f;
    auto to_lds = [&](int g, const float (&y)[8]) {
        *reinterpret_cast<v4f*>(row_y + 8 * g) = v4f{y[0], y[1], y[2], y[3]};
        *reinterpret_cast<v4f*>(row_y + 8 * g + 4) = v4f{y[4], y[5], y[6], y[7]};
    };

    // h of a row from what fetch() brought, and the sum of its squares
    auto residual = [&](int row, float (&y)[GPT][8], double& sum) {
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g >= G) continue;
            widen<XT>(x[k], y[k]);
            if constexpr (RT != NONE) {
                float add[8];
                widen<RT>(r[k], add);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[k][i] = y[k][i] + add[i];
                const Raw<RT> h = narrow<RT>(y[k]);
                store_raw<RT, RAGGED>(h, row_of(a.R_out, a.ldro, element_bytes<RT>(), row), g, K);
                widen<RT>(h, y[k]);
            }
            if (PASS != WITH_SCALE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)y[k][i], (double)y[k][i], sum);
            }
        }
        if (row + (int)gridDim.x < a.M) fetch(row + gridDim.x);
    };
    auto inverse_rms = [&](double sum) -> float { return (float)inverse_root(__builtin_fma(sum_of(sum, part), per_channel, (double)a.eps)); };

    // ---- the bound ----
    float bound = 0.0f;
    if constexpr (FIND) {
        float most[GPT][8];
        Largest largest;
#pragma unroll
        for (int k = 0; k < GPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) most[k][i] = 0.0f;
        for (int row = blockIdx.x; row < a.M; row += gridDim.x) {
            float y[GPT][8];
            double sum = 0.0;
            residual(row, y, sum);
            const float t = inverse_rms(sum);
            if (tid == 0) {
                if (PASS == BOTH) few_t[row] = t;
                else a.t[row] = t;
            }
#pragma unroll
            for (int k = 0; k < GPT; ++k) {
                const int g = tid + k * threads;
                if (g >= G) continue;
                normalise(k, t, y[k]);
                if (to_count) to_lds(g, y[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) most[k][i] = fmaxf(most[k][i], fabsf(y[k][i]));
            }
            strip_barrier();
            if (!to_count) continue;
            for (int p = base + tid; p < Kpad; p += threads) {
                const int j = a.src[p], n = a.rep[p];
                if (used(j, n)) largest.see(row_y[j], n);
            }
        }
        if constexpr (KEEP) {
#pragma unroll
            for (int k = 0; k < GPT; ++k)
                if (own(k)) {
                    if (PASS != BOTH) load8(a.rep + 8 * (tid + k * threads), own_rep[k]);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (own_rep[k][i] > 0) largest.see(most[k][i], own_rep[k][i]);
                }
        }
        bound = largest_of(largest.get(), best_of);
        if (PASS == FIND_SCALE) {
            if (tid == 0) a.found[blockIdx.x] = bound;
            return;
        }
    } else if (Kpad) {
        if (PASS == ONE_PASS) {
            bound = *a.absmax;
            if (!(bound >= 0.0f) || bound > 3.0e38f) bound = 0.0f;     // negative / NaN / Inf static bound: treated as 0
        } else {
#pragma unroll 8
            for (int i = tid; i < a.candidates / 4; i += threads) {
                const v4f c = reinterpret_cast<const v4f*>(a.found)[i];
                bound = fmaxf(bound, fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3])));
            }
            if (tid < a.candidates % 4) bound = fmaxf(bound, a.found[a.candidates / 4 * 4 + tid]);
            bound = largest_of(bound, best_of);
        }
    }

    // ---- multipliers ----
    const double qmax = a.bits == 8 ? 127.0 : 7.0;
    auto formed = [&](int n) -> float { return n > 0 && bound != 0.0f ? (float)(qmax / ((double)n * (double)bound)) : 0.0f; };
    auto multiplier = [&](int n) -> float { return (unsigned)n < TABLE ? table[n] : formed(n); };
    float other_m[KEPT];
    int other_at[KEPT];                  // the first of the other slots that this thread works on: places in the row, multipliers
    if (Kpad) {
        for (int n = tid; n < TABLE; n += threads) table[n] = formed(n);
        if (blockIdx.x == 0 && tid == 0) *a.s_x = bound == 0.0f ? 1.0f : (float)((double)bound / qmax);
        __syncthreads();
        if constexpr (KEEP) {
            if (far) {
                for (int p = tid; p < base; p += threads) row_m[p] = multiplier(a.rep[p]);
                __syncthreads();
            } else {                     // a thread's own, which it alone reads
#pragma unroll
                for (int k = 0; k < GPT; ++k)
                    if (own(k)) {
                        float m[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) m[i] = table[max(own_rep[k][i], 0)];
                        v4f* to = reinterpret_cast<v4f*>(row_m + 8 * (tid + k * threads));
                        to[0] = v4f{m[0], m[1], m[2], m[3]};
                        to[1] = v4f{m[4], m[5], m[6], m[7]};
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            const bool is = used(other_src[i], other_rep[i]);
            other_at[i] = is ? other_src[i] : zero_at;
            other_m[i] = is ? multiplier(other_rep[i]) : 0.0f;
        }
    }

    // ---- rows ----
    auto code = [&](float v, float m) -> uint8_t { return (uint8_t)(a.bits == 8 ? quantized_bits<8>(v, m) : quantized_bits<4>(v, m)); };
    auto codes_of_row = [&](int row, float t, float (&y)[GPT][8]) {
#pragma unroll
        for (int k = 0; k < GPT; ++k) {
            const int g = tid + k * threads;
            if (g >= G) continue;
            normalise(k, t, y[k]);
            if (a.Y) store_any<RAGGED>(y[k], row_of(a.Y, a.ldy, a.y_dtype == FQ_F32 ? 4 : 2, row), a.y_dtype, g, K);
            if (others) to_lds(g, y[k]);
            if constexpr (KEEP) {
                if (own(k)) store_eight(a.bits, y[k], row_m + 8 * g, a.out, Kpad, row, g);
            }
        }
        strip_barrier();                 // the row lies in LDS, and the sum's parts are read no more
        for (int from = base; from < Kpad; from += 16 * threads) {
#pragma unroll
            for (int i = 0; i < KEPT; ++i) {
                const int p = i * threads + tid;
                if (from == base && from + p < Kpad) row_q[p] = code(row_y[other_at[i]], other_m[i]);
            }
            for (int p = (from == base ? KEPT * threads : 0) + tid; p < min(Kpad - from, 16 * threads); p += threads) {
                const int j = a.src[from + p], n = a.rep[from + p];
                row_q[p] = used(j, n) ? code(row_y[j], multiplier(n)) : (uint8_t)0;
            }
            strip_barrier();
            if (from + 16 * tid < Kpad) store_packed(a.bits, *reinterpret_cast<const v4u*>(row_q + 16 * tid), a.out, Kpad, a.M, row, from / 16 + tid);
            if (from + 16 * threads < Kpad) strip_barrier();
        }
    };
    for (int row = blockIdx.x; row < a.M; row += gridDim.x) {
        float y[GPT][8];
        if constexpr (PASS == BOTH) {    // what this thread has stored itself
            const float t = few_t[row];
#pragma unroll
            for (int k = 0; k < GPT; ++k) {
                const int g = tid + k * threads;
                if (g < G) widen<HT>(load_raw<HT, RAGGED>(row_of(RT == NONE ? a.X : a.R_out, RT == NONE ? a.ldx : a.ldro, element_bytes<HT>(), row), g, K), y[k]);
            }
            strip_barrier();             // the row before is read no more
            codes_of_row(row, t, y);
        } else {
            double sum = 0.0;
            residual(row, y, sum);
            if constexpr (PASS == WITH_SCALE) {
                const float t = a.t[row];
                if (others) strip_barrier();
                codes_of_row(row, t, y);
            } else {
                codes_of_row(row, inverse_rms(sum), y);
            }
        }
    }
}

// Two pieces of 8 channels a thread, four of rows that 1024 threads do not hold so
int norm_threads(int K) { return std::min(1024, ((K + 7) / 8 + 127) / 128 * 64); }

template <int XT, int RT, int PASS> int launch(const Norm& a, int wgs, hipStream_t stream)
{
    const int threads = norm_threads(a.K);
    const bool two = a.K <= 2 * 8 * threads;
    const int smem = 16 * 8 + (16 + ALONE_PLACES + TABLE + row_places(a.K) + (two ? row_places(a.K) : 0)) * 4 + 16 * threads;
    const bool ragged = a.K % 8 != 0;
    auto kern = ragged ? (two ? rms_norm_kernel<XT, RT, PASS, 2, true> : rms_norm_kernel<XT, RT, PASS, 4, true>)
                       : (two ? rms_norm_kernel<XT, RT, PASS, 2, false> : rms_norm_kernel<XT, RT, PASS, 4, false>);
    static std::atomic<unsigned long long> attr_set[4];
    if (int rc = set_lds_limit(reinterpret_cast<const void*>(kern), 152 * 1024, attr_set[(two ? 0 : 1) + (ragged ? 2 : 0)])) return rc;
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
size_t rms_norm_workspace(int M) { return round_up((size_t)M * 4, 16) + NORM_WGS * 4; }

int launch_rms_norm_quant(const void* X, int x_dtype, int M, int K, int ldx, const void* R, int r_dtype, int ldr, void* R_out, int ldro,
                          const void* gamma, int g_dtype, float eps, void* Y, int y_dtype, int ldy, const int32_t* src, const int32_t* rep,
                          int Kpad, int bits, const float* absmax_in, void* Xq_out, float* s_x_out, void* workspace, hipStream_t stream)
{
    Norm a = {};
    a.X = X; a.R = R; a.gamma = gamma; a.R_out = R_out; a.Y = Y;
    a.ldx = ldx; a.ldr = ldr; a.ldro = ldro; a.ldy = ldy;
    a.M = M; a.K = K; a.Kpad = Kpad; a.g_dtype = g_dtype; a.y_dtype = y_dtype; a.bits = bits; a.eps = eps;
    a.src = src; a.rep = rep; a.absmax = absmax_in; a.out = static_cast<uint8_t*>(Xq_out); a.s_x = s_x_out;
    // 16 waves a CU
    const int wgs = std::min(M, std::min(NORM_WGS, compute_units() * std::max(1, 1024 / norm_threads(K)))), rt = R ? r_dtype : NONE;
    if (!Xq_out || absmax_in) return launch_types<ONE_PASS>(a, x_dtype, rt, wgs, stream);
    a.t = static_cast<float*>(workspace);
    a.found = a.t + round_up((size_t)M * 4, 16) / 4;
    a.candidates = wgs;
    // us, one workgroup / two launches: 1 x 4096 10 / 13, 2 x 4096 12.7 / 13, 3 x 4096 15.5 / 13, 2 x 8192 15.7 / 15.3, 1 x 16384 17 / 19.7
    if (M <= (K <= 4096 ? ALONE : 1)) return launch_types<BOTH>(a, x_dtype, rt, 1, stream);
    if (int rc = launch_types<FIND_SCALE>(a, x_dtype, rt, wgs, stream)) return rc;
    if (R) {        // the second pass reads what the first one stored
        a.X = R_out;
        a.ldx = ldro;
        x_dtype = r_dtype;
    }
    return launch_types<WITH_SCALE>(a, x_dtype, NONE, wgs, stream);
}

}  // namespace fq
