// fq_attn_prompt: attention over packed sequences of different lengths, causal or not, grouped heads.
//
// Bound by the matrix pipe for long sequences (4 D operations for every pair of a query and a key it sees).  One pass over the
// keys with the running maximum and sum of the softmax; a workgroup takes 128 queries of one head, 32 a wave, and walks the keys
// in tiles of 64 through LDS.
//   S^T = K Q^T   32 keys x 32 queries a product: a query's scores are in two lanes, so its maximum and sum need one exchange.
//   O^T += V^T P  the scores' registers are the second operand as they stand: which key of the tile stands at which place of the
//                 reduction is free as long as the values follow, and their transposed reads from LDS take four consecutive
//                 keys of a dimension, as a lane holds them.
// P is rounded to the input's type, the row sums are taken before that in 32 bits.
#include "fq_attn_common.h"

namespace fq {
namespace {

struct PromptAttn {
    const void *Q, *K, *V;
    void* Y;
    long long ldq, ldk, ldv, ldy;
    const int32_t *cu_q, *cu_k;
    float factor;            // scale * log2(e), positive
    int tokens_q, tokens_k, max_q, heads_q, heads_kv, group, causal, batch, tiles;
};

constexpr int PROMPT_KEYS = 64;   // a tile
constexpr float SLACK = 8.0f;   // the accumulators are rescaled only when a maximum has grown by more than a factor 2^8

template <int DT> struct Mma;
template <> struct Mma<FQ_BF16> {
    typedef __bf16 T;
    typedef v8bf v8;
    typedef v4bf v4;
    static __device__ __forceinline__ v16f mul(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<FQ_F16> {
    typedef _Float16 T;
    typedef v8h v8;
    typedef v4h v4;
    static __device__ __forceinline__ v16f mul(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Rows of LDS: keys an odd number of 16-byte pieces apart, so that the rows that lanes read together lie on different banks;
// values 8 or 24 banks (of 32) apart, as four of them are read together, 32 bytes each.
constexpr int key_row(int D) { return 2 * D + 16; }
constexpr int value_row(int D)
{
    int words = D / 2;
    while (words % 32 != 8 && words % 32 != 24) words += 4;
    return 4 * words;
}

// Four 2-byte elements of a column out of row-major LDS: of 16 neighbouring lanes, lanes 4 r .. 4 r + 3 point at 16 consecutive
// elements of row r, and lane i receives element i of the four rows.
__device__ __forceinline__ v2u read_transposed(uint32_t lds_address)
{
    typedef __attribute__((ext_vector_type(4))) __fp16 v4fp;
    typedef __attribute__((address_space(3))) v4fp* lds_ptr;
    const v4fp r = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_ptr)(uintptr_t)lds_address);
    return __builtin_bit_cast(v2u, r);
}

template <int DT, int D> __global__ __launch_bounds__(PROMPT_THREADS, 2) void attn_prompt_kernel(const PromptAttn a)
{
    typedef Mma<DT> M;
    typedef typename M::T T;
    typedef typename M::v8 v8;
    constexpr int KS = D / 16, VT = (D + 31) / 32, C = D / 8, KROW = key_row(D), VROW = value_row(D);
    constexpr int KBYTES = PROMPT_KEYS * KROW, VBYTES = PROMPT_KEYS * VROW, STAGE = KBYTES + VBYTES;
    constexpr int PIECES = (PROMPT_KEYS * C + PROMPT_THREADS - 1) / PROMPT_THREADS;   // 16-byte pieces of each operand's tile per thread
    constexpr bool EVEN = PROMPT_KEYS * C % PROMPT_THREADS == 0;
    // reads of the last 32 dimensions reach beyond a row of 80: within the tile, or the 64 bytes behind the last
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE + 64];

    // workgroups of one sequence and key head on one XCD, the longest rows first
    const unsigned total = gridDim.x, id = blockIdx.x, quot = total >> 3, rem = total & 7, xcd = id & 7, at_xcd = id >> 3;
    const unsigned logical = xcd < rem ? xcd * (quot + 1) + at_xcd : rem * (quot + 1) + (xcd - rem) * quot + at_xcd;
    const unsigned per_pair = (unsigned)a.tiles * a.group, pair = logical / per_pair, item = logical - pair * per_pair;
    const int tile = a.tiles - 1 - (int)(item / a.group), b = pair / a.heads_kv, hk = pair - b * a.heads_kv;
    const int head = hk * a.group + item % a.group;

    const Rows rq = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens_q, a.max_q), rk = packed_rows(a.cu_k[b], a.cu_k[b + 1], a.tokens_k, a.tokens_k);
    const int q0 = tile * PROMPT_ROWS;
    if (q0 >= rq.count) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 32, half = lane / 32;
    const int row = q0 + 32 * wave + col, keys = rk.count;
    const auto visible = [&](int i) { return a.causal ? visible_keys(keys, rq.count, i) : keys; };
    const int mine = visible(min(row, rq.count - 1)), least = visible(min(q0 + 32 * wave, rq.count - 1));
    const int wave_keys = q0 + 32 * wave >= rq.count ? 0 : visible(min(q0 + 32 * wave + 31, rq.count - 1)), most = visible(min(q0 + PROMPT_ROWS, rq.count) - 1);

    const T* qp = static_cast<const T*>(a.Q) + (rq.first + (size_t)min(row, rq.count - 1)) * a.ldq + (size_t)head * D + 8 * half;
    v8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8*>(qp + 16 * s);

    // pieces of the tiles that this thread carries
    const T *kp = static_cast<const T*>(a.K) + (size_t)rk.first * a.ldk + (size_t)hk * D, *vp = static_cast<const T*>(a.V) + (size_t)rk.first * a.ldv + (size_t)hk * D;
    v4u kreg[PIECES], vreg[PIECES];
    const auto fetch = [&](int k0) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int i = p * PROMPT_THREADS + tid, r = i / C, c = i - r * C, key = min(k0 + r, keys - 1);   // rows behind the last: it again
            if (!EVEN && r >= PROMPT_KEYS) continue;
            kreg[p] = *reinterpret_cast<const v4u*>(kp + (size_t)key * a.ldk + 8 * c);
            vreg[p] = *reinterpret_cast<const v4u*>(vp + (size_t)key * a.ldv + 8 * c);
        }
    };
    const auto put = [&](int stage) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int i = p * PROMPT_THREADS + tid, r = i / C, c = i - r * C;
            if (!EVEN && r >= PROMPT_KEYS) continue;
            *reinterpret_cast<v4u*>(lds + stage * STAGE + r * KROW + 16 * c) = kreg[p];
            *reinterpret_cast<v4u*>(lds + stage * STAGE + KBYTES + r * VROW + 16 * c) = vreg[p];
        }
    };

    v16f o[VT];
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;      // of the unscaled scores; the sum over this lane's keys only

    const uint32_t key_at = col * KROW + 16 * half;
    const uint32_t value_at = KBYTES + (4 * half + lane % 16 / 4) * VROW + 32 * (lane / 16 % 2) + 8 * (lane % 4);
    const uint32_t base_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    if (most > 0) {
        fetch(0);
        put(0);
    }
    for (int k0 = 0, stage = 0; k0 < most; k0 += PROMPT_KEYS, stage ^= 1) {
        const bool more = k0 + PROMPT_KEYS < most;
        if (more) fetch(k0 + PROMPT_KEYS);
        __syncthreads();
        if (k0 < wave_keys) {
            const uint8_t* st = lds + stage * STAGE;
            v16f s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
                for (int e = 0; e < KS; ++e) s[t] = M::mul(*reinterpret_cast<const v8*>(st + key_at + 32 * t * KROW + 32 * e), q[e], s[t]);
            }
            // register i of tile t: key 32 t + 8 (i / 4) + 4 half + i % 4
            if (k0 + PROMPT_KEYS > least) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (k0 + 32 * t + 8 * (i / 4) + 4 * half + i % 4 >= mine) s[t][i] = -INFINITY;
            }
            float m = fmaxf(s[0][0], s[1][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) m = fmaxf(m, fmaxf(s[0][i], s[1][i]));
            m = fmaxf(m, __shfl_xor(m, 32));
            if (__ballot((m - top) * a.factor > SLACK || top == -INFINITY)) {
                const float now = fmaxf(m, top), keep = now == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((top - now) * a.factor);
                top = now;
                sum *= keep;
#pragma unroll
                for (int t = 0; t < VT; ++t) o[t] *= keep;
            }
            const float base = top == -INFINITY ? 0.0f : top * a.factor;
            v8 p[4];      // 16 keys each
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.factor, -base));
                    sum += e;
                    p[2 * t + i / 8][i % 8] = (T)e;
                }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int t = 0; t < VT; ++t) {
                    const uint32_t v = base_at + stage * STAGE + value_at + 16 * c * VROW + 64 * t;
                    const v2u lo = read_transposed(v), hi = read_transposed(v + 8 * VROW);
                    o[t] = M::mul(__builtin_bit_cast(v8, (v4u{lo[0], lo[1], hi[0], hi[1]})), p[c], o[t]);
                }
        }
        if (more) put(stage ^ 1);
    }

    sum += __shfl_xor(sum, 32);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    if (row >= rq.count) return;
    T* yp = static_cast<T*>(a.Y) + (rq.first + (size_t)row) * a.ldy + (size_t)head * D + 4 * half;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (32 * t + 8 * i >= D) continue;
            typename M::v4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (T)(o[t][4 * i + e] * inv);
            *reinterpret_cast<typename M::v4*>(yp + 32 * t + 8 * i) = y;
        }
}

template <int DT> int launch(const PromptAttn& a, int head_dim, hipStream_t stream)
{
    const unsigned grid = (unsigned)(a.batch * (long long)a.heads_q * a.tiles);
    switch (head_dim) {
    case 64: attn_prompt_kernel<DT, 64><<<grid, PROMPT_THREADS, 0, stream>>>(a); break;
    case 80: attn_prompt_kernel<DT, 80><<<grid, PROMPT_THREADS, 0, stream>>>(a); break;
    case 96: attn_prompt_kernel<DT, 96><<<grid, PROMPT_THREADS, 0, stream>>>(a); break;
    default: attn_prompt_kernel<DT, 128><<<grid, PROMPT_THREADS, 0, stream>>>(a); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "prompt attention launch failed: %s", hipGetErrorString(e));
}

}  // namespace

int launch_attn_prompt(const void* Q, const void* K, const void* V, int x_dtype, int tokens_q, int tokens_k, int heads_q, int heads_kv,
                       int head_dim, long long ldq, long long ldk, long long ldv, const int32_t* cu_q, const int32_t* cu_k, int batch, int max_q,
                       int causal, float scale, void* Y, long long ldy, hipStream_t stream)
{
    const PromptAttn a{Q, K, V, Y, ldq, ldk, ldv, ldy, cu_q, cu_k, scale * LOG2E, tokens_q, tokens_k, max_q, heads_q, heads_kv, heads_q / heads_kv,
                       causal, batch, (int)prompt_tiles(max_q)};
    return x_dtype == FQ_F16 ? launch<FQ_F16>(a, head_dim, stream) : launch<FQ_BF16>(a, head_dim, stream);
}

}  // namespace fq
