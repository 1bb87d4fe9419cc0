// fq_kv_append: new tokens' queries and keys turned by their positions, keys and values stored in the paged 8-bit cache.
//
// A workgroup owns what one call adds to one page of one head (of the keys, of the values, or the queries of that head's
// group at the same tokens): the scale of a (page, head) is the maximum over just these elements, so one workgroup finds it,
// rewrites the page's older codes where the scale grows, and stores the new ones; no atomics, no second pass over the input.
// A page of 64 tokens of 128 elements is 32 elements per thread, held in registers between the maximum and the codes.
// Keys lie token by token and values transposed, dimension by dimension, within a page: both are then read 16 consecutive
// bytes a lane in the order in which the matrix instruction of the attention wants them.
#include "fq_attn_common.h"

namespace fq {
namespace {

struct Append {
    const void *Q, *K, *V;
    void *Q_out, *K_out;
    long long ldq, ldk, ldv, ldqo, ldko;
    const int32_t *cu_new, *past, *table;
    const float *cosine, *sine;
    int8_t *k_cache, *v_cache;
    float *k_scale, *v_scale;
    int tokens, max_new, heads_kv, group, half, interleaved, capacity, pages, page, width, slots;
};

template <int DT> __device__ __forceinline__ void load8(const void* base, size_t at, float* out)
{
    typedef typename Stored<DT>::type T;
    const T* p = static_cast<const T*>(base) + at;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        const vec v = *reinterpret_cast<const vec*>(p + i);
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) out[i + e] = (float)v[e];
    }
}
template <int DT> __device__ __forceinline__ void store8(void* base, size_t at, const float* x)
{
    typedef typename Stored<DT>::type T;
    T* p = static_cast<T*>(base) + at;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        vec v;
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) v[e] = (T)x[i + e];
        *reinterpret_cast<vec*>(p + i) = v;
    }
}

// Elements d .. d + 7 of the head that begins at element `at`, turned by the angles of position `pos`.  Pairs of the first
// 2 * half elements: (i, i + half), or (2 i, 2 i + 1).  Every product and sum is rounded by itself.
template <int DT> __device__ __forceinline__ void rotated8(const Append& a, const void* base, size_t at, int d, int pos, float* x)
{
    load8<DT>(base, at + d, x);
    const int h = a.half;
    if (d >= 2 * h) return;
    const float *c = a.cosine + (size_t)pos * h, *s = a.sine + (size_t)pos * h;
    if (a.interleaved) {
        if (h % 4 == 0) {
            const v4f cv = *reinterpret_cast<const v4f*>(c + d / 2), sv = *reinterpret_cast<const v4f*>(s + d / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = x[2 * i], w = x[2 * i + 1];
                x[2 * i] = u * cv[i] - w * sv[i];
                x[2 * i + 1] = w * cv[i] + u * sv[i];
            }
        } else {
            for (int i = 0; i < 4; ++i)
                if (d / 2 + i < h) {
                    const float u = x[2 * i], w = x[2 * i + 1], cv = c[d / 2 + i], sv = s[d / 2 + i];
                    x[2 * i] = u * cv - w * sv;
                    x[2 * i + 1] = w * cv + u * sv;
                }
        }
    } else if (h % 8 == 0) {
        const bool second = d >= h;
        const int i = second ? d - h : d;
        float y[8];
        load8<DT>(base, at + (second ? d - h : d + h), y);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const v4f cv = *reinterpret_cast<const v4f*>(c + i + e), sv = *reinterpret_cast<const v4f*>(s + i + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p = x[e + k] * cv[k], q = y[e + k] * sv[k];
                x[e + k] = second ? p + q : p - q;
            }
        }
    } else {
        typedef typename Stored<DT>::type T;
        const T* row = static_cast<const T*>(base) + at;
        for (int e = 0; e < 8; ++e) {
            const int k = d + e;
            if (k >= 2 * h) continue;
            const bool second = k >= h;
            const int i = second ? k - h : k;
            const float p = x[e] * c[i], q = (float)row[second ? k - h : k + h] * s[i];
            x[e] = second ? p + q : p - q;
        }
    }
}

__device__ __forceinline__ int code_of(float x, float turn) { return (int)rintf(fminf(fmaxf(x * turn, -127.0f), 127.0f)); }
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d)
{
    return (a & 0xff) | (b & 0xff) << 8 | (c & 0xff) << 16 | (uint32_t)d << 24;
}
// Four codes in a scale that is `ratio` times finer than the new one.
__device__ __forceinline__ uint32_t rescaled(uint32_t codes, float ratio)
{
    int q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = (int)rintf((float)(int8_t)(codes >> (8 * i)) * ratio);
    return pack4(q[0], q[1], q[2], q[3]);
}

template <int DT, int D> __global__ __launch_bounds__(4 * MAX_PAGE) void kv_append_kernel(const Append a)
{
    constexpr int C = D / 8, PASSES = (MAX_PAGE * C + 4 * MAX_PAGE - 1) / (4 * MAX_PAGE), LDS_ROW = D + 4;
    __shared__ float peaks[4 * MAX_PAGE / 64];
    __shared__ __attribute__((aligned(16))) uint8_t staged[MAX_PAGE * LDS_ROW];
    const int b = blockIdx.x / a.slots, j = blockIdx.x - b * a.slots, kind = blockIdx.y / a.heads_kv, h = blockIdx.y - kind * a.heads_kv;
    const int tid = threadIdx.x, threads = blockDim.x;
    const Fill f = page_fill(packed_rows(a.cu_new[b], a.cu_new[b + 1], a.tokens, a.max_new), a.past[b], j, a.page, a.capacity);
    const int m = f.slot1 - f.slot0;
    if (m <= 0) return;

    if (kind == 2) {   // queries: whole heads in every pass, all read before any is written (Q_out may be Q)
        const int per_pass = threads / C, rows = m * a.group, row0 = tid / C, d = tid % C * 8;
        for (int at = 0; at < rows; at += per_pass) {
            const int r = at + row0, t = r / a.group, g = r - t * a.group;
            const bool mine = row0 < per_pass && r < rows;
            float x[8];
            if (mine) rotated8<DT>(a, a.Q, (f.row + t) * (size_t)a.ldq + (size_t)(h * a.group + g) * D, d, f.pos + t, x);
            __syncthreads();
            if (mine) store8<DT>(a.Q_out, (f.row + t) * (size_t)a.ldqo + (size_t)(h * a.group + g) * D + d, x);
        }
        return;
    }

    const bool keys = kind == 0;
    const int page = a.table[(size_t)b * a.width + f.index];
    const bool stored = page >= 0 && page < a.pages;
    float* scale_at = (keys ? a.k_scale : a.v_scale) + (stored ? (size_t)page * a.heads_kv + h : 0);
    const float old = stored && f.slot0 > 0 ? *scale_at : 0.0f;

    float x[PASSES][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int i = p * threads + tid, t = i / C, d = i % C * 8;
        if (i < m * C) {
            if (keys) rotated8<DT>(a, a.K, (f.row + t) * (size_t)a.ldk + (size_t)h * D, d, f.pos + t, x[p]);
            else load8<DT>(a.V, (f.row + t) * (size_t)a.ldv + (size_t)h * D + d, x[p]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[p][e]));
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
    if (tid % 64 == 0) peaks[tid / 64] = top;
    __syncthreads();   // after it everything of this page, head and call has been read: K_out may be K
    for (int w = 0; w < threads / 64; ++w) top = fmaxf(top, peaks[w]);

    if (keys && a.K_out) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int i = p * threads + tid, t = i / C, d = i % C * 8;
            if (i < m * C) store8<DT>(a.K_out, (f.row + t) * (size_t)a.ldko + (size_t)h * D + d, x[p]);
        }
    }
    if (!stored) return;

    // 127 steps to the largest magnitude; below 2^-126 a step has no reciprocal in fp32 and the block holds zeros
    float wanted = top / 127.0f;
    if (wanted < 0x1p-126f) wanted = 0.0f;
    const float scale = fmaxf(old, wanted), turn = scale > 0.0f ? 1.0f / scale : 0.0f, ratio = scale > 0.0f ? old / scale : 0.0f;
    const bool grown = f.slot0 > 0 && scale > old;
    if (tid == 0) *scale_at = scale;
    const size_t block = ((size_t)page * a.heads_kv + h) * a.page * D;
    if (keys) {
        int8_t* out = a.k_cache + block;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int i = p * threads + tid, t = i / C, d = i % C * 8;
            if (i >= m * C) continue;
            int q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = code_of(x[p][e], turn);
            *reinterpret_cast<v2u*>(out + (f.slot0 + t) * D + d) = v2u{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
        }
        if (grown)
            for (int i = tid; i < f.slot0 * D / 16; i += threads) {
                v4u* at = reinterpret_cast<v4u*>(out) + i;
                v4u v = *at;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = rescaled(v[e], ratio);
                *at = v;
            }
        return;
    }

    // values: through LDS into runs of 16 tokens of one dimension
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int i = p * threads + tid, t = i / C, d = i % C * 8;
        if (i >= m * C) continue;
        int q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = code_of(x[p][e], turn);
        uint32_t* at = reinterpret_cast<uint32_t*>(staged + t * LDS_ROW + d);
        at[0] = pack4(q[0], q[1], q[2], q[3]);
        at[1] = pack4(q[4], q[5], q[6], q[7]);
    }
    __syncthreads();
    const int from = grown ? 0 : f.slot0 / 16, runs = (f.slot1 + 15) / 16 - from;
    for (int i = tid; i < D * runs; i += threads) {
        const int d = i / runs, s = (i - d * runs + from) * 16;
        int8_t* out = a.v_cache + block + (size_t)d * a.page + s;
        if (s >= f.slot0 && s + 16 <= f.slot1) {
            v4u v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint8_t* c = staged + (s - f.slot0 + 4 * e) * LDS_ROW + d;
                v[e] = c[0] | c[LDS_ROW] << 8 | c[2 * LDS_ROW] << 16 | (uint32_t)c[3 * LDS_ROW] << 24;
            }
            *reinterpret_cast<v4u*>(out) = v;
        } else {
            if (grown)
                for (int t = s; t < f.slot0 && t < s + 16; ++t) out[t - s] = (int8_t)rintf((float)out[t - s] * ratio);
            for (int t = s < f.slot0 ? f.slot0 : s; t < f.slot1 && t < s + 16; ++t) out[t - s] = (int8_t)staged[(t - f.slot0) * LDS_ROW + d];
        }
    }
}

template <int DT> int launch(const Append& a, int head_dim, int batch, hipStream_t stream)
{
    const dim3 grid((unsigned)(batch * a.slots), (unsigned)((a.Q_out ? 3 : 2) * a.heads_kv));
    const int threads = 4 * a.page;
    switch (head_dim) {
    case 64: kv_append_kernel<DT, 64><<<grid, threads, 0, stream>>>(a); break;
    case 80: kv_append_kernel<DT, 80><<<grid, threads, 0, stream>>>(a); break;
    case 96: kv_append_kernel<DT, 96><<<grid, threads, 0, stream>>>(a); break;
    default: kv_append_kernel<DT, 128><<<grid, threads, 0, stream>>>(a); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "cache append launch failed: %s", hipGetErrorString(e));
}

}  // namespace

int launch_kv_append(const void* Q, const void* K, const void* V, int x_dtype, int tokens, int heads_q, int heads_kv, int head_dim,
                     long long ldq, long long ldk, long long ldv, const int32_t* cu_new, const int32_t* past, int batch, int max_new,
                     const float* rope_cos, const float* rope_sin, int rope_rows, int rope_dim, int interleaved, void* Q_out,
                     long long ldqo, void* K_out, long long ldko, int8_t* k_cache, int8_t* v_cache, float* k_scale, float* v_scale,
                     int pages, int page_size, const int32_t* page_table, int table_width, hipStream_t stream)
{
    int capacity = table_width * page_size;
    if (rope_dim > 0) capacity = std::min(capacity, rope_rows);
    const Append a{Q, K, V, Q_out, K_out, ldq, ldk, ldv, ldqo, ldko, cu_new, past, page_table, rope_cos, rope_sin, k_cache, v_cache,
                   k_scale, v_scale, tokens, max_new, heads_kv, heads_q / heads_kv, rope_dim / 2, interleaved, capacity, pages, page_size,
                   table_width, (int)pages_touched(max_new, page_size)};
    switch (x_dtype) {
    case FQ_F32: return launch<FQ_F32>(a, head_dim, batch, stream);
    case FQ_F16: return launch<FQ_F16>(a, head_dim, batch, stream);
    default: return launch<FQ_BF16>(a, head_dim, batch, stream);
    }
}

}  // namespace fq
