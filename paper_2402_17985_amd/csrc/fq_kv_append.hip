// fq_kv_append: new tokens' queries and keys turned by their positions, keys and values stored in the paged 8-bit cache.
//
// A workgroup owns what one call adds to one page of one head (of the keys, of the values, or the queries of that head's
// group at the same tokens): the scale of a (page, head) is the maximum over just these elements, so one workgroup finds it,
// rewrites the page's older codes where the scale grows, and stores the new ones; no atomics, no second pass over the input.
// A page of 64 tokens of 128 elements is 32 elements per thread, held in registers between the maximum and the codes.
// Keys lie token by token and values transposed, dimension by dimension, within a page: both are then read 16 consecutive
// bytes a lane in the order in which the matrix instruction of the attention wants them.
// Bound by bytes for prompts: 4 x 2048 tokens, 40 heads of 128, fp16: 106 us, 4.7 TB/s read and written, the rate of a large copy; by latency for single
// tokens: 4.3 us for one, 5.2 for 64 sequences (offsets, table, row and scale one after the other, then a reduction).
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
    int tokens, max_new, heads_kv, group, half, interleaved, capacity, pages, page, width, parts, batch, each;      // parts: key heads times two (keys, values) or three (queries too)
};

template <int DT> __device__ __forceinline__ void load8(const typename Stored<DT>::type* base, uint32_t at, float* out)
{
    typedef typename Stored<DT>::type T;
    const T* p = base + at;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        const vec v = *reinterpret_cast<const vec*>(p + i);
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) out[i + e] = (float)v[e];
    }
}
template <int DT> __device__ __forceinline__ void store8(typename Stored<DT>::type* base, uint32_t at, const float* x)
{
    typedef typename Stored<DT>::type T;
    T* p = base + at;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        vec v;
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) v[e] = (T)x[i + e];
        *reinterpret_cast<vec*>(p + i) = v;
    }
}

// How the pairs of a head's first 2 * half elements lie: (i, i + half) or (2 i, 2 i + 1); by 16-byte loads where the halves are whole pieces
// of 8 elements, or the pairs' angles of 4.
enum Turn { TURN_NONE, TURN_HALVES, TURN_PAIRS, TURN_ANY };

// Elements d .. d + 7 of the head that begins at element `at`, turned by the angles of position `pos`.  Every product and sum is rounded by
// itself.  Without branches (but for odd widths), so that a thread's loads all go out before the first is awaited: an append of 4 x 2048
// tokens of 40 heads of 128 136 -> 106 us (4.7 TB/s).
template <int DT, int TURN>
__device__ __forceinline__ void rotated8(const Append& a, const typename Stored<DT>::type* base, uint32_t at, int d, int pos, float* x)
{
    load8<DT>(base, at + d, x);
    if constexpr (TURN == TURN_NONE) return;
    const int h = a.half;
    const float *c = a.cosine + (size_t)pos * h, *s = a.sine + (size_t)pos * h;
    const bool turned = d < 2 * h;
    if constexpr (TURN == TURN_PAIRS) {
        const int i = turned ? d / 2 : 0;
        const v4f cv = *reinterpret_cast<const v4f*>(c + i), sv = *reinterpret_cast<const v4f*>(s + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float u = x[2 * k], w = x[2 * k + 1], p = u * cv[k] - w * sv[k], q = w * cv[k] + u * sv[k];
            x[2 * k] = turned ? p : u;
            x[2 * k + 1] = turned ? q : w;
        }
    } else if constexpr (TURN == TURN_HALVES) {
        const bool second = d >= h;
        const int other = !turned ? d : second ? d - h : d + h, i = !turned ? 0 : second ? d - h : d;
        float y[8];
        load8<DT>(base, at + other, y);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const v4f cv = *reinterpret_cast<const v4f*>(c + i + e), sv = *reinterpret_cast<const v4f*>(s + i + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p = x[e + k] * cv[k], q = y[e + k] * sv[k], r = second ? p + q : p - q;
                x[e + k] = turned ? r : x[e + k];
            }
        }
    } else {
        const typename Stored<DT>::type* row = base + at;
#pragma unroll 1
        for (int i = a.interleaved ? d / 2 : 0; i < h; ++i) {
            const int lo = a.interleaved ? 2 * i : i, hi = a.interleaved ? 2 * i + 1 : i + h;
            if (lo >= d + 8) break;
            const float u = (float)row[lo], w = (float)row[hi], p = u * c[i] - w * s[i], q = w * c[i] + u * s[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = lo - d == e ? p : hi - d == e ? q : x[e];
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

// FEW: a thread takes 8 elements, else up to 32.  Registers: as many waves per SIMD as go without scratch.
template <int DT, int D, int TURN, bool FEW>
__global__ __launch_bounds__(4 * MAX_PAGE, TURN == TURN_HALVES ? (DT == FQ_F32 ? 3 : 4) : TURN == TURN_NONE && D % 64 != 0 ? 4 : 5) void kv_append_kernel(const Append a)
{
    typedef typename Stored<DT>::type T;
    constexpr int C = D / 8, PASSES = FEW ? 1 : (C + 3) / 4, LDS_ROW = D + 4;
    __shared__ float peaks[4 * MAX_PAGE / 64];
    __shared__ __attribute__((aligned(16))) uint8_t staged[MAX_PAGE * LDS_ROW];
    // the heads of the same tokens one after the other: together they read and write whole rows
    const unsigned at_page = blockIdx.x / a.parts, part = blockIdx.x - at_page * a.parts;
    const auto first_of = [&](int b) { return first_page_place(min(max(a.cu_new[b], 0), a.tokens), a.page, b); };
    const int b = a.each ? at_page / a.each : sequence_at(at_page, a.batch, first_of), j = a.each ? (int)at_page - b * a.each : (int)at_page - first_of(b);
    const int kind = part / a.heads_kv, h = part - kind * a.heads_kv;
    const int tid = threadIdx.x, threads = blockDim.x;
    const Fill f = page_fill(packed_rows(a.cu_new[b], a.cu_new[b + 1], a.tokens, a.max_new), a.past[b], j, a.page, a.capacity);
    const int m = f.slot1 - f.slot0;
    if (m <= 0) return;

    if (kind == 2) {   // queries: whole heads in every round, all of a round read before any is written (Q_out may be Q)
        const T* from = static_cast<const T*>(a.Q) + (size_t)f.row * a.ldq + (size_t)h * a.group * D;
        T* to = static_cast<T*>(a.Q_out) + (size_t)f.row * a.ldqo + (size_t)h * a.group * D;
        const int per_pass = threads / C, rows = m * a.group, row0 = tid / C, d = tid % C * 8;
        for (int at = row0; at - row0 < rows; at += PASSES * per_pass) {
            float x[PASSES][8];
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int r = min(at + p * per_pass, rows - 1), t = r / a.group;      // behind the last it again
                rotated8<DT, TURN>(a, from, t * (uint32_t)a.ldq + (r - t * a.group) * D, d, f.pos + t, x[p]);
            }
            __syncthreads();
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int r = at + p * per_pass, t = r / a.group;
                if (row0 < per_pass && r < rows) store8<DT>(to, t * (uint32_t)a.ldqo + (r - t * a.group) * D + d, x[p]);
            }
        }
        return;
    }

    const bool keys = kind == 0;
    const int page = a.table[(size_t)b * a.width + f.index];
    const bool stored = page >= 0 && page < a.pages;
    float* scale_at = (keys ? a.k_scale : a.v_scale) + (stored ? (size_t)page * a.heads_kv + h : 0);
    const float old = stored && f.slot0 > 0 ? *scale_at : 0.0f;

    const T* from = keys ? static_cast<const T*>(a.K) + (size_t)f.row * a.ldk + (size_t)h * D : static_cast<const T*>(a.V) + (size_t)f.row * a.ldv + (size_t)h * D;
    float x[PASSES][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int i = p * threads + tid, t = min(i / C, m - 1), d = i % C * 8;      // behind the last token it again
        if (keys) rotated8<DT, TURN>(a, from, t * (uint32_t)a.ldk, d, f.pos + t, x[p]);
        else load8<DT>(from, t * (uint32_t)a.ldv + d, x[p]);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[p][e]));
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
    if (tid % 64 == 0) peaks[tid / 64] = top;
    __syncthreads();   // after it everything of this page, head and call has been read: K_out may be K
    for (int w = 0; w < threads / 64; ++w) top = fmaxf(top, peaks[w]);

    if (keys && a.K_out) {
        T* to = static_cast<T*>(a.K_out) + (size_t)f.row * a.ldko + (size_t)h * D;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int i = p * threads + tid, t = i / C, d = i % C * 8;
            if (i < m * C) store8<DT>(to, t * (uint32_t)a.ldko + d, x[p]);
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
    const int first = grown ? 0 : f.slot0 / 16, runs = (f.slot1 + 15) / 16 - first;
    for (int i = tid; i < D * runs; i += threads) {
        const int d = i / runs, s = (i - d * runs + first) * 16;
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

template <int DT, int D, bool FEW> void launch_turn(const Append& a, unsigned grid, int threads, hipStream_t stream)
{
    if (a.half == 0) kv_append_kernel<DT, D, TURN_NONE, FEW><<<grid, threads, 0, stream>>>(a);
    else if (a.interleaved && a.half % 4 == 0) kv_append_kernel<DT, D, TURN_PAIRS, FEW><<<grid, threads, 0, stream>>>(a);
    else if (!a.interleaved && a.half % 8 == 0) kv_append_kernel<DT, D, TURN_HALVES, FEW><<<grid, threads, 0, stream>>>(a);
    else kv_append_kernel<DT, D, TURN_ANY, FEW><<<grid, threads, 0, stream>>>(a);
}

template <int DT, int D> int launch(const Append& a, unsigned grid, hipStream_t stream)
{
    const AppendPlan plan = append_plan(a.max_new, a.page, D);
    if (plan.few) launch_turn<DT, D, true>(a, grid, plan.threads, stream);
    else launch_turn<DT, D, false>(a, grid, plan.threads, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "cache append launch failed: %s", hipGetErrorString(e));
}

template <int DT> int launch_dim(const Append& a, int head_dim, unsigned grid, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch<DT, 64>(a, grid, stream);
    case 80: return launch<DT, 80>(a, grid, stream);
    case 96: return launch<DT, 96>(a, grid, stream);
    default: return launch<DT, 128>(a, grid, stream);
    }
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
    const AppendPages places = append_pages(batch, tokens, max_new, page_size);
    const Append a{Q, K, V, Q_out, K_out, ldq, ldk, ldv, ldqo, ldko, cu_new, past, page_table, rope_cos, rope_sin, k_cache, v_cache,
                   k_scale, v_scale, tokens, max_new, heads_kv, heads_q / heads_kv, rope_dim / 2, interleaved, capacity, pages, page_size,
                   table_width, (Q_out ? 3 : 2) * heads_kv, batch, places.each};
    const unsigned grid = (unsigned)(places.places * a.parts);
    switch (x_dtype) {
    case FQ_F32: return launch_dim<FQ_F32>(a, head_dim, grid, stream);
    case FQ_F16: return launch_dim<FQ_F16>(a, head_dim, grid, stream);
    default: return launch_dim<FQ_BF16>(a, head_dim, grid, stream);
    }
}

}  // namespace fq
