// fq_attn_cache: the last tokens of every sequence attend to all that the paged 8-bit cache holds of it.
//
// The reduction is bound by the cache's bytes: a key and a value byte serve at most the few queries of their group, so the
// kernel is a stream from HBM into registers, and everything else has to fit beside it.  What a wave does with 64 keys:
//   S^T = K Q^T   16 keys x 16 columns a product (a column is one query token of one head of the group), 32 elements of the
//                 head deep.  The 8-bit codes become fp16 exactly; the queries are fp16 too (bf16 ones are brought into its
//                 range by a power of two per column, which goes back in with the scale).
//   softmax       running maximum and sum per column.  The product leaves a column's 64 scores in four lanes, 16 each.
//   O^T += V^T P  16 dimensions x 16 columns, 32 keys deep, P rounded to fp16 (values in [0, 1]: half a step is 2^-12, below
//                 what the 2-byte output keeps).  A step's keys lie in one page, whose scale multiplies its product in 32 bits.
// No operand passes through LDS: which key of the page stands in which row of the first product is free, and with key
// 16 (r / 4) + 4 t + r % 4 in row r of tile t a lane's scores are those of 16 consecutive keys, the very ones whose values it
// reads as 16 consecutive bytes of a dimension (the cache holds values transposed for that) in the second product.
#include "fq_attn_common.h"

namespace fq {
namespace {

struct CacheAttn {
    const void* Q;
    void* Y;
    long long ldq, ldy;
    const int32_t *cu_q, *lens, *table;
    const int8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    float *part, *stat;     // with more than one split: [row, head, split, head_dim] and [row, head, split, (maximum, sum)]
    float scale;
    int tokens, max_q, max_len, heads_q, heads_kv, group, capacity, pages, page, width, splits;
};

constexpr int CACHE_THREADS = 64 * CACHE_WAVES;

// Eight signed bytes to fp16: with the sign bit turned a byte is q + 128, which as the low byte of 0x64.. is 1152 + q.
__device__ __forceinline__ v8h widen8(uint32_t lo, uint32_t hi)
{
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
    union {
        uint32_t u[4];
        v2h h[4];
        v8h all;
    } r;
    r.u[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
    r.u[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
    r.u[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
    r.u[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] -= off;
    return r.all;
}

__device__ __forceinline__ float over_groups_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_groups_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// NT tiles of 16 columns.  Grid: x the splits of all column tiles, y the key heads, z the sequences.
template <int DT, int D, int NT> __global__ __launch_bounds__(CACHE_THREADS) void attn_cache_kernel(const CacheAttn a)
{
    typedef typename Stored<DT>::type T;
    constexpr int KC = (D + 63) / 64, VT = D / 16, ROW = D + 4;   // 64-byte pieces of a key, 16-dimension tiles, LDS row
    __shared__ float gathered[CACHE_WAVES][16][ROW];
    __shared__ float tops[CACHE_WAVES][16 * NT], sums[CACHE_WAVES][16 * NT];

    const int tile = blockIdx.x / a.splits, split = blockIdx.x - tile * a.splits, h = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, col = lane % 16, g = lane / 16;
    const Rows rows = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens, a.max_q);
    const int columns = rows.count * a.group, c0 = tile * 16 * NT;
    if (c0 >= columns) return;
    const int keys = cached_keys(a.lens[b], a.max_len, a.capacity), share = share_keys(keys, a.splits);
    if (split > 0 && split * (long long)share >= keys) return;
    const int last = min(c0 + 16 * NT, columns) - 1;
    const int most = visible_keys(keys, rows.count, last / a.group), least = visible_keys(keys, rows.count, c0 / a.group);
    const int from = split * share, to = min((int)min(from + (long long)share, (long long)most), most);

    // the queries, as the second operand: lane (col, g) holds elements 64 j + 16 g + 8 i + 0..7 of its column's head
    v8h q[NT][KC][2];
    float factor[NT];
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = c0 + 16 * n + col, cc = min(c, columns - 1), t = cc / a.group;
        const T* p = static_cast<const T*>(a.Q) + (rows.first + t) * (size_t)a.ldq + (size_t)(h * a.group + cc - t * a.group) * D;
        limit[n] = visible_keys(keys, rows.count, t);
        typedef T v8 __attribute__((ext_vector_type(8)));
        v8 raw[KC][2];
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < KC; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int d = 64 * j + 16 * g + 8 * i;
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[j][i][e] = (T)0.0f;
                if (d < D) raw[j][i] = *reinterpret_cast<const v8*>(p + d);
                if constexpr (DT == FQ_BF16)
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)raw[j][i][e]));
            }
        factor[n] = a.scale * LOG2E;
        if constexpr (DT == FQ_F16) {
#pragma unroll
            for (int j = 0; j < KC; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) q[n][j][i] = raw[j][i];
        } else {
            // the largest magnitude of the head to [1, 4): what fp16 cannot hold then is below 2^-24 of it
            const uint32_t e = min(__float_as_uint(over_groups_max(top)) >> 23, 253u);
            const float down = __uint_as_float((254u - e) << 23);
            factor[n] *= e == 0 ? 0x1p-127f : __uint_as_float(e << 23);
#pragma unroll
            for (int j = 0; j < KC; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e2 = 0; e2 < 8; ++e2) q[n][j][i][e2] = (_Float16)((float)raw[j][i][e2] * down);
        }
    }

    v4f o[NT][VT];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < VT; ++t) o[n][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const size_t block = (size_t)a.page * D;
    const int32_t* table = a.table + (size_t)b * a.width;
    const int key_at = (16 * (col / 4) + col % 4) * D + 16 * g, value_at = col * a.page + 16 * g;
    for (int k0 = from + wave * CACHE_STEP; k0 < to; k0 += CACHE_SHARE) {
        const int index = k0 / a.page, off = k0 - index * a.page, page = table[index];
        if (page < 0 || page >= a.pages) continue;      // no such page: its keys are left out
        const size_t at = (size_t)page * a.heads_kv + h;
        const int8_t* kp = a.k_cache + at * block + (size_t)off * D + key_at;
        const int8_t* vp = a.v_cache + at * block + off + value_at;
        const float ks = a.k_scale[at], vs = a.v_scale[at];
        v4u kraw[4][KC], vraw[VT];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < KC; ++j) {
                kraw[t][j] = v4u{0, 0, 0, 0};
                if (64 * j + 16 * g < D) kraw[t][j] = *reinterpret_cast<const v4u*>(kp + 4 * t * D + 64 * j);
            }
#pragma unroll
        for (int t = 0; t < VT; ++t) vraw[t] = *reinterpret_cast<const v4u*>(vp + 16 * t * a.page);

        v4f s[NT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < KC; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const v8h k = widen8(kraw[t][j][2 * i], kraw[t][j][2 * i + 1]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[n][j][i], s[n][t], 0, 0, 0);
                }
        }

        v8h p[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float f = factor[n] * ks;
            float m = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = s[n][t][i] * f;
                    if (k0 + CACHE_STEP > least && k0 + 16 * g + 4 * t + i >= limit[n]) v = -INFINITY;
                    s[n][t][i] = v;
                    m = fmaxf(m, v);
                }
            m = fmaxf(over_groups_max(m), top[n]);
            const float base = m == -INFINITY ? 0.0f : m, keep = __builtin_amdgcn_exp2f(top[n] - base);
            top[n] = m;
            float add = 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(s[n][t][i] - base);
                    add += e;
                    p[n][t / 2][4 * (t % 2) + i] = (_Float16)e;
                }
            sum[n] = sum[n] * keep + add;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[n][t] *= keep;
        }

#pragma unroll
        for (int t = 0; t < VT; ++t) {
            const v8h v0 = widen8(vraw[t][0], vraw[t][1]), v1 = widen8(vraw[t][2], vraw[t][3]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                v4f r = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][0], v4f{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
                r = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][1], r, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][t][i] = __builtin_fmaf(r[i], vs, o[n][t][i]);
            }
        }
    }

    // the waves' shares meet in LDS, one tile of columns after the other
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float total = over_groups_sum(sum[n]);
        if (g == 0) {
            tops[wave][16 * n + col] = top[n];
            sums[wave][16 * n + col] = total;
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
        float m = tops[0][16 * n + col];
#pragma unroll
        for (int w = 1; w < CACHE_WAVES; ++w) m = fmaxf(m, tops[w][16 * n + col]);
        const float mine = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[n] - m);
#pragma unroll
        for (int t = 0; t < VT; ++t) *reinterpret_cast<v4f*>(&gathered[wave][col][16 * t + 4 * g]) = o[n][t] * mine;
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += CACHE_THREADS) {
            const int cl = i / (D / 4), d = (i - cl * (D / 4)) * 4, c = c0 + 16 * n + cl;
            if (c >= columns) continue;
            float best = tops[0][16 * n + cl], l = 0.0f;
#pragma unroll
            for (int w = 1; w < CACHE_WAVES; ++w) best = fmaxf(best, tops[w][16 * n + cl]);
            v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < CACHE_WAVES; ++w) {
                if (best != -INFINITY) l += sums[w][16 * n + cl] * __builtin_amdgcn_exp2f(tops[w][16 * n + cl] - best);
                y += *reinterpret_cast<const v4f*>(&gathered[w][cl][d]);
            }
            const int t = c / a.group, head = h * a.group + c - t * a.group;
            const size_t row = rows.first + t;
            if (a.splits > 1) {
                const size_t to_part = (row * a.heads_q + head) * a.splits + split;
                *reinterpret_cast<v4f*>(a.part + to_part * D + d) = y;
                if (d == 0) {
                    a.stat[2 * to_part] = best;
                    a.stat[2 * to_part + 1] = l;
                }
            } else {
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                typedef T v4 __attribute__((ext_vector_type(4)));
                v4 out;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (T)(y[e] * inv);
                *reinterpret_cast<v4*>(static_cast<T*>(a.Y) + row * (size_t)a.ldy + (size_t)head * D + d) = out;
            }
        }
    }
}

// The shares of one (row, head) joined by one wave.  Grid: x the query heads in groups of the waves, y the query tokens, z the sequences.
template <int DT, int D> __global__ __launch_bounds__(CACHE_THREADS) void attn_cache_join_kernel(const CacheAttn a)
{
    typedef typename Stored<DT>::type T;
    const int b = blockIdx.z, t = blockIdx.y, head = blockIdx.x * CACHE_WAVES + threadIdx.x / 64, lane = threadIdx.x % 64;
    const Rows rows = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens, a.max_q);
    if (t >= rows.count || head >= a.heads_q) return;
    const int keys = cached_keys(a.lens[b], a.max_len, a.capacity), share = share_keys(keys, a.splits), used = shares_used(keys, share);
    const size_t at = ((size_t)(rows.first + t) * a.heads_q + head) * a.splits;
    float best = -INFINITY;
    for (int s = lane; s < used; s += 64) best = fmaxf(best, a.stat[2 * (at + s)]);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) best = fmaxf(best, __shfl_xor(best, s));
    float y[2] = {0.0f, 0.0f}, l = 0.0f;
    const int d = 2 * lane;
    if (best != -INFINITY)
#pragma unroll 4
        for (int s = 0; s < used; ++s) {
            const float w = __builtin_amdgcn_exp2f(a.stat[2 * (at + s)] - best);
            l += a.stat[2 * (at + s) + 1] * w;
            if (d < D) {
                y[0] += a.part[(at + s) * D + d] * w;
                y[1] += a.part[(at + s) * D + d + 1] * w;
            }
        }
    if (d >= D) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    typedef T v2 __attribute__((ext_vector_type(2)));
    const v2 out = {(T)(y[0] * inv), (T)(y[1] * inv)};
    *reinterpret_cast<v2*>(static_cast<T*>(a.Y) + (size_t)(rows.first + t) * a.ldy + (size_t)head * D + d) = out;
}

template <int DT, int D> int launch(const CacheAttn& a, int batch, hipStream_t stream)
{
    const long long columns = (long long)a.max_q * a.group;
    const int nt = cache_tiles(columns);
    const dim3 grid((unsigned)((columns + 16 * nt - 1) / (16 * nt) * a.splits), (unsigned)a.heads_kv, (unsigned)batch);
    if (nt == 1) attn_cache_kernel<DT, D, 1><<<grid, CACHE_THREADS, 0, stream>>>(a);
    else if (nt == 2) attn_cache_kernel<DT, D, 2><<<grid, CACHE_THREADS, 0, stream>>>(a);
    else attn_cache_kernel<DT, D, 4><<<grid, CACHE_THREADS, 0, stream>>>(a);
    if (a.splits > 1)
        attn_cache_join_kernel<DT, D><<<dim3((unsigned)((a.heads_q + CACHE_WAVES - 1) / CACHE_WAVES), (unsigned)a.max_q, (unsigned)batch), CACHE_THREADS, 0,
                                        stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "cache attention launch failed: %s", hipGetErrorString(e));
}

template <int DT> int launch_dim(const CacheAttn& a, int head_dim, int batch, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch<DT, 64>(a, batch, stream);
    case 80: return launch<DT, 80>(a, batch, stream);
    case 96: return launch<DT, 96>(a, batch, stream);
    default: return launch<DT, 128>(a, batch, stream);
    }
}

}  // namespace

int launch_attn_cache(const void* Q, int x_dtype, int tokens, int heads_q, int heads_kv, int head_dim, long long ldq, const int32_t* cu_q,
                      const int32_t* lens, int batch, int max_q, int max_len, const int8_t* k_cache, const int8_t* v_cache,
                      const float* k_scale, const float* v_scale, int pages, int page_size, const int32_t* page_table, int table_width,
                      float scale, void* Y, long long ldy, void* workspace, int splits, hipStream_t stream)
{
    float* part = static_cast<float*>(workspace);
    float* stat = part + (splits > 1 ? (size_t)tokens * heads_q * splits * head_dim : 0);
    const CacheAttn a{Q, Y, ldq, ldy, cu_q, lens, page_table, k_cache, v_cache, k_scale, v_scale, part, stat, scale, tokens, max_q, max_len,
                      heads_q, heads_kv, heads_q / heads_kv, table_width * page_size, pages, page_size, table_width, splits};
    return x_dtype == FQ_F16 ? launch_dim<FQ_F16>(a, head_dim, batch, stream) : launch_dim<FQ_BF16>(a, head_dim, batch, stream);
}

}  // namespace fq
