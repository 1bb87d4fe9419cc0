// fq_attn_cache: the last tokens of every sequence attend to all that the paged 8-bit cache holds of it.
//
// The reduction is bound by the cache's bytes: a key and a value byte serve at most the few queries of their group, so the
// kernel is a stream from HBM into registers, and everything else has to fit beside it.  What a wave does with 64 keys:
//   S^T = K Q^T   16 keys x 16 columns a product (a column is one query token of one head of the group), 64 elements of the head deep, in
//                 8-bit integers: the codes go into the matrix instruction as they come.  The queries are integers of up to 127 * 256 steps,
//                 two limbs, so that each product is done twice; the sums are exact.  (Codes widened to fp16 take five instructions
//                 for four of them; a step of 64 keys is 300 vector instructions beside 32 products as it is.)
//   softmax       running maximum and sum per column.  The product leaves a column's 64 scores in four lanes, 16 each.
//   O^T += V^T P  16 dimensions x 16 columns, 32 keys deep, P in fp16: half a step is 2^-11 of each, little beside the 2^-8 that a bf16 output is
//                 rounded by.  For an fp16 output it would be as much as that one's own rounding (error against 64 bits 1.4 times that of
//                 exact probabilities, 1.03 so), so that P is the sum of two there: another product, 0.5 to 4 % of the time of single tokens.
//                 What fp16 cannot hold is below 2^-32 of the running maximum and below 2^-24 of the step's own: steps whose weights all are far
//                 below the maximum have a unit of their own.  (Without it all of 131072 keys 17.7 nats below one vanished.)
//                 The sum that divides is that of the rounded ones.  A step's keys lie in one page, whose scale multiplies
//                 its product in 32 bits.
// No operand passes through LDS: which key of the page stands in which row of the first product is free, and with key
// 16 (r / 4) + 4 t + r % 4 in row r of tile t a lane's scores are those of 16 consecutive keys, the very ones whose values it
// reads as 16 consecutive bytes of a dimension (the cache holds values transposed for that) in the second product.
// Each wave has a step of keys and values under way while it works on the one before, 16 KiB for heads of 128.  The waves of a workgroup share the keys
// of one sequence and head, their parts meet in LDS; few workgroups share them once more, and a second kernel joins the shares.
// Measured, reads of the cache: 64 sequences of 8192 tokens, 64 heads over 8, 181 to 190 us, 5.7 to 5.9 TB/s (a large sum reads 6.0); two of 131072 tokens 93 to 97 us, 5.5 to 5.8 TB/s,
// 5 us of it the join of 16 shares; one of 1001 tokens, 32 heads, 8.5 us, a chain of latencies: 2.5 to the first scores, 3 for 256 keys through one CU, the
// second launch.  Two steps under way instead of one, or the first step's loads before the queries', took up to 1 us more on short sequences, as
// longer code has to come in first, and no less on long ones.
#include "fq_attn_cache.h"

namespace fq {
namespace {

// Over the four lanes of a column, 16 apart.
__device__ __forceinline__ float over_groups_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float over_groups_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// The sequence of the z-th workgroups, at most 64 of them, by length: longest first, as long ones begun last would run on alone; or, where all
// workgroups are on the device at once, two to a CU, the longer half so and then the shorter half, shortest first: the second of a CU's is then as
// short as the first is long.  (64 sequences of 160 to 8192 tokens, 64 heads over 8: 124 us as they come, 106 so.)
__device__ __forceinline__ int by_length(const CacheAttn& a, int z, int batch)
{
    const int lane = threadIdx.x % 64, mine = a.lens[min(lane, batch - 1)], half = (batch + 1) / 2;
    const int nth = a.order == CACHE_FOLDED && z >= half ? batch - 1 - (z - half) : z;
    const uint32_t key = lane < batch ? length_key(mine) : 0;
    const int longer = sum_of_longer(key, 1, batch);
    return __builtin_ctzll(__ballot(lane < batch && longer == nth));
}

constexpr float STEP_SHIFT = 7.0f, STEP_UNIT = 0x1p-7f;      // a probability of 1 is 2^7 in fp16; accumulators and sums count in 1

// NT tiles of 16 columns.  Grid: x the shares of the keys, y the key heads of one block of columns after the other (with 8 key heads the blocks of one are on
// one XCD), z the sequences.
template <int DT, int D, int NT, int WAVES> __global__ __launch_bounds__(64 * WAVES, 2) void attn_cache_kernel(const CacheAttn a)
{
    constexpr int ROUND = CACHE_STEP * WAVES;
    constexpr int LIMBS = DT == FQ_F16 ? 2 : 1;      // of a probability
    typedef typename Stored<DT>::type T;
    constexpr int KC = (D + 63) / 64, VT = D / 16, ROW = D + 4;   // 64-byte pieces of a key, 16-dimension tiles, LDS row
    __shared__ float gathered[WAVES][16][ROW];
    __shared__ float tops[WAVES][16 * NT], sums[WAVES][16 * NT];

    const int split = blockIdx.x, tile = blockIdx.y / a.heads_kv, h = blockIdx.y - tile * a.heads_kv;
    const int b = a.order != CACHE_AS_GIVEN ? by_length(a, blockIdx.z, gridDim.z) : (int)blockIdx.z;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 16, g = lane / 16;
    const Rows rows = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens, a.max_q);
    const int columns = rows.count * a.group, c0 = 16 * NT * tile;
    if (c0 >= columns) return;
    const int keys = cached_keys(a.lens[b], a.max_len, a.capacity), share = share_keys(keys, a.splits, WAVES);
    if (split > 0 && split * (long long)share >= keys) return;
    const int last = min(c0 + 16 * NT, columns) - 1;
    const int most = visible_keys(keys, rows.count, last / a.group), least = visible_keys(keys, rows.count, c0 / a.group);
    const int from = split * share, to = min((int)min(from + (long long)share, (long long)most), most);

    // the queries, as the second operand: lane (col, g) holds elements 64 j + 16 g + 0..15 of its column's head, as integers of up to 127 * 256
    // steps, in two limbs of 8 bits: 256 high + low
    v4i high[NT][KC], low[NT][KC];
    float factor[NT];
    int limit[NT];
    bool spoiled[NT];      // a query that is not finite, with keys to see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = c0 + 16 * n + col, cc = min(c, columns - 1), t = cc / a.group;
        const T* p = static_cast<const T*>(a.Q) + (rows.first + t) * (size_t)a.ldq + (size_t)(h * a.group + cc - t * a.group) * D + 16 * g;
        limit[n] = visible_keys(keys, rows.count, t);
        typedef T v8 __attribute__((ext_vector_type(8)));
        v8 raw[KC][2];
        typedef uint16_t bits8 __attribute__((ext_vector_type(8)));
        bits8 most8 = {0, 0, 0, 0, 0, 0, 0, 0};      // magnitudes: without the sign the 16 bits of either type are in the order of their values
#pragma unroll
        for (int j = 0; j < KC; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[j][i][e] = (T)0.0f;
                if (64 * j + 16 * g < D) raw[j][i] = *reinterpret_cast<const v8*>(p + 64 * j + 8 * i);
                most8 = __builtin_elementwise_max(most8, __builtin_bit_cast(bits8, raw[j][i]) & (uint16_t)0x7fff);
            }
        uint16_t most_bits = most8[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) most_bits = max(most_bits, most8[e]);
        // no number counts as infinite: maxima would drop it
        float top = (float)__builtin_bit_cast(T, min(most_bits, (uint16_t)(DT == FQ_F16 ? 0x7c00 : 0x7f80)));
        // the power of two first: the largest magnitude to [1, 2) (or what there is below), so that no size of query over- or underflows
        top = over_groups_max(top);
        spoiled[n] = top == INFINITY && limit[n] > 0;
        const uint32_t power = min(max(__float_as_uint(top) >> 23, 1u), 253u);
        const float down = __uint_as_float((254u - power) << 23), up = __uint_as_float(power << 23);
        top *= down;
        const float steps = top > 0.0f ? 32512.0f / top : 0.0f;
        factor[n] = a.scale * LOG2E * (top * (1.0f / 32512.0f)) * up;
#pragma unroll
        for (int j = 0; j < KC; ++j)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                // rounded to integers by the addition of 1.5 * 2^23, whose sums have steps of 1: the value's low bits are the integer's.  With
                // 128 more the second byte is the high limb and the first the low one, plus 128.
                uint32_t v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = __float_as_uint(__builtin_fmaf((float)raw[j][w / 2][4 * (w % 2) + e] * down, steps, 0x1.8p23f + 128.0f));
                const uint32_t front = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), back = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u);
                low[n][j][w] = (int)(__builtin_amdgcn_perm(back, front, 0x05040100u) ^ 0x80808080u);
                high[n][j][w] = (int)__builtin_amdgcn_perm(back, front, 0x07060302u);
            }
    }

    v4f o[NT][VT];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = LOWEST;
        sum[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < VT; ++t) o[n][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Where a step's keys lie.  A page that does not exist becomes page 0 with none of its keys visible and scales of 0.
    struct Step {
        const int8_t *keys, *values;
        float k_scale, v_scale;
        bool exists;
    };
    const size_t block = (size_t)a.page * D;
    const int32_t* table = a.table + (size_t)b * a.width;
    const int key_at = (16 * (col / 4) + col % 4) * D + 16 * g, value_at = col * a.page + 16 * g;
    const auto place = [&](int k0, int page) {
        const int off = k0 & (a.page - 1);
        const bool exists = page >= 0 && page < a.pages;
        const size_t at = (size_t)(exists ? page : 0) * a.heads_kv + h;
        return Step{a.k_cache + at * block + (size_t)off * D, a.v_cache + at * block + off, exists ? scalar(a.k_scale, at) : 0.0f, exists ? scalar(a.v_scale, at) : 0.0f, exists};
    };
    v4u kraw[4][KC], vraw[VT];
    const auto load_keys = [&](const Step& at) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < KC; ++j) {
                if (D % 64 != 0 && j == KC - 1) kraw[t][j] = v4u{0, 0, 0, 0};
                if (D % 64 == 0 || j < KC - 1 || 64 * j + 16 * g < D) kraw[t][j] = *reinterpret_cast<const v4u*>(at.keys + key_at + 4 * t * D + 64 * j);
            }
    };
    const auto load_values = [&](const Step& at) {
#pragma unroll
        for (int t = 0; t < VT; ++t) vraw[t] = *reinterpret_cast<const v4u*>(at.values + value_at + 16 * t * a.page);
    };

    // Both operands of a step are on their way while the step before it is worked on, its page number one step earlier still; behind the
    // last step it again, which costs less than a branch around the loads (the compiler then waits for all of them on either side).
    const int first = from + wave * CACHE_STEP, steps = first < to ? (to - 1 - first) / ROUND : -1, final = first + steps * ROUND;
    Step now{};
    int page_after = -1;
    if (steps >= 0) {
        now = place(first, scalar(table, first >> a.page_shift));
        load_keys(now);
        load_values(now);
        page_after = scalar(table, min(first + ROUND, final) >> a.page_shift);
    }
    for (int k0 = first; k0 < to; k0 += ROUND) {
        const Step next = place(min(k0 + ROUND, final), page_after);
        page_after = scalar(table, min(k0 + 2 * ROUND, final) >> a.page_shift);
        const float ks = now.k_scale, vs = now.v_scale;

        v4f s[NT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                v4i hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < KC; ++j) {
                    const v4i k = __builtin_bit_cast(v4i, kraw[t][j]);
                    hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, high[n][j], hi, 0, 0, 0);
                    lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, low[n][j], lo, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][t][i] = (float)((hi[i] << 8) + lo[i]);      // below 2^30
            }

        __builtin_amdgcn_sched_barrier(0);
        load_keys(next);
        __builtin_amdgcn_sched_barrier(0);

        v8h p[NT][LIMBS][2];
        float step_sum[NT], unit[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float f = fmaxf(factor[n] * ks, 0x1p-126f);      // not 0: that times a masked score would be no number
            if (k0 + CACHE_STEP > least || !now.exists) {
                asm volatile("");      // a branch
                const int left = now.exists ? limit[n] - k0 - 16 * g : 0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * t + i >= left) s[n][t][i] = -INFINITY;
            }
            float m = s[n][0][0];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, s[n][t][i]);
            const float largest = over_groups_max(m);
            m = fmaxf(largest * f, LOWEST);
            float above = m - top[n];      // of large scores a single step can be more than the slack
            if (__ballot(above > SLACK)) {      // only where it is so: a column's result does not depend on its neighbours
                const float rise = above > SLACK ? above : 0.0f, keep = __builtin_amdgcn_exp2f(-rise);
                top[n] = above > SLACK ? m : top[n];
                above -= rise;
                sum[n] *= keep;
#pragma unroll
                for (int t = 0; t < VT; ++t) o[n][t] *= keep;
            }
            // P's 1 is 2^7 (at most 2^15 with the slack).  Far below the running maximum it is the step's own largest weight that becomes 2^7, and the
            // product is turned to the running unit in 32 bits.  (In every step: 2 x 131072 tokens 98 us instead of 93, as a wave waits for its own
            // chain of instructions there.)
            const bool apart = above < -SLACK || fabsf(m) > FAR;
            float base = top[n] - STEP_SHIFT;
            unit[n] = STEP_UNIT;
            if (__builtin_expect(__ballot(apart) != 0, false)) {
                asm volatile("");      // a branch
                const float below = above < -SLACK ? above : 0.0f, less = apart ? fmaxf(largest, LOWEST) : 0.0f;
                unit[n] = __builtin_amdgcn_exp2f(below - STEP_SHIFT);
                base = apart ? below - above - STEP_SHIFT : base;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][t][i] -= less;
            }
            float add = 0.0f;
            const v2h ones = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    float w[2] = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][t][i], f, -base)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][t][i + 1], f, -base))};
#pragma unroll
                    for (int l = 0; l < LIMBS; ++l) {
                        const v2h e = {(_Float16)w[0], (_Float16)w[1]};
                        add = __builtin_amdgcn_fdot2(e, ones, add, false);      // of the rounded ones: they weigh the values
                        p[n][l][t / 2][4 * (t % 2) + i] = e[0];
                        p[n][l][t / 2][4 * (t % 2) + i + 1] = e[1];
                        w[0] -= (float)e[0];
                        w[1] -= (float)e[1];
                    }
                }
            step_sum[n] = over_groups_sum(add);
            sum[n] = __builtin_fmaf(step_sum[n], unit[n], sum[n]);
        }

#pragma unroll
        for (int t = 0; t < VT; ++t) {
            const v8h v0 = widen8(vraw[t][0], vraw[t][1]), v1 = widen8(vraw[t][2], vraw[t][3]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float start = -WIDEN_BIAS * step_sum[n], to_sum = vs * unit[n];
                v4f r = {start, start, start, start};
#pragma unroll
                for (int l = 0; l < LIMBS; ++l) {
                    r = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][l][0], r, 0, 0, 0);
                    r = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][l][1], r, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][t][i] = __builtin_fmaf(r[i], to_sum, o[n][t][i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        load_values(next);
        __builtin_amdgcn_sched_barrier(0);
        now = next;
    }

    // the waves' shares meet in LDS, one tile of columns after the other
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (g == 0) {
            tops[wave][16 * n + col] = top[n];
            sums[wave][16 * n + col] = sum[n];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
        float m = tops[0][16 * n + col];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, tops[w][16 * n + col]);
        // a spoiled query's integers mean nothing, and its result is to show that: no product with this is finite
        const float mine = spoiled[n] ? INFINITY : __builtin_amdgcn_exp2f(top[n] - m);
#pragma unroll
        for (int t = 0; t < VT; ++t) *reinterpret_cast<v4f*>(&gathered[wave][col][16 * t + 4 * g]) = o[n][t] * mine;
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += 64 * WAVES) {
            const int cl = i / (D / 4), d = (i - cl * (D / 4)) * 4, c = c0 + 16 * n + cl;
            if (c >= columns) continue;
            float best = tops[0][16 * n + cl], l = 0.0f;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) best = fmaxf(best, tops[w][16 * n + cl]);
            v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                l += sums[w][16 * n + cl] * __builtin_amdgcn_exp2f(tops[w][16 * n + cl] - best);
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

// The shares of one (row, head) joined: what is left is latency and, for many rows, the parts' bytes.

// Up to MOST shares: half a wave to a (row, head), four elements a lane, or to COLUMNS heads in a row where there are few shares; every load that
// a lane makes is on its way before the first is awaited.  Grid: x the heads, y the query tokens, z the sequences.
constexpr int JOIN_THREADS = 256, JOIN_FEW = 16;
constexpr int join_columns(int most) { return most == 2 ? 2 : 1; }
template <int DT, int D, int MOST> __global__ __launch_bounds__(JOIN_THREADS) void attn_cache_join_kernel(const CacheAttn a)
{
    typedef typename Stored<DT>::type T;
    typedef T v4 __attribute__((ext_vector_type(4)));
    constexpr int COLUMNS = join_columns(MOST);
    const int b = blockIdx.z, t = blockIdx.y, d = 4 * (threadIdx.x % 32);
    const int first = scalar(a.cu_q, b), behind = scalar(a.cu_q, b + 1), len = scalar(a.lens, b);
    const Rows rows = packed_rows(first, behind, a.tokens, a.max_q);
    const int head = (blockIdx.x * (JOIN_THREADS / 32) + threadIdx.x / 32) * COLUMNS;
    if (t >= rows.count || head >= a.heads_q || d >= D) return;
    const int keys = cached_keys(len, a.max_len, a.capacity), used = shares_used(keys, share_keys(keys, a.splits, a.round));

    v2f stat[COLUMNS][MOST];
    v4f part[COLUMNS][MOST];
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c)
#pragma unroll
        for (int s = 0; s < MOST; ++s) {
            const size_t at = ((size_t)(rows.first + t) * a.heads_q + min(head + c, a.heads_q - 1)) * a.splits + max(min(s, used - 1), 0);
            stat[c][s] = *reinterpret_cast<const v2f*>(a.stat + 2 * at);
            part[c][s] = *reinterpret_cast<const v4f*>(a.part + at * D + d);
        }
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c) {
        float best = -INFINITY, l = 0.0f;
        v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < MOST; ++s) best = fmaxf(best, s < used ? stat[c][s][0] : -INFINITY);
        if (best == -INFINITY) best = 0.0f;
#pragma unroll
        for (int s = 0; s < MOST; ++s)
            if (s < used) {
                const float w = __builtin_amdgcn_exp2f(stat[c][s][0] - best);
                l += stat[c][s][1] * w;
                y += part[c][s] * w;
            }
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        v4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = (T)(y[e] * inv);
        if (head + c < a.heads_q) *reinterpret_cast<v4*>(static_cast<T*>(a.Y) + (size_t)(rows.first + t) * a.ldy + (size_t)(head + c) * D + d) = out;
    }
}

// More shares: a workgroup to a (row, head), half a wave to a share.  Grid: x the heads, y the query tokens, z the sequences.
template <int DT, int D> __global__ __launch_bounds__(JOIN_THREADS) void attn_cache_join_many_kernel(const CacheAttn a)
{
    typedef typename Stored<DT>::type T;
    constexpr int WAVES = JOIN_THREADS / 64, SLOTS = 2 * WAVES, TURNS = MAX_SPLITS / 64;
    __shared__ v4f met[WAVES][32];
    const int b = blockIdx.z, t = blockIdx.y, wave = threadIdx.x / 64, lane = threadIdx.x % 64, head = blockIdx.x;
    const int first = scalar(a.cu_q, b), behind = scalar(a.cu_q, b + 1), len = scalar(a.lens, b);
    const Rows rows = packed_rows(first, behind, a.tokens, a.max_q);
    if (t >= rows.count) return;      // the whole workgroup
    const int keys = cached_keys(len, a.max_len, a.capacity), used = shares_used(keys, share_keys(keys, a.splits, a.round));
    const size_t at = ((size_t)(rows.first + t) * a.heads_q + head) * a.splits;
    float top[TURNS], sum[TURNS], best = -INFINITY, l = 0.0f;
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
        const int s = 64 * k + lane;
        top[k] = s < used ? a.stat[2 * (at + s)] : -INFINITY;
        sum[k] = s < used ? a.stat[2 * (at + s) + 1] : 0.0f;
        best = fmaxf(best, top[k]);
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) best = fmaxf(best, __shfl_xor(best, s));
    if (best == -INFINITY) best = 0.0f;
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
        top[k] = __builtin_amdgcn_exp2f(top[k] - best);      // the share's weight
        l += sum[k] * top[k];
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) l += __shfl_xor(l, s);
    v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
    const int d = 4 * (lane % 32), slot = wave * 2 + lane / 32;
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
        if (64 * k >= used) break;
        v4f part[64 / SLOTS];
#pragma unroll
        for (int i = 0; i < 64 / SLOTS; ++i) part[i] = *reinterpret_cast<const v4f*>(a.part + (at + min(64 * k + SLOTS * i + slot, used - 1)) * D + min(d, D - 4));
#pragma unroll
        for (int i = 0; i < 64 / SLOTS; ++i) {
            const float w = __shfl(top[k], SLOTS * i + slot);
            if (64 * k + SLOTS * i + slot < used) y += part[i] * w;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], 32);
    if (lane < 32) met[wave][lane] = y;
    __syncthreads();
    y = met[0][lane % 32];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) y += met[w][lane % 32];
    if (d >= D || slot > 0) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    typedef T v4 __attribute__((ext_vector_type(4)));
    v4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)(y[e] * inv);
    *reinterpret_cast<v4*>(static_cast<T*>(a.Y) + (size_t)(rows.first + t) * a.ldy + (size_t)head * D + d) = out;
}

template <int DT, int D, int MOST> void join(const CacheAttn& a, int batch, hipStream_t stream)
{
    const int heads = JOIN_THREADS / 32 * join_columns(MOST);      // of a workgroup
    attn_cache_join_kernel<DT, D, MOST><<<dim3((unsigned)((a.heads_q + heads - 1) / heads), (unsigned)std::min(a.max_q, a.tokens), (unsigned)batch), JOIN_THREADS, 0, stream>>>(a);
}

template <int DT, int D> int launch(const CacheAttn& a, int tiles, int batch, int blocks, unsigned wide_grid, hipStream_t stream)
{
    const dim3 grid((unsigned)a.splits, (unsigned)(a.heads_kv * blocks), (unsigned)batch);
    if (tiles * 16 == WIDE_COLUMNS) {
        const int rc = launch_attn_cache_wide(a, DT, D, batch, wide_grid, stream);
        if (rc) return rc;
    } else if (tiles == 1 && a.round == 2) attn_cache_kernel<DT, D, 1, 2><<<grid, 128, 0, stream>>>(a);
    else if (tiles == 1) attn_cache_kernel<DT, D, 1, 4><<<grid, 256, 0, stream>>>(a);
    else attn_cache_kernel<DT, D, 2, 4><<<grid, 256, 0, stream>>>(a);
    if (a.splits > JOIN_FEW) attn_cache_join_many_kernel<DT, D><<<dim3((unsigned)a.heads_q, (unsigned)std::min(a.max_q, a.tokens), (unsigned)batch), JOIN_THREADS, 0, stream>>>(a);
    else if (a.splits > 4) join<DT, D, JOIN_FEW>(a, batch, stream);
    else if (a.splits > 2) join<DT, D, 4>(a, batch, stream);
    else if (a.splits > 1) join<DT, D, 2>(a, batch, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "cache attention launch failed: %s", hipGetErrorString(e));
}

template <int DT> int launch_dim(const CacheAttn& a, int tiles, int head_dim, int batch, int blocks, unsigned wide_grid, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch<DT, 64>(a, tiles, batch, blocks, wide_grid, stream);
    case 80: return launch<DT, 80>(a, tiles, batch, blocks, wide_grid, stream);
    case 96: return launch<DT, 96>(a, tiles, batch, blocks, wide_grid, stream);
    default: return launch<DT, 128>(a, tiles, batch, blocks, wide_grid, stream);
    }
}

}  // namespace

int launch_attn_cache(const void* Q, int x_dtype, int tokens, int heads_q, int heads_kv, int head_dim, long long ldq, const int32_t* cu_q,
                      const int32_t* lens, int batch, int max_q, int max_len, const int8_t* k_cache, const int8_t* v_cache,
                      const float* k_scale, const float* v_scale, int pages, int page_size, const int32_t* page_table, int table_width,
                      float scale, void* Y, long long ldy, void* workspace, hipStream_t stream)
{
    const CachePlan plan = cache_plan(batch, tokens, max_q, max_len, heads_q, heads_kv);
    const int splits = plan.splits;
    float* part = static_cast<float*>(workspace);
    float* stat = part + (splits > 1 ? (size_t)tokens * heads_q * splits * head_dim : 0);
    const CacheAttn a{Q, Y, ldq, ldy, cu_q, lens, page_table, k_cache, v_cache, k_scale, v_scale, part, stat, scale, tokens, max_q, max_len,
                      heads_q, heads_kv, heads_q / heads_kv, table_width * page_size, pages, page_size,
                      page_size == 128 ? 7 : 6, table_width, splits, plan.round, plan.order};
    const int blocks = plan.tiles > 2 ? 1 : (int)plan.places;
    const unsigned wide_grid = (unsigned)tile_workgroups(plan.places, splits, heads_kv);
    return x_dtype == FQ_F16 ? launch_dim<FQ_F16>(a, plan.tiles, head_dim, batch, blocks, wide_grid, stream)
                             : launch_dim<FQ_BF16>(a, plan.tiles, head_dim, batch, blocks, wide_grid, stream);
}

}  // namespace fq
