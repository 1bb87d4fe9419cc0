// fq_attn_cache for many columns (query token, head of the group): pieces of a prompt that follow what the cache holds.
//
// Here every key serves many columns and the matrix pipe bounds the call, so the codes are widened to fp16 once per workgroup, on
// their way into LDS, and the rest is the prompt's attention (fq_attn_prompt.hip): 128 columns of one sequence and key head, 32 a wave,
// tiles of 64 keys, S^T = K Q^T and O^T += V^T P with P as it lies in the scores' registers.  A tile lies in one page:
//   its keys' scale goes into the factor of the scores; the keys stay 1152 too large each (see widen8), which adds 1152 times the sum of
//     the query's elements to every score of a column and is taken off where the maximum is;
//   its values' scale goes into P as an addend of the exponent.  So P's unit, which the accumulators count in, is the largest product of a weight and
//     a scale so far, kept apart from the largest weight, which the sum counts in: whatever the scales, neither is ever changed to something
//     smaller, and what fp16 cannot hold of a P (HALF_SHIFT) is little beside the largest one's products.
// Measured: 512 tokens behind 7680, 64 heads of 128 over 8 (256 workgroups of columns, keys in two shares): 153 to 163 us for the call, 0.85 PFLOP/s at 1.7 GHz
// (under the profiler, with launches further apart, 157 and 8.4 for the join); the matrix pipe is busy for 48 % of the cycles, the vector pipe for 58 %: 240
// vector instructions a tile and wave beside 32 products, a third of them to widen and store its part of the codes.  By 64 columns straight from registers, as the
// kernel for few columns works, 268 us (where that one is faster all the same: cache_plan).
#include "fq_attn_cache.h"

namespace fq {
namespace {

constexpr int WIDE_WAVES = WIDE_COLUMNS / 32, WIDE_THREADS = 64 * WIDE_WAVES;

// Where piece 2 e + half of row r lies among its row's C: both the eight lanes that write neighbouring pairs' first (or second) pieces and the
// 16 rows that are read at a time, the same piece of each, then meet all banks.  (Widths of 10 and 12 pieces are only turned for the reads.)
constexpr int pair_place(int C, int r, int e, int half)
{
    return C == 16 ? (e + r) % 8 + 8 * ((half + r / 8) % 2) : C == 8 ? (e + 4 * ((half + r) % 2) + r / 2) % 8 : (2 * e + half + key_turn(C, r)) % C;
}

// The tile of columns at a place: of which sequence; of none: -1.  Of at most 64 sequences the longest come first.
struct WideTile {
    int sequence, nth;
};
__device__ __forceinline__ WideTile tile_at(const CacheAttn& a, int batch, int place)
{
    const int lane = threadIdx.x % 64;
    const auto tiles_of = [&](int b) { return (packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens, a.max_q).count * a.group + WIDE_COLUMNS - 1) / WIDE_COLUMNS; };
    if (batch <= SORTED_SEQUENCES) {
        const int j = min(lane, batch - 1), len = a.lens[j], tiles = lane < batch ? tiles_of(j) : 0, before = sum_of_longer(length_key(len), tiles, batch);
        const uint64_t here = __ballot(place >= before && place - before < tiles);
        const int from = here ? __builtin_ctzll(here) : 0;
        return {here ? from : -1, place - __builtin_amdgcn_readlane(before, from)};
    }
    const auto first = [&](int b) { return first_place((long long)min(max(a.cu_q[b], 0), a.tokens) * a.group, WIDE_COLUMNS, b); };
    const int b = sequence_at(place, batch, first), nth = place - first(b);
    return {nth >= 0 && nth < tiles_of(b) ? b : -1, nth};
}

template <int DT, int D> __global__ __launch_bounds__(WIDE_THREADS, 2) void attn_cache_wide_kernel(const CacheAttn a, int batch)
{
    typedef typename Stored<DT>::type T;
    typedef Mma<FQ_F16> M;
    constexpr int KS = D / 16, VT = (D + 31) / 32, C = D / 8, ROW = 2 * D, KTILE = CACHE_STEP * ROW, VROW = 2 * CACHE_STEP, VTILE = 32 * VT * VROW;
    constexpr int PIECES = (CACHE_STEP * D / 16 + WIDE_THREADS - 1) / WIDE_THREADS;      // 16 codes each, of keys and of values, per thread
    constexpr bool EVEN = CACHE_STEP * D / 16 % WIDE_THREADS == 0;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * (KTILE + VTILE)];            // [keys, two stages][values, two stages]

    // The tiles of a share next to each other: 64 tokens behind 8128, 64 heads over 8, 39 us; the shares of a tile so, 42.
    const unsigned of_share = gridDim.x / a.splits;      // whole eights
    const int split = blockIdx.x / of_share;
    const TileUnit work = tile_unit(blockIdx.x - split * of_share, 1, (unsigned)a.heads_kv);
    const int h = work.head_kv;
    const WideTile at_tile = tile_at(a, batch, work.place);
    const int b = at_tile.sequence;
    if (b < 0) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 32, half = lane / 32;
    const Rows rows = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens, a.max_q);
    const int columns = rows.count * a.group, c0 = at_tile.nth * WIDE_COLUMNS;
    const int keys = cached_keys(a.lens[b], a.max_len, a.capacity), share = share_keys(keys, a.splits, a.round);
    if (split > 0 && split * (long long)share >= keys) return;
    const auto visible = [&](int c) { return visible_keys(keys, rows.count, min(c, columns - 1) / a.group); };
    const int w0 = c0 + 32 * wave, c = w0 + col, cc = min(c, columns - 1), token = cc / a.group, head = h * a.group + cc - token * a.group;
    const int from = split * share, to = (int)min(from + (long long)share, (long long)visible(c0 + WIDE_COLUMNS - 1));
    const int mine = visible(c), least = visible(w0), tiles = to > from ? (to - from + CACHE_STEP - 1) / CACHE_STEP : 0;
    const int wave_to = w0 >= columns ? from : min(to, visible(w0 + 31)), own = wave_to > from ? (wave_to - from + CACHE_STEP - 1) / CACHE_STEP : 0;

    // the queries in fp16: lane (col, half) holds elements 16 e + 8 half + 0..7 of its column's head
    v8h q[KS];
    float factor = a.scale * LOG2E, bias = 0.0f;
    {
        typedef T v8 __attribute__((ext_vector_type(8)));
        const T* p = static_cast<const T*>(a.Q) + (rows.first + (size_t)token) * a.ldq + (size_t)head * D + 8 * half;
        v8 raw[KS];
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < KS; ++e) {
            raw[e] = *reinterpret_cast<const v8*>(p + 16 * e);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf((float)raw[e][i]));
        }
        if constexpr (DT == FQ_F16) {
#pragma unroll
            for (int e = 0; e < KS; ++e) q[e] = raw[e];
        } else {
            // the largest magnitude to [1, 4): what fp16 cannot hold then is below 2^-24 of it
            const uint32_t power = min(max(__float_as_uint(over_halves_max(top)) >> 23, 1u), 253u);
            const float down = __uint_as_float((254u - power) << 23);
            factor *= __uint_as_float(power << 23);
#pragma unroll
            for (int e = 0; e < KS; ++e)
#pragma unroll
                for (int i = 0; i < 8; ++i) q[e][i] = (_Float16)((float)raw[e][i] * down);
        }
        const v2h ones = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
        for (int e = 0; e < KS; ++e)
#pragma unroll
            for (int i = 0; i < 8; i += 2) bias = __builtin_amdgcn_fdot2(v2h{q[e][i], q[e][i + 1]}, ones, bias, false);
        bias = WIDEN_BIAS * over_halves_sum(bias);
    }

    // Where a tile lies; behind the last tile it again.  A page that does not exist: page 0 with none of its keys visible and scales of 0.
    struct Place {
        const int8_t *keys, *values;
        float k_scale, v_scale;
        bool exists;
    };
    const size_t page_bytes = (size_t)a.page * D;
    const int32_t* table = a.table + (size_t)b * a.width;
    const auto first_key = [&](int i) { return from + CACHE_STEP * min(i, tiles - 1); };
    const auto page_of = [&](int i) { return scalar(table, first_key(i) >> a.page_shift); };
    const auto place = [&](int i, int page) {
        const int off = first_key(i) & (a.page - 1);
        const bool exists = page >= 0 && page < a.pages;
        const size_t at = (size_t)(exists ? page : 0) * a.heads_kv + h;
        return Place{a.k_cache + at * page_bytes + (size_t)off * D, a.v_cache + at * page_bytes + off, exists ? scalar(a.k_scale, at) : 0.0f,
                     exists ? scalar(a.v_scale, at) : 0.0f, exists};
    };
    // What a thread has under way: two tiles of each, those of even and those of odd number.
    v4u kreg[2][PIECES], vreg[2][PIECES];
    const uint32_t key_from = 16 * tid, value_from = tid / 4 * a.page + 16 * (tid % 4);
    const auto load_keys = [&](const Place& at, v4u (&reg)[PIECES]) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (EVEN || p * WIDE_THREADS + tid < CACHE_STEP * D / 16) reg[p] = *reinterpret_cast<const v4u*>(at.keys + p * 16 * WIDE_THREADS + key_from);
        }
    };
    const auto load_values = [&](const Place& at, v4u (&reg)[PIECES]) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (EVEN || p * WIDE_THREADS + tid < 4 * D) reg[p] = *reinterpret_cast<const v4u*>(at.values + p * (WIDE_THREADS / 4) * a.page + value_from);
        }
    };
    // A row of keys holds 16-byte pieces of the head's elements; a row of values the 64 keys of a dimension, of each 16 first 0..3, 8..11, then
    // 4..7, 12..15: what a lane of either half needs for a product lies together.  A thread writes two neighbouring pieces.
    const auto key_put = [&](int i, int j) { return i / (D / 16) * ROW + pair_place(C, i / (D / 16), i % (D / 16), j) * 16; };
    const auto value_put = [&](int i, int j) { return 2 * KTILE + i / 4 * VROW + pair_place(8, i / 4, i % 4, j) * 16; };
    const int key_puts[2] = {key_put(tid, 0), key_put(tid, 1)}, value_puts[2] = {value_put(tid, 0), value_put(tid, 1)};
    const auto put_keys = [&](int stage, const v4u (&reg)[PIECES], int p, int j) {
        const int i = p * WIDE_THREADS + tid;
        if (!EVEN && i >= CACHE_STEP * D / 16) return;
        // whole rows, a multiple of 32, from one of a thread's pieces to the next: in the same places
        const int at = EVEN ? key_puts[j] + p * (16 * WIDE_THREADS / D) * ROW : key_put(i, j);
        *reinterpret_cast<v8h*>(lds + stage * KTILE + at) = widen8(reg[p][2 * j], reg[p][2 * j + 1]);
    };
    const auto put_values = [&](int stage, const v4u (&reg)[PIECES], int p, int j) {
        if (!EVEN && p * WIDE_THREADS + tid >= 4 * D) return;
        *reinterpret_cast<v8h*>(lds + stage * VTILE + value_puts[j] + p * (WIDE_THREADS / 4) * VROW) = widen8(reg[p][j], reg[p][j + 2]) - (_Float16)WIDEN_BIAS;
    };
    const auto put_all_keys = [&](int stage, const v4u (&reg)[PIECES]) {
#pragma unroll
        for (int p = 0; p < 2 * PIECES; ++p) put_keys(stage, reg, p / 2, p % 2);
    };
    const auto put_all_values = [&](int stage, const v4u (&reg)[PIECES]) {
#pragma unroll
        for (int p = 0; p < 2 * PIECES; ++p) put_values(stage, reg, p / 2, p % 2);
    };
    // Piece n of those that a thread puts in a step: keys for stage `odd`, values for the other.
    constexpr int PUTS = 4 * PIECES;
    const auto put = [&](int odd, int n) {
        if (n < PUTS / 2) put_keys(odd, kreg[odd], n / 2, n % 2);
        else put_values(1 - odd, vreg[1 - odd], (n - PUTS / 2) / 2, n % 2);
    };

    v16f o[VT], s[2];
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    float top = LOWEST, sum = 0.0f;                      // of the scaled scores; over this lane's keys
    float unit = LOWEST;                                 // log2 of what o counts in, weights times values' scales, less top
    v8h p[4];                                            // 16 keys each

    uint32_t key_at[KS], value_at[4];
#pragma unroll
    for (int e = 0; e < KS; ++e) key_at[e] = col * ROW + pair_place(C, col, e, half) * 16;
#pragma unroll
    for (int n = 0; n < 4; ++n) value_at[n] = 2 * KTILE + col * VROW + pair_place(8, col, n, half) * 16;

    // O^T += V^T P of a tile (PV), then S^T of the next (QK); first operands come from LDS AHEAD - 1 products early, the order is kept
    const auto products = [&](auto with_pv, auto with_qk, auto odd, auto between) {      // odd: whether the values' tile has an odd number
        constexpr int VSTAGE = decltype(odd)::value, KSTAGE = 1 - VSTAGE;
        constexpr int PV = decltype(with_pv)::value ? 4 * VT : 0, N = PV + (decltype(with_qk)::value ? 2 * KS : 0), AHEAD = 4;
        v8h ring[AHEAD];
        const auto fetch = [&](int n) {
            const uint32_t at = n < PV ? value_at[n / VT] + VSTAGE * VTILE + 32 * (n % VT) * VROW : key_at[(n - PV) / 2] + KSTAGE * KTILE + 32 * ((n - PV) % 2) * ROW;
            ring[n % AHEAD] = *reinterpret_cast<const v8h*>(lds + at);
        };
#pragma unroll
        for (int n = 0; n < AHEAD - 1; ++n) fetch(n);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (n + AHEAD - 1 < N) fetch(n + AHEAD - 1);
            __builtin_amdgcn_sched_barrier(0);
            if (n < PV) {
                o[n % VT] = M::mul(ring[n % AHEAD], p[n / VT], o[n % VT]);
            } else {
                const int e = (n - PV) / 2, t = (n - PV) % 2;
                if (e == 0)
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[t][k] = 0.0f;
                s[t] = M::mul(ring[n % AHEAD], q[e], s[t]);
            }
            between(n);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto nothing = [](int) {};
    const std::true_type yes;
    const std::false_type no;
    const auto softmax = [&](int i, const Place& at) __attribute__((always_inline)) {
        const int k0 = from + CACHE_STEP * i;
        const float f = fmaxf(factor * at.k_scale, 0x1p-126f), shift = bias * f;      // f is not 0: that times a masked score would be no number
        if (k0 + CACHE_STEP > least || !at.exists) {
            asm volatile("");      // a branch
            const int left = at.exists ? mine - k0 - 4 * half : 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * t + 8 * (e / 4) + e % 4 >= left || !at.exists) s[t][e] = -INFINITY;
        }
        float m = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) m = fmaxf(fmaxf(m, s[0][e]), s[1][e]);
        m = over_halves_max(m);
        const float largest = fmaxf(m, LOWEST);
        m = fmaxf(__builtin_fmaf(m, f, -shift), LOWEST);      // infinite where none is visible: LOWEST whatever f
        const float log_scale = fmaxf(__builtin_amdgcn_logf(at.v_scale), -200.0f);      // below 2^-126: 0, which counts as 2^-200
        float above = m - top;
        if (__ballot(above > HALF_SLACK || above + log_scale > unit + HALF_SLACK)) {
            const float rise = fmaxf(above, 0.0f);
            top = fmaxf(m, top);
            above -= rise;
            sum *= __builtin_amdgcn_exp2f(-rise);
            const float now = fmaxf(above + log_scale, unit - rise), keep = __builtin_amdgcn_exp2f(unit - rise - now);
            unit = now;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[t] *= keep;
        }
        // from the tile's largest weight to that with P = 1; where its P are too small for fp16, 2^60 at most, so that the sum still counts them
        const float to_one = fminf(unit - log_scale - above, 60.0f) - HALF_SHIFT;
        float off = __builtin_fmaf(largest, f, to_one);
        if (__ballot(fabsf(off) > FAR)) {
            asm volatile("");
            const float less = fabsf(off) > FAR ? largest : 0.0f;
            off = fabsf(off) > FAR ? to_one : off;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] -= less;
        }
        float add = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], f, -off));
                add += w;
                p[2 * t + e / 8][e % 8] = (_Float16)w;
            }
        sum = __builtin_fmaf(add, __builtin_amdgcn_exp2f(to_one + above), sum);
    };

    // Step i: what has arrived goes into LDS (keys of tile i + 2, values of i + 1), more is asked for (keys of i + 4, values of i + 3), PV of
    // tile i, QK and softmax of i + 1
    if (tiles > 0) {
        Place now = place(0, page_of(0)), line[3] = {place(1, page_of(1)), place(2, page_of(2)), place(3, page_of(3))};      // line: tiles i + 1 .. i + 3
        load_keys(now, kreg[0]);
        load_values(now, vreg[0]);
        load_keys(line[0], kreg[1]);
        put_all_keys(0, kreg[0]);
        put_all_values(0, vreg[0]);
        put_all_keys(1, kreg[1]);
        // in the order of the steps' loads, so that a step waits for no later one
        __builtin_amdgcn_sched_barrier(0);
        load_keys(line[1], kreg[0]);
        __builtin_amdgcn_sched_barrier(0);
        load_values(line[0], vreg[1]);
        __builtin_amdgcn_sched_barrier(0);
        load_keys(line[2], kreg[1]);
        __builtin_amdgcn_sched_barrier(0);
        load_values(line[1], vreg[0]);
        __builtin_amdgcn_sched_barrier(0);
        Place fourth = place(4, page_of(4));
        int page_then = page_of(5);
        __syncthreads();
        if (own > 0) {
            products(no, yes, yes, nothing);
            softmax(0, now);
        }
        __syncthreads();
        int i = 0;
        const auto begin_step = [&](auto odd) {
            constexpr int O = decltype(odd)::value;
#pragma unroll
            for (int n = 0; n < PUTS; ++n) put(O, n);
            load_keys(fourth, kreg[O]);
            __builtin_amdgcn_sched_barrier(0);
            load_values(line[2], vreg[1 - O]);
        };
        const auto end_step = [&] {
            line[0] = line[1];
            line[1] = line[2];
            line[2] = fourth;
            fourth = place(i + 5, page_then);
            page_then = page_of(i + 6);
            ++i;
            __syncthreads();
        };
        const auto step = [&](auto odd) {
            constexpr int O = decltype(odd)::value, APART = (4 * VT + 2 * KS) / PUTS;
            __builtin_amdgcn_s_setprio(1);
            products(yes, yes, odd, [&](int n) {
                if (n % APART == APART - 1 && n / APART < PUTS) put(O, n / APART);
            });
            __builtin_amdgcn_s_setprio(0);
            load_keys(fourth, kreg[O]);
            __builtin_amdgcn_sched_barrier(0);
            load_values(line[2], vreg[1 - O]);
            softmax(i + 1, line[0]);
            end_step();
        };
        while (i + 2 < own) {
            step(no);
            step(yes);
        }
        if (i + 1 < own) step(no);
        if (own > 0) {
            if (i % 2) {
                begin_step(yes);
                products(yes, no, yes, nothing);
            } else {
                begin_step(no);
                products(yes, no, no, nothing);
            }
            end_step();
        }
        while (i < tiles) {
            if (i % 2) begin_step(yes);
            else begin_step(no);
            end_step();
        }
    }

    sum = over_halves_sum(sum);
    if (c >= columns) return;
    // Twice, as the whole may be beyond fp32 where a product with it is not.  Where the query is not finite (nor its sum then), no product with it is.
    const bool spoiled = (__float_as_uint(bias) & 0x7f800000u) == 0x7f800000u && mine > 0;
    const float half_unit = spoiled ? INFINITY : __builtin_amdgcn_exp2f(0.5f * (unit - HALF_SHIFT));
    const size_t row = rows.first + (size_t)token;
    if (a.splits > 1) {
        const size_t at = (row * a.heads_q + head) * a.splits + split;
        if (half == 0) {
            a.stat[2 * at] = top;
            a.stat[2 * at + 1] = sum;
        }
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (32 * t + 8 * e < D) *reinterpret_cast<v4f*>(a.part + at * D + 32 * t + 8 * e + 4 * half) =
                    v4f{o[t][4 * e], o[t][4 * e + 1], o[t][4 * e + 2], o[t][4 * e + 3]} * half_unit * half_unit;
        return;
    }
    const float inv = sum > 0.0f ? half_unit / sum : 0.0f;
    typedef T v4 __attribute__((ext_vector_type(4)));
    T* yp = static_cast<T*>(a.Y) + row * (size_t)a.ldy + (size_t)head * D + 4 * half;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (32 * t + 8 * e >= D) continue;
            v4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (T)(o[t][4 * e + i] * inv * half_unit);
            *reinterpret_cast<v4*>(yp + 32 * t + 8 * e) = y;
        }
}

template <int DT> int launch(const CacheAttn& a, int head_dim, int batch, unsigned grid, hipStream_t stream)
{
    switch (head_dim) {
    case 64: attn_cache_wide_kernel<DT, 64><<<grid, WIDE_THREADS, 0, stream>>>(a, batch); break;
    case 80: attn_cache_wide_kernel<DT, 80><<<grid, WIDE_THREADS, 0, stream>>>(a, batch); break;
    case 96: attn_cache_wide_kernel<DT, 96><<<grid, WIDE_THREADS, 0, stream>>>(a, batch); break;
    default: attn_cache_wide_kernel<DT, 128><<<grid, WIDE_THREADS, 0, stream>>>(a, batch); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FQ_OK : fail(FQ_ERR_HIP, "cache attention launch failed: %s", hipGetErrorString(e));
}

}  // namespace

int launch_attn_cache_wide(const CacheAttn& a, int x_dtype, int head_dim, int batch, unsigned grid, hipStream_t stream)
{
    return x_dtype == FQ_F16 ? launch<FQ_F16>(a, head_dim, batch, grid, stream) : launch<FQ_BF16>(a, head_dim, batch, grid, stream);
}

}  // namespace fq
