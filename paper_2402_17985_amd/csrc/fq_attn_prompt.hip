// fq_attn_prompt: attention over packed sequences of different lengths, causal or not, grouped heads.
//
// Bound by the matrix pipe for long sequences (4 D operations for every pair of a query and a key it sees).  One pass over the
// keys with the running maximum and sum of the softmax; a workgroup takes 128 queries of one head, 32 a wave, and walks the keys
// in tiles of 64 through LDS.
//   S^T = K Q^T   32 keys x 32 queries a product: a query's scores are in two lanes, so its maximum and sum need one exchange.
//   O^T += V^T P  the scores' registers are the second operand as they stand: which key of the tile stands at which place of the
//                 reduction is free as long as the values follow, and their transposed reads from LDS take four consecutive
//                 keys of a dimension, as a lane holds them.
// P is rounded to the input's type (the values' type has to match; its rounding is what the output's is), the row sums are taken before that in
// 32 bits.
// Two workgroups a CU (four for heads of 64), independent of each other: one's softmax runs beside the other's products.  Eight waves in one workgroup
// that take turns by barriers gave the same busy cycles (61 % of them the matrix pipe) and lost 12 % on prompts of 256.
// Measured: 8192 tokens, 64 heads of 128 over 8, causal, bf16: 0.95 to 1.05 ms, 1.05 to 1.15 PFLOP/s (a library product of 8192^3: 1.6); the pipe is busy for
// 68 % of the cycles at 1.4 to 1.6 GHz, the clock that the power limit leaves: variants of 4.1e8 to 5.4e8 busy CU cycles all took 1.04 to 1.18 ms.  Eight
// prompts of 438 to 2048 tokens, 40 heads: 225 us, 0.7 PFLOP/s, 43 % of the cycles: of a workgroup's 27 us 6 are the way to the first tile and the end, 3 or 4 more
// pass between two workgroups.  8 x 256 tokens, 32 heads: 16 us for 67 MB, 4.2 TB/s; of a workgroup's 11 us there 5 are the way to the first tile.
#include "fq_attn_common.h"

namespace fq {
namespace {

struct PromptAttn {
    const void *Q, *K, *V;
    void* Y;
    long long ldq, ldk, ldv, ldy;
    const int32_t *cu_q, *cu_k;
    float factor;            // scale * log2(e), positive
    int tokens_q, tokens_k, max_q, heads_q, heads_kv, group, causal, batch;
};

constexpr int PROMPT_KEYS = 64;   // a tile

// A tile in LDS is rows of D elements without gaps, as the direct copies from global memory fill it, with the 16-byte pieces of a
// row rotated: piece c of row r lies at place (c + turn(r)) mod (D / 8), so that rows that are read together lie on different banks
// (64 of them, 256 bytes).  Keys are read 16 rows at a time, the same piece of each; values 4 rows at a time, 4 pieces of each.
constexpr int value_turn(int C, int r) { return C == 16 ? r % 4 * 4 : C == 8 ? r % 4 / 2 * 4 : 0; }

// Four 2-byte elements of a column out of row-major LDS: of 16 neighbouring lanes, lanes 4 r .. 4 r + 3 point at 16 consecutive
// elements of row r, and lane i receives element i of the four rows.
__device__ __forceinline__ v2u read_transposed(uint32_t lds_address)
{
    typedef __attribute__((ext_vector_type(4))) __fp16 v4fp;
    typedef __attribute__((address_space(3))) v4fp* lds_ptr;
    const v4fp r = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_ptr)(uintptr_t)lds_address);
    return __builtin_bit_cast(v2u, r);
}

// 64 lanes times 16 bytes from global memory straight to LDS bytes [lds_base, + 1024) (lds_base is wave-uniform).
__device__ __forceinline__ void copy_to_lds(const void* uniform_base, uint32_t lane_offset, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(uniform_base), "v"(lane_offset), "s"(lds_base) : "memory");
}
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

// The tile of queries at a place; of none: -1.  Of at most 64 sequences those with the most keys come first: long ones begun last would run on
// alone (8 uneven prompts: 293 us as they come, 280 so).  All offsets are loaded at once, one sequence a lane, so that the order costs no further
// trip to memory; of more sequences the one at the place is searched.
struct PromptTile {
    Rows q, k;
    int tile;
};
__device__ __forceinline__ PromptTile tile_at(const PromptAttn& a, int place)
{
    const int lane = threadIdx.x % 64;
    const auto tiles_of = [](const Rows& q) { return (int)(((unsigned)q.count + PROMPT_ROWS - 1) / PROMPT_ROWS); };
    if (a.batch <= SORTED_SEQUENCES) {
        const int j = min(lane, a.batch - 1);
        const Rows k = packed_rows(a.cu_k[j], a.cu_k[j + 1], a.tokens_k, a.tokens_k), q = packed_rows(a.cu_q[j], a.cu_q[j + 1], a.tokens_q, a.max_q);
        const int tiles = lane < a.batch ? tiles_of(q) : 0;
        const int before = sum_of_longer(length_key(k.count), tiles, a.batch);
        const uint64_t here = __ballot(place >= before && place - before < tiles);
        const int from = here ? __builtin_ctzll(here) : 0, nth = place - __builtin_amdgcn_readlane(before, from);
        return {{__builtin_amdgcn_readlane(q.first, from), __builtin_amdgcn_readlane(q.count, from)},
                {__builtin_amdgcn_readlane(k.first, from), __builtin_amdgcn_readlane(k.count, from)},
                here ? __builtin_amdgcn_readlane(tiles, from) - 1 - nth : -1};
    }
    const auto first = [&](int b) { return first_place(min(max(a.cu_q[b], 0), a.tokens_q), PROMPT_ROWS, b); };
    const int b = sequence_at(place, a.batch, first);
    const Rows k = packed_rows(a.cu_k[b], a.cu_k[b + 1], a.tokens_k, a.tokens_k), q = packed_rows(a.cu_q[b], a.cu_q[b + 1], a.tokens_q, a.max_q);
    const int tiles = tiles_of(q), nth = place - first(b);
    return {q, k, nth >= 0 && nth < tiles ? tiles - 1 - nth : -1};
}

template <int DT, int D> __global__ __launch_bounds__(PROMPT_THREADS, D == 64 ? 4 : D <= 96 ? 3 : 2) void attn_prompt_kernel(const PromptAttn a)
{
    typedef Mma<DT> M;
    typedef typename M::T T;
    typedef typename M::v8 v8;
    constexpr int KS = D / 16, VT = (D + 31) / 32, C = D / 8, ROW = 2 * D, TILE = PROMPT_KEYS * ROW;
    constexpr int COPIES = (C + PROMPT_WAVES - 1) / PROMPT_WAVES;   // wave-wide copies per wave, operand and tile
    // [keys, two stages][values, two stages]; reads of the last 32 dimensions reach behind a row of 80
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TILE + 64];

    const TileUnit unit = tile_unit(blockIdx.x, (unsigned)a.group, (unsigned)a.heads_kv);
    const int hk = unit.head_kv, head = hk * a.group + unit.member;
    const PromptTile at = tile_at(a, unit.place);
    if (at.tile < 0) return;
    const Rows rq = at.q, rk = at.k;
    const int q0 = at.tile * PROMPT_ROWS;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 32, half = lane / 32;
    const int row = q0 + 32 * wave + col, keys = rk.count;
    const auto visible = [&](int i) { return a.causal ? visible_keys(keys, rq.count, i) : keys; };
    const int mine = visible(min(row, rq.count - 1)), least = visible(min(q0 + 32 * wave, rq.count - 1));
    const int wave_keys = q0 + 32 * wave >= rq.count ? 0 : visible(min(q0 + 32 * wave + 31, rq.count - 1)), most = visible(min(q0 + PROMPT_ROWS, rq.count) - 1);
    const int tiles = (most + PROMPT_KEYS - 1) / PROMPT_KEYS;

    // copies into LDS: each lane's places in a tile, and the piece of a row that belongs there (where the waves outnumber what is
    // left, several copy the same)
    const T *kp = static_cast<const T*>(a.K) + (size_t)rk.first * a.ldk + (size_t)hk * D, *vp = static_cast<const T*>(a.V) + (size_t)rk.first * a.ldv + (size_t)hk * D;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    uint32_t from_at[2][COPIES];
    const auto set_offsets = [&](int values, int i) {      // of tile i; for rows behind the last key that one
        const int last = min(keys - i * PROMPT_KEYS, PROMPT_KEYS) - 1;
#pragma unroll
        for (int p = 0; p < COPIES; ++p) {
            const int at = 64 * min(wave + PROMPT_WAVES * p, C - 1) + lane, r = at / C, turned = at - r * C - (values ? value_turn(C, r) : key_turn(C, r));
            from_at[values][p] = (uint32_t)min(r, last) * (uint32_t)(2 * (values ? a.ldv : a.ldk)) + 16 * (turned < 0 ? turned + C : turned);
        }
    };
    const auto copy = [&](int values, int i) {
        if ((i + 1) * PROMPT_KEYS > keys) set_offsets(values, i);      // the last tile
        const T* from = (values ? vp : kp) + (size_t)i * PROMPT_KEYS * (values ? a.ldv : a.ldk);
#pragma unroll
        for (int p = 0; p < COPIES; ++p)
            copy_to_lds(from, from_at[values][p], base + (2 * values + i % 2) * TILE + 1024 * min(wave + PROMPT_WAVES * p, C - 1));
    };

    if (tiles > 0) {
        set_offsets(0, 0);
        copy(0, 0);
    }
    const T* qp = static_cast<const T*>(a.Q) + (rq.first + (size_t)min(row, rq.count - 1)) * a.ldq + (size_t)head * D + 8 * half;
    v8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8*>(qp + 16 * s);

    if (tiles > 0) {
        set_offsets(1, 0);
        copy(1, 0);
        if (tiles > 1) copy(0, 1);
    }

    v16f o[VT], s[2];
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;      // of the unscaled scores; the sum over this lane's keys only
    v8 p[4];                                // 16 keys each

    uint32_t key_at[KS], value_at[VT];
#pragma unroll
    for (int e = 0; e < KS; ++e) key_at[e] = col * ROW + (2 * e + half + key_turn(C, col)) % C * 16;
    const int vr = lane % 16 / 4;
#pragma unroll
    for (int t = 0; t < VT; ++t) {
        const int piece = 4 * t + 2 * (lane / 16 % 2) + lane % 4 / 2;
        value_at[t] = base + 2 * TILE + (4 * half + vr) * ROW + (piece < C ? (piece + value_turn(C, vr)) % C : piece) * 16 + 8 * (lane % 2);
    }

    // The matrix work of a step: O^T += V^T P of tile i (PV), then S^T of tile i + 1 (QK).  Every product's first operand comes from LDS
    // AHEAD - 1 products early; the order is kept as written.  (Left to the compiler, each pair of transposed reads is awaited before the
    // next: 5.9e8 busy CU cycles for a causal prompt of 8192 tokens and 64 heads of 128, so 4.5e8.)
    const auto products = [&](auto with_pv, auto with_qk) {
        constexpr int PV = decltype(with_pv)::value ? 4 * VT : 0, N = PV + (decltype(with_qk)::value ? 2 * KS : 0), AHEAD = D == 64 ? 4 : 5;
        v8 ring[AHEAD];
        const auto fetch = [&](int n) {
            if (n < PV) {
                const uint32_t v = value_at[n % VT] + 16 * (n / VT) * ROW;
                const v2u lo = read_transposed(v), hi = read_transposed(v + 8 * ROW);
                ring[n % AHEAD] = __builtin_bit_cast(v8, (v4u{lo[0], lo[1], hi[0], hi[1]}));
            } else {
                ring[n % AHEAD] = *reinterpret_cast<const v8*>(lds + key_at[(n - PV) / 2] + 32 * ((n - PV) % 2) * ROW);
            }
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
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const std::true_type yes;
    const std::false_type no;
    // its probabilities
    constexpr float LAG = DT == FQ_F16 ? HALF_SLACK : SLACK, SHIFT = DT == FQ_F16 ? HALF_SHIFT : 0.0f;      // bf16 holds all that fp32 does
    float off = -SHIFT;            // what is taken off a scaled score: its maximum, or (far) nothing, as the unscaled one is taken off the score before
    bool any_far = false;          // in this wave
    const auto softmax = [&](int i) __attribute__((always_inline)) {
        const int k0 = i * PROMPT_KEYS;
        // register e of tile t: key 32 t + 8 (e / 4) + 4 half + e % 4
        if (k0 + PROMPT_KEYS > least) {
            asm volatile("");      // a branch: the comparisons are not worth making where they change nothing
            const int left = mine - k0 - 4 * half;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * t + 8 * (e / 4) + e % 4 >= left) s[t][e] = -INFINITY;
        }
        float m = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) m = fmaxf(fmaxf(m, s[0][e]), s[1][e]);
        m = over_halves_max(m);
        if (__ballot(top == -INFINITY || (m - top) * a.factor > LAG)) {
            const float now = fmaxf(m, top), keep = now == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((top - now) * a.factor);
            top = now;
            const bool far = fabsf(top * a.factor) > FAR && top != -INFINITY;
            off = (far || top == -INFINITY ? 0.0f : top * a.factor) - SHIFT;
            any_far = __ballot(far) != 0;
            sum *= keep;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[t] *= keep;
        }
        if (__builtin_expect(any_far, false)) {
            asm volatile("");
            const float less = fabsf(top * a.factor) > FAR && top != -INFINITY ? top : 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] -= less;
        }
        float add = 0.0f;      // of the tile by itself: weights that the whole sum has no bit for count together
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], a.factor, -off));
                add += w;
                p[2 * t + e / 8][e % 8] = (T)w;
            }
        sum += add;
    };
    // Step i: copies of the next tiles, PV of tile i, QK and softmax of tile i + 1.  A stage's keys are copied over when QK has read them,
    // a step before its values.  While one workgroup's wave on a SIMD is at the softmax the other's uses the matrix pipe; the priority of the
    // products keeps the two apart (1088 -> 1075 us for the prompt above).
    if (tiles > 0) {
        wait_copies();
        __syncthreads();
        const int own = (wave_keys + PROMPT_KEYS - 1) / PROMPT_KEYS;      // tiles that this wave's queries see
        if (own > 0) {
            products(no, yes);
            softmax(0);
        }
        __syncthreads();
        const auto begin_step = [&](int i) {
            if (i + 1 < tiles) copy(1, i + 1);
            if (i + 2 < tiles) copy(0, i + 2);
        };
        const auto end_step = [&] {
            wait_copies();
            __syncthreads();
        };
        int i = 0, other = TILE;      // from one stage to the other
#pragma unroll
        for (int e = 0; e < KS; ++e) key_at[e] += TILE;
        for (; i + 1 < own; ++i) {
            begin_step(i);
            __builtin_amdgcn_s_setprio(1);
            products(yes, yes);
            __builtin_amdgcn_s_setprio(0);
            softmax(i + 1);
#pragma unroll
            for (int e = 0; e < KS; ++e) key_at[e] -= other;
#pragma unroll
            for (int t = 0; t < VT; ++t) value_at[t] += other;
            other = -other;
            end_step();
        }
        if (own > 0) {
            begin_step(i);
            products(yes, no);
            end_step();
            ++i;
        }
        for (; i < tiles; ++i) {
            begin_step(i);
            end_step();
        }
    }

    // a lane holds dimensions 8 j + 4 half + 0..3 of its query: the two halves trade every other four for 16-byte stores
    sum = over_halves_sum(sum);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    T* yp = static_cast<T*>(a.Y) + (rq.first + (size_t)row) * a.ldy + (size_t)head * D + 8 * half;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            if (32 * t + 8 * i >= D) continue;
            typename M::v4 y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[j][e] = (T)(o[t][4 * (i + j) + e] * inv);
            const v2u u0 = __builtin_bit_cast(v2u, y[0]), u1 = __builtin_bit_cast(v2u, y[1]);
            const auto lo = __builtin_amdgcn_permlane32_swap(u0[0], u1[0], false, false), hi = __builtin_amdgcn_permlane32_swap(u0[1], u1[1], false, false);
            if (row < rq.count) *reinterpret_cast<v4u*>(yp + 32 * t + 8 * i) = v4u{lo[0], hi[0], lo[1], hi[1]};
        }
}

template <int DT> int launch(const PromptAttn& a, int head_dim, hipStream_t stream)
{
    const unsigned grid = (unsigned)prompt_workgroups(a.tokens_q, a.batch, a.max_q, a.heads_q, a.heads_kv);
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
                       causal, batch};
    return x_dtype == FQ_F16 ? launch<FQ_F16>(a, head_dim, stream) : launch<FQ_BF16>(a, head_dim, stream);
}

}  // namespace fq
