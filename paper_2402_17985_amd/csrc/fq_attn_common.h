// What the attention translation units share (GPU code only; everything has internal linkage).
#pragma once
#include <type_traits>

#include "fq_attn_rules.h"
#include "fq_internal.h"

namespace fq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int DT> struct Stored;
template <> struct Stored<FQ_F32> { typedef float type; };
template <> struct Stored<FQ_F16> { typedef _Float16 type; };
template <> struct Stored<FQ_BF16> { typedef __bf16 type; };

constexpr float SLACK = 8.0f;   // accumulators are rescaled only when a maximum has grown by more than a factor 2^8
// Where accumulators run over all keys with probabilities in fp16 it is 2^4, and a probability's 1 is 2^11: at most 2^15 then, and what is below 2^-36 of the
// largest vanishes, little even of 2^17 of them (as 1 and 2^8 everything below 2^-25 did: the whole of 131072 keys 17.7 nats below one).
constexpr float HALF_SLACK = 4.0f, HALF_SHIFT = 11.0f;
// Exponents of probabilities are one fused product and sum, s f - off, whose off is rounded as scores of its size are.  Beyond this the largest score is taken off
// first: half a step of off would make the largest probability too large for fp16 from 2^24 on.
constexpr float FAR = 0x1p16f;
constexpr float LOG2E = 1.44269504088896340736f;

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

// Rows of C 16-byte pieces lie in LDS without gaps; where 16 rows are read at a time, the same piece of each, piece c of row r lies at place
// (c + key_turn(C, r)) mod C, which spreads them over the 64 banks (256 bytes).
constexpr int key_turn(int C, int r) { return C == 16 ? r % 16 : C == 12 ? r % 16 / 4 : C == 10 ? r % 16 / 8 : r % 16 / 2; }

// Of the two lanes that share a query, lane and lane + 32.
__device__ __forceinline__ float over_halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What orders up to 64 sequences, one a lane, by their lengths: no two are equal.  (Lengths of 2^26 and more count as equally long.)
__device__ __forceinline__ uint32_t length_key(int length)
{
    return (uint32_t)min(max(length, 0), (1 << 26) - 1) << 6 | (63 - threadIdx.x % 64);
}

// The sum of `value` over the lanes of the batch with a larger key (a lane without a sequence has key 0 or value 0).
__device__ __forceinline__ int sum_of_longer(uint32_t key, int value, int batch)
{
    int sum = 0;
    for (int i0 = 0; i0 < batch; i0 += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int its = __builtin_amdgcn_readlane(value, i0 + i);
            sum += (uint32_t)__builtin_amdgcn_readlane((int)key, i0 + i) > key ? its : 0;
        }
    return sum;
}

// The sequence of a batch whose tiles lie at `place` where sequence b's begin at first(b), which does not fall: 64 probes at a time.
template <typename First> __device__ __forceinline__ int sequence_at(int place, int batch, First first)
{
    const int lane = threadIdx.x % 64;
    int b = 0;
    for (int n = batch; n > 1;) {      // it is one of n from b on
        const int apart = (n + 63) / 64, probe = b + lane * apart;
        const bool reached = lane * apart < n && first(min(probe, batch - 1)) <= place;
        const int skip = max((int)__builtin_popcountll(__ballot(reached)) - 1, 0) * apart;
        b += skip;
        n = min(apart, n - skip);
    }
    return b;
}

}  // namespace
}  // namespace fq
