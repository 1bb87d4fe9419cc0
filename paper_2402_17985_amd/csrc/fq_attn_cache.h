// What the two kernels of fq_attn_cache share (GPU code only; everything has internal linkage).
#pragma once
#include "fq_attn_common.h"

namespace fq {

struct CacheAttn {
    const void* Q;
    void* Y;
    long long ldq, ldy;
    const int32_t *cu_q, *lens, *table;
    const int8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    float *part, *stat;     // with more than one split: [row, head, split, head_dim] and [row, head, split, (maximum, sum)]
    float scale;
    int tokens, max_q, max_len, heads_q, heads_kv, group, capacity, pages, page, page_shift, width, splits, round, order;
};

// The kernel for many columns (fq_attn_cache_wide.hip)
int launch_attn_cache_wide(const CacheAttn& a, int x_dtype, int head_dim, int batch, unsigned grid, hipStream_t stream);

namespace {

// A wave-uniform value that no kernel writes while this one runs, by the scalar path: vector loads would queue behind the keys' and values'.
template <typename T> __device__ __forceinline__ T scalar(const T* p, size_t i)
{
    return ((const __attribute__((address_space(4))) T*)(uintptr_t)p)[i];
}

// Eight signed bytes, each plus 1152, in fp16: with its sign bit turned a byte is v + 128, and that as the low byte of 0x64.. is 1152 + v.
// What the 1152 add to a product is taken off again by its accumulator's start: a subtraction a step instead of one a pair of values.
__device__ __forceinline__ v8h widen8(uint32_t lo, uint32_t hi)
{
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const v4u r = {__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u),
                   __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)};
    return __builtin_bit_cast(v8h, r);
}
constexpr float WIDEN_BIAS = 1152.0f;

// The maximum of no scores: below every score, and finite, so that differences of maxima are numbers.
constexpr float LOWEST = -0x1p100f;

}  // namespace
}  // namespace fq
