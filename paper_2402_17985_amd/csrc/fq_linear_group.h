// What the kernels of fq_linear_group_i4 share (GPU code only; everything has internal linkage).
#pragma once
#include "fq_internal.h"

namespace fq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

struct GroupProduct {
    const void* X;
    const uint8_t* Wq;
    const void *S, *B;
    const float* bias;
    void* Y;
    size_t ldx, ldy;
    int M, N, K, groups, s_dtype, y_dtype, tiles_n;

    __device__ __forceinline__ float scale(const void* base, size_t at) const
    {
        if (s_dtype == FQ_F32) return static_cast<const float*>(base)[at];
        if (s_dtype == FQ_F16) return (float)static_cast<const _Float16*>(base)[at];
        return (float)static_cast<const __bf16*>(base)[at];
    }
    __device__ __forceinline__ void store(float v, size_t at) const
    {
        if (y_dtype == FQ_F32) static_cast<float*>(Y)[at] = v;
        else if (y_dtype == FQ_F16) static_cast<_Float16*>(Y)[at] = (_Float16)v;
        else static_cast<__bf16*>(Y)[at] = (__bf16)v;
    }
};

// Eight codes (a word of nibbles, two's complement) as eight 16-bit numbers, and eight activations in the same order: nibbles 0, 4, 1, 5, 2, 6,
// 3, 7, as a shift and a mask bring nibbles j and j + 4 into the halves of a register.
// A nibble in the top four of the mantissa bits of 16 makes 16 + u; u = q + 8 is q with its highest bit turned.
template <int XT> struct GroupMma;
template <> struct GroupMma<FQ_BF16> {
    typedef v8bf v8;
    static __device__ __forceinline__ v8 widen(uint32_t w)      // q + 24
    {
        constexpr uint32_t MASK = 0x00780078u, BASE = 0x41c041c0u;
        return __builtin_bit_cast(v8, v4u{((w << 3) & MASK) ^ BASE, ((w >> 1) & MASK) ^ BASE, ((w >> 5) & MASK) ^ BASE, ((w >> 9) & MASK) ^ BASE});
    }
    static __device__ __forceinline__ v8 ones() { return __builtin_bit_cast(v8, v4u{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}); }
    static __device__ __forceinline__ v8 activations(const v4u x);
    static __device__ __forceinline__ v4f mul(v8 x, v8 w, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};
template <> struct GroupMma<FQ_F16> {
    typedef v8h v8;
    static __device__ __forceinline__ uint32_t less(uint32_t v, _Float16 by) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, v) - v2h{by, by}); }
    // q: nibbles at bits 0 .. 3 of 1024 and at bits 4 .. 7 of 64 count 1 without a shift
    static __device__ __forceinline__ v8 widen(uint32_t w)
    {
        constexpr uint32_t LOW = 0x000f000fu, HIGH = 0x00f000f0u, BASE_LOW = 0x64086408u, BASE_HIGH = 0x54805480u;
        const uint32_t v = w >> 8;
        return __builtin_bit_cast(v8, v4u{less((w & LOW) ^ BASE_LOW, 1032.0f16), less((w & HIGH) ^ BASE_HIGH, 72.0f16), less((v & LOW) ^ BASE_LOW, 1032.0f16),
                                          less((v & HIGH) ^ BASE_HIGH, 72.0f16)});
    }
    static __device__ __forceinline__ v8 ones() { return __builtin_bit_cast(v8, v4u{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}); }
    static __device__ __forceinline__ v8 activations(const v4u x);
    static __device__ __forceinline__ v4f mul(v8 x, v8 w, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0); }
};
__device__ __forceinline__ v4u in_code_order(const v4u x)
{
    return v4u{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
               __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}
__device__ __forceinline__ v8bf GroupMma<FQ_BF16>::activations(const v4u x) { return __builtin_bit_cast(v8bf, in_code_order(x)); }
__device__ __forceinline__ v8h GroupMma<FQ_F16>::activations(const v4u x) { return __builtin_bit_cast(v8h, in_code_order(x)); }

// Lane quarter c (16 lanes) holds words 4 c .. 4 c + 3 of a row; afterwards word j of it is the row's word 4 j + c: the 4 x 4 words of
// lanes r, r + 16, r + 32, r + 48 are transposed.
__device__ __forceinline__ void transpose_quarters(v4u& v)
{
    auto swap32 = [](uint32_t& a, uint32_t& b) {        // lanes 32 .. 63 of a with lanes 0 .. 31 of b
        const auto t = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        a = t[0];
        b = t[1];
    };
    auto swap16 = [](uint32_t& a, uint32_t& b) {        // odd quarters of a with even quarters of b
        const auto t = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = t[0];
        b = t[1];
    };
    uint32_t v0 = v[0], v1 = v[1], v2 = v[2], v3 = v[3];
    swap32(v0, v2);
    swap32(v1, v3);
    swap16(v0, v1);
    swap16(v2, v3);
    v = v4u{v0, v1, v2, v3};
}

}  // namespace
}  // namespace fq
