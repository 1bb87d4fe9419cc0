// What the kernels of fq_linear_group_i4 share (GPU code only).
#pragma once
#include "fq_internal.h"

namespace fq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int PER> struct StepScales {
    uint32_t v[PER];
};
// words at any 16-bit place (global memory takes wide loads from there)
template <int N> struct __attribute__((packed, aligned(2))) Pairs {
    uint32_t v[N];
};
template <> struct Pairs<0> {
    uint32_t v[1];
};

struct GroupProduct {
    const void* X;
    const uint8_t* Wq;
    const void *S, *B;
    const float* bias;
    void* Y;
    size_t ldx, ldy;
    int M, N, K, groups, s_dtype, y_dtype, tiles_n, tiles, group_shift;

    // The scales (or offsets) of a step's PER groups as they are stored, 16-bit ones two to a word; those of groups behind the row's last are its last one.
    template <int PER> __device__ __forceinline__ StepScales<PER> step_scales(const void* base, size_t row, int group) const
    {
        StepScales<PER> r = {};
        if (s_dtype == FQ_F32) {
#pragma unroll
            for (int g = 0; g < PER; ++g) r.v[g] = static_cast<const uint32_t*>(base)[row + min(group + g, groups - 1)];
        } else if (PER > 1 && group + PER <= groups) {
            const Pairs<PER / 2> p = *reinterpret_cast<const Pairs<PER / 2>*>(static_cast<const uint16_t*>(base) + row + group);
#pragma unroll
            for (int g = 0; g < PER / 2; ++g) r.v[g] = p.v[g];
        } else {
#pragma unroll
            for (int g = 0; g < PER; ++g) r.v[g / 2] |= (uint32_t)static_cast<const uint16_t*>(base)[row + min(group + g, groups - 1)] << (16 * (g % 2));
        }
        return r;
    }
    // the value of a single one
    __device__ __forceinline__ float value(uint32_t v) const
    {
        return s_dtype == FQ_F32 ? __uint_as_float(v) : s_dtype == FQ_BF16 ? __uint_as_float(v << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)v);
    }
    // four columns of a row (those from N on are left out), plus the bias
    __device__ __forceinline__ void store4(v4f v, int m, int n) const
    {
        const size_t at = (size_t)m * ldy + n;
        if (bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) v[e] += bias[n + e];
        }
        if (n + 4 <= N && ldy % 4 == 0) {
            if (y_dtype == FQ_F32) *reinterpret_cast<v4f*>(static_cast<float*>(Y) + at) = v;
            else if (y_dtype == FQ_F16) *reinterpret_cast<v4h*>(static_cast<_Float16*>(Y) + at) = v4h{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
            else *reinterpret_cast<v4bf*>(static_cast<__bf16*>(Y) + at) = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) store(v[e], at + e);
        }
    }
    // the value of group g of a step, from the word that holds it (words: from another lane)
    template <typename Word> __device__ __forceinline__ float scale_at(int g, Word word) const
    {
        if (s_dtype == FQ_F32) return __uint_as_float(word(g));
        const uint32_t v = word(g / 2) >> (16 * (g % 2));
        return s_dtype == FQ_BF16 ? __uint_as_float(v << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)v);
    }
    __device__ __forceinline__ void store(float v, size_t at) const
    {
        if (y_dtype == FQ_F32) static_cast<float*>(Y)[at] = v;
        else if (y_dtype == FQ_F16) static_cast<_Float16*>(Y)[at] = (_Float16)v;
        else static_cast<__bf16*>(Y)[at] = (__bf16)v;
    }
};

// Kernels of more rows than the one of single tokens takes (fq_linear_group_tile.hip, built once for each type of activations)
template <int XT> int launch_group_tile(const GroupProduct& a, int group, hipStream_t stream);

namespace {

// Eight codes (a word of nibbles, two's complement) as eight 16-bit numbers in the columns' order: a byte's two nibbles into the halves of a register.
// u = q + 8 is q with its highest bit turned.
template <int XT> struct GroupMma;
// q + 24: a nibble in the top four mantissa bits of 16 makes 16 + u.  The multiplication brings a byte's low nibble there in the low half and its high one in the
// high half; it takes the byte as its operand, so two codes cost two instructions (shifts, masks and a subtraction in fp32: seven).
template <uint32_t FACTOR, uint32_t MASK, uint32_t BASE> __device__ __forceinline__ v4u surplus_codes(uint32_t w)
{
    v4u r;
#pragma unroll
    for (int p = 0; p < 4; ++p) r[p] = ((((w >> (8 * p)) & 0xffu) * FACTOR) & MASK) ^ BASE;
    return r;
}
template <> struct GroupMma<FQ_BF16> {
    typedef v8bf v8;
    static constexpr bool SURPLUS = true;      // widen() gives q + 24, exactly; a product with all(true), -24 everywhere, takes the surplus out
    static __device__ __forceinline__ v8 widen(uint32_t w) { return widen24(w); }
    static __device__ __forceinline__ v8 widen24(uint32_t w) { return __builtin_bit_cast(v8, surplus_codes<0x8008u, 0x00780078u, 0x41c041c0u>(w)); }
    static __device__ __forceinline__ v8 all(bool less) { const uint32_t v = less ? 0xc1c0c1c0u : 0x3f803f80u; return __builtin_bit_cast(v8, v4u{v, v, v, v}); }
    static __device__ __forceinline__ v4f mul(v8 x, v8 w, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};
template <> struct GroupMma<FQ_F16> {
    typedef v8h v8;
    static constexpr bool SURPLUS = false;     // widen() gives q: there is a packed subtraction, the third instruction for two codes
    static __device__ __forceinline__ v8 widen24(uint32_t w) { return __builtin_bit_cast(v8, surplus_codes<0x40040u, 0x03c003c0u, 0x4e004e00u>(w)); }
    // nibbles at bits 0 .. 3 of 1024 and at bits 4 .. 7 of 64 count 1 where they are
    static __device__ __forceinline__ v8 widen(uint32_t w)
    {
        v4u r;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t both = __builtin_amdgcn_perm(w, w, 0x0c000c00u | (uint32_t)(p * 0x00010001));
            r[p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, (both & 0x00f0000fu) ^ 0x54806408u) - v2h{1032.0f16, 72.0f16});
        }
        return __builtin_bit_cast(v8, r);
    }
    static __device__ __forceinline__ v8 all(bool) { return __builtin_bit_cast(v8, v4u{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}); }
    static __device__ __forceinline__ v4f mul(v8 x, v8 w, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0); }
};

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
