// Rows of floating-point elements taken 16 at a time: loaded as they are stored, widened to fp32, rounded and stored (GPU code only).
#pragma once
#include "fq_quant_common.h"

namespace fq {
namespace {

constexpr int NONE = -1;          // no such array

// 16 elements as they are stored
template <int DT> struct Raw {
    v4u v[16 / Elem<DT>::VEC];
};
template <> struct Raw<NONE> {};

// Elements 16 g .. 16 g + 15 of a row of K; those from K on are zeros and are not read.
template <int DT> __device__ __forceinline__ Raw<DT> load_raw(const void* base, size_t row, int g, int K)
{
    Raw<DT> r = {};
    if constexpr (DT != NONE) {
        typedef typename Elem<DT>::type T;
        constexpr int VEC = Elem<DT>::VEC;
        const T* p = static_cast<const T*>(base) + row + 16 * g;
        if (16 * g + 16 <= K) {
#pragma unroll
            for (int i = 0; i < 16 / VEC; ++i) r.v[i] = reinterpret_cast<const v4u*>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (16 * g + i >= K) continue;
                if constexpr (VEC == 4) r.v[i / 4][i % 4] = __float_as_uint(p[i]);
                else r.v[i / 8][i / 2 % 4] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i % 2));
            }
        }
    }
    return r;
}
template <int DT> __device__ __forceinline__ void widen(const Raw<DT>& r, float (&x)[16])
{
    constexpr int VEC = Elem<DT>::VEC;
#pragma unroll
    for (int i = 0; i < 16 / VEC; ++i) widen16<DT>(r.v[i], x + i * VEC);
}
__device__ __forceinline__ void load_any(const void* base, int dtype, int g, int K, float (&x)[16])
{
    if (dtype == FQ_F32) widen<FQ_F32>(load_raw<FQ_F32>(base, 0, g, K), x);
    else if (dtype == FQ_F16) widen<FQ_F16>(load_raw<FQ_F16>(base, 0, g, K), x);
    else widen<FQ_BF16>(load_raw<FQ_BF16>(base, 0, g, K), x);
}

// x rounded to the type, half to even
template <int DT> __device__ __forceinline__ Raw<DT> narrow(const float (&x)[16])
{
    Raw<DT> r;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if constexpr (DT == FQ_F32) {
            r.v[i / 4][i % 4] = __float_as_uint(x[i]);
        } else {
            uint16_t h;
            if constexpr (DT == FQ_F16) h = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
            else h = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
            if (i % 2) r.v[i / 8][i / 2 % 4] |= (uint32_t)h << 16;
            else r.v[i / 8][i / 2 % 4] = h;
        }
    }
    return r;
}
template <int DT> __device__ __forceinline__ void store_raw(const Raw<DT>& r, void* base, size_t row, int g, int K)
{
    typedef typename Elem<DT>::type T;
    constexpr int VEC = Elem<DT>::VEC;
    T* p = static_cast<T*>(base) + row + 16 * g;
    if (16 * g + 16 <= K) {
#pragma unroll
        for (int i = 0; i < 16 / VEC; ++i) reinterpret_cast<v4u*>(p)[i] = r.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (16 * g + i >= K) continue;
            if constexpr (VEC == 4) p[i] = __uint_as_float(r.v[i / 4][i % 4]);
            else p[i] = __builtin_bit_cast(T, (uint16_t)(r.v[i / 8][i / 2 % 4] >> (16 * (i % 2))));
        }
    }
}
__device__ __forceinline__ void store_any(const float (&y)[16], void* base, int dtype, size_t row, int g, int K)
{
    if (dtype == FQ_F32) store_raw<FQ_F32>(narrow<FQ_F32>(y), base, row, g, K);
    else if (dtype == FQ_F16) store_raw<FQ_F16>(narrow<FQ_F16>(y), base, row, g, K);
    else store_raw<FQ_BF16>(narrow<FQ_BF16>(y), base, row, g, K);
}

}  // namespace
}  // namespace fq
