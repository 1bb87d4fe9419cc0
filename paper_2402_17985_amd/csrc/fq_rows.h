// Rows of floating-point elements taken 8 at a time: loaded as they are stored, widened to fp32, rounded and stored (GPU code only).
#pragma once
#include "fq_quant_common.h"

namespace fq {
namespace {

constexpr int NONE = -1;          // no such array

// 8 elements as they are stored
template <int DT> struct Raw {
    v4u v[8 / Elem<DT>::VEC];
};
template <> struct Raw<NONE> {};

// Elements 8 g .. 8 g + 7 of the row at `row`, of K; those from K on are zeros and are not read.  RAGGED: K need not be a multiple of 8.
template <int DT, bool RAGGED = true> __device__ __forceinline__ Raw<DT> load_raw(const void* row, int g, int K)
{
    Raw<DT> r = {};
    if constexpr (DT != NONE) {
        typedef typename Elem<DT>::type T;
        constexpr int VEC = Elem<DT>::VEC;
        const T* p = static_cast<const T*>(row) + (uint32_t)(8 * g);
        if (!RAGGED || 8 * g + 8 <= K) {
#pragma unroll
            for (int i = 0; i < 8 / VEC; ++i) r.v[i] = reinterpret_cast<const v4u*>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (8 * g + i >= K) continue;
                if constexpr (VEC == 4) r.v[i / 4][i % 4] = __float_as_uint(p[i]);
                else r.v[0][i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i % 2));
            }
        }
    }
    return r;
}
template <int DT> __device__ __forceinline__ void widen(const Raw<DT>& r, float (&x)[8])
{
    constexpr int VEC = Elem<DT>::VEC;
#pragma unroll
    for (int i = 0; i < 8 / VEC; ++i) widen16<DT>(r.v[i], x + i * VEC);
}
template <bool RAGGED> __device__ __forceinline__ void load_any(const void* row, int dtype, int g, int K, float (&x)[8])
{
    if (dtype == FQ_F32) widen<FQ_F32>(load_raw<FQ_F32, RAGGED>(row, g, K), x);
    else if (dtype == FQ_F16) widen<FQ_F16>(load_raw<FQ_F16, RAGGED>(row, g, K), x);
    else widen<FQ_BF16>(load_raw<FQ_BF16, RAGGED>(row, g, K), x);
}

// x rounded to the type, half to even
template <int DT> __device__ __forceinline__ Raw<DT> narrow(const float (&x)[8])
{
    Raw<DT> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (DT == FQ_F32) {
            r.v[i / 4][i % 4] = __float_as_uint(x[i]);
        } else {
            uint16_t h;
            if constexpr (DT == FQ_F16) h = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
            else h = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
            if (i % 2) r.v[0][i / 2] |= (uint32_t)h << 16;
            else r.v[0][i / 2] = h;
        }
    }
    return r;
}
template <int DT, bool RAGGED> __device__ __forceinline__ void store_raw(const Raw<DT>& r, void* row, int g, int K)
{
    typedef typename Elem<DT>::type T;
    constexpr int VEC = Elem<DT>::VEC;
    T* p = static_cast<T*>(row) + (uint32_t)(8 * g);
    if (!RAGGED || 8 * g + 8 <= K) {
#pragma unroll
        for (int i = 0; i < 8 / VEC; ++i) reinterpret_cast<v4u*>(p)[i] = r.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (8 * g + i >= K) continue;
            if constexpr (VEC == 4) p[i] = __uint_as_float(r.v[i / 4][i % 4]);
            else p[i] = __builtin_bit_cast(T, (uint16_t)(r.v[0][i / 2] >> (16 * (i % 2))));
        }
    }
}
template <bool RAGGED> __device__ __forceinline__ void store_any(const float (&y)[8], void* row, int dtype, int g, int K)
{
    if (dtype == FQ_F32) store_raw<FQ_F32, RAGGED>(narrow<FQ_F32>(y), row, g, K);
    else if (dtype == FQ_F16) store_raw<FQ_F16, RAGGED>(narrow<FQ_F16>(y), row, g, K);
    else store_raw<FQ_BF16, RAGGED>(narrow<FQ_BF16>(y), row, g, K);
}

// The bytes of an element, where the type is known (0: no such array)
template <int DT> constexpr int element_bytes() { return DT == FQ_F32 ? 4 : DT == NONE ? 0 : 2; }
// Row of an array of that many bytes an element; the same for all lanes
__device__ __forceinline__ const char* row_of(const void* base, size_t ld, int bytes, int row) { return static_cast<const char*>(base) + (size_t)row * ld * bytes; }
__device__ __forceinline__ char* row_of(void* base, size_t ld, int bytes, int row) { return static_cast<char*>(base) + (size_t)row * ld * bytes; }

}  // namespace
}  // namespace fq
