// Argument checks that the C-ABI layers share (host code).
#pragma once
#include "fq_internal.h"

namespace fq {

inline bool float_dtype(int d) { return d == FQ_F32 || d == FQ_F16 || d == FQ_BF16; }

// Checks shared by the calls that read a floating-point matrix [rows, K] with stride ld.
inline int check_matrix(const char* what, const void* p, int dtype, int rows, int K, int ld)
{
    if (!p) return fail(FQ_ERR_NULL, "%s is NULL", what);
    if (!float_dtype(dtype)) return fail(FQ_ERR_DTYPE, "%s: dtype %d is not F32/F16/BF16", what, dtype);
    if (rows <= 0 || K <= 0) return fail(FQ_ERR_SHAPE, "%s: non-positive shape %d x %d", what, rows, K);
    if (ld < K) return fail(FQ_ERR_SHAPE, "%s: row stride %d < K = %d", what, ld, K);
    if (((size_t)ld * elem_size(dtype)) % 16 != 0)
        return fail(FQ_ERR_SHAPE, "%s: row stride of %d elements is not a multiple of 16 bytes", what, ld);
    if (!aligned16(p)) return fail(FQ_ERR_ALIGN, "%s is not 16-byte aligned", what);
    return FQ_OK;
}

// bytes of one row of a quantized array: a byte, a nibble or a 6-bit code per slot
inline size_t quantized_row_bytes(int Kpad, int bits)
{
    return bits == 8 ? (size_t)Kpad : (bits == 4 ? (size_t)Kpad / 2 : (size_t)Kpad / 4 * 3);
}

inline int check_map(const int32_t* src_idx, int Kpad, int bits)
{
    if (!src_idx) return fail(FQ_ERR_NULL, "src_idx is NULL");
    if (bits != 8 && bits != 4 && bits != FQ_BITS_I4_E3M2)
        return fail(FQ_ERR_DTYPE, "bits = %d, must be 8, 4 or %d (4-bit values in E3M2 storage)", bits, FQ_BITS_I4_E3M2);
    if (Kpad <= 0 || Kpad % 32 != 0) return fail(FQ_ERR_SHAPE, "Kpad = %d must be a positive multiple of 32", Kpad);
    if (bits == FQ_BITS_I4_E3M2 && Kpad % 128 != 0)
        return fail(FQ_ERR_SHAPE, "Kpad = %d must be a multiple of 128 for E3M2 storage", Kpad);
    if (Kpad >= 131072) return fail(FQ_ERR_RANGE, "Kpad = %d: int32 accumulators could overflow (needs Kpad < 131072)", Kpad);
    if (!aligned16(src_idx)) return fail(FQ_ERR_ALIGN, "src_idx is not 16-byte aligned");
    return FQ_OK;
}

}  // namespace fq
