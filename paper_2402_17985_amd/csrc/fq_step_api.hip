// C-ABI layer of the calls around the quantized products and the cache (norm with a quantized output, 4-bit weights with group
// scales, page copies): argument validation.  Nothing here allocates or synchronizes.
#include <cmath>

#include "fq_attn_rules.h"
#include "fq_checks.h"
#include "fq_rules.h"

namespace fq {
namespace {

int check_group(int group, int K)
{
    if (group != 32 && group != 64 && group != 128) return fail(FQ_ERR_SHAPE, "group = %d must be 32, 64 or 128", group);
    if (K % 32 != 0) return fail(FQ_ERR_SHAPE, "K = %d must be a multiple of 32", K);
    if (K > MAX_GROUP_WIDTH) return fail(FQ_ERR_RANGE, "K = %d: at most 2^24", K);
    return FQ_OK;
}

int check_dense(const char* what, const void* p, bool wanted)
{
    if (!p) return wanted ? fail(FQ_ERR_NULL, "%s is NULL", what) : FQ_OK;
    if (!aligned16(p)) return fail(FQ_ERR_ALIGN, "%s is not 16-byte aligned", what);
    return FQ_OK;
}

}  // namespace
}  // namespace fq

using namespace fq;

extern "C" {

size_t fq_rms_norm_workspace_bytes(int M, int K, int Kpad)
{
    if (M <= 0 || K <= 0 || Kpad <= 0) return 16;
    return rms_norm_workspace(M);
}

int fq_rms_norm_quant(const void* X, int x_dtype, int M, int K, int ldx, const void* R, int r_dtype, int ldr, void* R_out, int ldro,
                      const void* gamma, int g_dtype, float eps, void* Y, int y_dtype, int ldy,
                      const int32_t* src_idx, const int32_t* rep, int Kpad, int bits, const float* absmax_in,
                      void* Xq_out, float* s_x_out, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    int rc = check_matrix("X", X, x_dtype, M, K, ldx);
    if (!rc && (R || R_out)) rc = check_matrix("R", R, r_dtype, M, K, ldr);
    if (!rc && (R || R_out)) rc = check_matrix("R_out", R_out, r_dtype, M, K, ldro);
    if (!rc) rc = check_dense("gamma", gamma, true);
    if (rc) return rc;
    if (!float_dtype(g_dtype)) return fail(FQ_ERR_DTYPE, "gamma: dtype %d is not F32/F16/BF16", g_dtype);
    if (K > 32768) return fail(FQ_ERR_RANGE, "K = %d: at most 32768", K);
    if (M > MAX_NORM_ROWS) return fail(FQ_ERR_RANGE, "M = %d: at most %d", M, MAX_NORM_ROWS);
    if (!(eps > 0.0f) || std::isinf(eps)) return fail(FQ_ERR_RANGE, "eps = %g must be positive and finite", (double)eps);
    if (!Y && !Xq_out) return fail(FQ_ERR_NULL, "neither Y nor Xq_out is wanted");
    if (Y && (rc = check_matrix("Y", Y, y_dtype, M, K, ldy))) return rc;
    if (Y && R && Y == R_out) return fail(FQ_ERR_RANGE, "Y and R_out are the same array");
    if (Xq_out) {
        rc = check_map(src_idx, Kpad, bits);
        if (!rc && !rep) rc = fail(FQ_ERR_NULL, "rep is NULL");
        if (!rc && reinterpret_cast<uintptr_t>(rep) % 4 != 0) rc = fail(FQ_ERR_ALIGN, "rep is not 4-byte aligned");
        if (!rc) rc = check_dense("Xq_out", Xq_out, true);
        if (!rc && !s_x_out) rc = fail(FQ_ERR_NULL, "s_x_out is NULL");
        if (rc) return rc;
        if (!absmax_in) {
            if (!workspace) return fail(FQ_ERR_NULL, "workspace is NULL with a dynamic scale");
            if (!aligned16(workspace)) return fail(FQ_ERR_ALIGN, "workspace is not 16-byte aligned");
            const size_t need = fq_rms_norm_workspace_bytes(M, K, Kpad);
            if (workspace_bytes < need) return fail(FQ_ERR_WORKSPACE, "workspace of %zu bytes < %zu required", workspace_bytes, need);
        }
    }
    return launch_rms_norm_quant(X, x_dtype, M, K, ldx, R, r_dtype, ldr, R_out, ldro, gamma, g_dtype, eps, Y, y_dtype, ldy, src_idx, rep, Kpad, bits,
                                 absmax_in, Xq_out, s_x_out, workspace, static_cast<hipStream_t>(stream));
}

int fq_group_weights_i4(const void* W, int w_dtype, int N, int K, int ldw, int group, void* Wq_out, void* S_out, void* B_out, int s_dtype,
                        void* stream)
{
    clear_error();
    int rc = check_matrix("W", W, w_dtype, N, K, ldw);
    if (!rc) rc = check_group(group, K);
    if (!rc && !float_dtype(s_dtype)) rc = fail(FQ_ERR_DTYPE, "scales: dtype %d is not F32/F16/BF16", s_dtype);
    if (!rc) rc = check_dense("Wq_out", Wq_out, true);
    if (!rc) rc = check_dense("S_out", S_out, true);
    if (!rc) rc = check_dense("B_out", B_out, false);
    if (rc) return rc;
    if (((long long)K + group - 1) / group * (group / 16) * N >= (1LL << 31)) return fail(FQ_ERR_RANGE, "%d x %d weights are more than one launch holds", N, K);
    return launch_group_weights(W, w_dtype, N, K, ldw, group, Wq_out, S_out, B_out, s_dtype, static_cast<hipStream_t>(stream));
}

int fq_linear_group_i4(const void* X, int x_dtype, int M, int K, int ldx, const void* Wq, const void* S, const void* B, int s_dtype, int group,
                       int N, const float* bias, void* Y, int y_dtype, int ldy, void* stream)
{
    clear_error();
    int rc = check_matrix("X", X, x_dtype, M, K, ldx);
    if (!rc && x_dtype == FQ_F32) rc = fail(FQ_ERR_DTYPE, "X: dtype F32 is not F16/BF16");
    if (!rc) rc = check_group(group, K);
    if (!rc && (!float_dtype(s_dtype) || !float_dtype(y_dtype))) rc = fail(FQ_ERR_DTYPE, "scales or Y: dtype %d or %d is not F32/F16/BF16", s_dtype, y_dtype);
    if (!rc) rc = check_dense("Wq", Wq, true);
    if (!rc) rc = check_dense("S", S, true);
    if (!rc) rc = check_dense("B", B, false);
    if (!rc) rc = check_dense("bias", bias, false);
    if (!rc) rc = check_dense("Y", Y, true);
    if (rc) return rc;
    if (ldx > MAX_GROUP_WIDTH) return fail(FQ_ERR_RANGE, "X: row stride of %d elements, at most 2^24", ldx);
    if (N <= 0) return fail(FQ_ERR_SHAPE, "N = %d must be positive", N);
    if (ldy < N) return fail(FQ_ERR_SHAPE, "ldy = %d < N = %d", ldy, N);
    if (M > MAX_GROUP_SIDE || N > MAX_GROUP_SIDE) return fail(FQ_ERR_RANGE, "%d x %d outputs: at most %d each way", M, N, MAX_GROUP_SIDE);
    return launch_linear_group(X, x_dtype, M, K, ldx, Wq, S, B, s_dtype, group, N, bias, Y, y_dtype, ldy, static_cast<hipStream_t>(stream));
}

int fq_kv_copy_pages(int8_t* k_cache, int8_t* v_cache, float* k_scale, float* v_scale, int pages, int heads_kv, int page_size, int head_dim,
                     const int32_t* from, const int32_t* to, int count, void* stream)
{
    clear_error();
    if (count < 0) return fail(FQ_ERR_SHAPE, "count = %d", count);
    if (heads_kv <= 0 || heads_kv > 16384) return fail(FQ_ERR_RANGE, "heads_kv = %d must be in 1 .. 16384", heads_kv);
    if (!head_dim_ok(head_dim)) return fail(FQ_ERR_SHAPE, "head_dim = %d must be 64, 80, 96 or 128", head_dim);
    if (page_size != 64 && page_size != 128) return fail(FQ_ERR_SHAPE, "page_size = %d must be 64 or 128", page_size);
    if (pages <= 0) return fail(FQ_ERR_SHAPE, "%d pages", pages);
    int rc = check_dense("k_cache", k_cache, true);
    if (!rc) rc = check_dense("v_cache", v_cache, true);
    if (!rc) rc = check_dense("k_scale", k_scale, true);
    if (!rc) rc = check_dense("v_scale", v_scale, true);
    if (rc) return rc;
    if (count == 0) return FQ_OK;
    if (!from || !to) return fail(FQ_ERR_NULL, "from or to is NULL");
    if (reinterpret_cast<uintptr_t>(from) % 4 != 0 || reinterpret_cast<uintptr_t>(to) % 4 != 0) return fail(FQ_ERR_ALIGN, "from or to is not 4-byte aligned");
    if (!launch_holds(2 * copy_parts((size_t)heads_kv * page_size * head_dim) * count, COPY_THREADS))
        return fail(FQ_ERR_RANGE, "%d pages of %d heads are more than one launch holds", count, heads_kv);
    return launch_kv_copy_pages(k_cache, v_cache, k_scale, v_scale, pages, heads_kv, page_size, head_dim, from, to, count, static_cast<hipStream_t>(stream));
}

}  // extern "C"
