// C-ABI layer of the attention calls: argument validation and composition of the kernels.  Nothing here allocates or synchronizes.
#include <cmath>

#include "fq_internal.h"
#include "fq_attn_rules.h"
#include "fq_rules.h"

namespace fq {
namespace {

int check_heads(int heads_q, int heads_kv, int head_dim)
{
    if (heads_q <= 0 || heads_kv <= 0 || heads_q % heads_kv != 0)
        return fail(FQ_ERR_SHAPE, "%d query heads over %d key heads: must be positive, the first a multiple of the second", heads_q, heads_kv);
    if (heads_q > 16384) return fail(FQ_ERR_RANGE, "%d query heads: at most 16384", heads_q);
    for (int d : ATTN_DIMS)
        if (d == head_dim) return FQ_OK;
    return fail(FQ_ERR_SHAPE, "head_dim = %d must be 64, 80, 96 or 128", head_dim);
}

// A packed array [tokens, heads, head_dim] with dense heads and `ld` elements from one token to the next.
int check_packed(const char* what, const void* p, int dtype, int tokens, int heads, int head_dim, long long ld)
{
    if (tokens < 0) return fail(FQ_ERR_SHAPE, "%s: %d tokens", what, tokens);
    if (ld < (long long)heads * head_dim) return fail(FQ_ERR_SHAPE, "%s: token stride %lld < %d heads of %d", what, ld, heads, head_dim);
    if (ld > MAX_TOKEN_STRIDE) return fail(FQ_ERR_RANGE, "%s: token stride of %lld elements, at most 2^22", what, ld);
    if (ld * elem_size(dtype) % 16 != 0) return fail(FQ_ERR_SHAPE, "%s: token stride of %lld elements is not a multiple of 16 bytes", what, ld);
    if (tokens == 0) return FQ_OK;
    if (!p) return fail(FQ_ERR_NULL, "%s is NULL", what);
    if (!aligned16(p)) return fail(FQ_ERR_ALIGN, "%s is not 16-byte aligned", what);
    return FQ_OK;
}

int check_indices(const char* what, const int32_t* p)
{
    if (!p) return fail(FQ_ERR_NULL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return fail(FQ_ERR_ALIGN, "%s is not 4-byte aligned", what);
    return FQ_OK;
}

int check_cache(const int8_t* k_cache, const int8_t* v_cache, const float* k_scale, const float* v_scale, int pages, int page_size,
                const int32_t* page_table, int table_width)
{
    if (!k_cache || !v_cache || !k_scale || !v_scale) return fail(FQ_ERR_NULL, "k_cache, v_cache, k_scale or v_scale is NULL");
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_scale) || !aligned16(v_scale))
        return fail(FQ_ERR_ALIGN, "k_cache, v_cache, k_scale or v_scale is not 16-byte aligned");
    if (page_size != 64 && page_size != 128) return fail(FQ_ERR_SHAPE, "page_size = %d must be 64 or 128", page_size);
    if (pages <= 0 || table_width <= 0) return fail(FQ_ERR_SHAPE, "%d pages, a page table of %d columns", pages, table_width);
    if ((long long)table_width * page_size > (1LL << 30)) return fail(FQ_ERR_RANGE, "a page table that reaches %lld tokens: at most 2^30", (long long)table_width * page_size);
    return check_indices("page_table", page_table);
}

int check_batch(int batch, const char* what, int most)
{
    if (batch <= 0 || batch > 65535) return fail(FQ_ERR_RANGE, "batch = %d must be in 1 .. 65535", batch);
    if (most <= 0) return fail(FQ_ERR_SHAPE, "%s = %d must be positive", what, most);
    return FQ_OK;
}

int check_attention(int x_dtype, float scale)
{
    if (x_dtype != FQ_F16 && x_dtype != FQ_BF16) return fail(FQ_ERR_DTYPE, "dtype %d is not F16 or BF16", x_dtype);
    // the kernels count in powers of two: scale * log2(e) must be finite as well
    if (!(scale > 0.0f) || std::isinf(scale * 1.44269504f)) return fail(FQ_ERR_RANGE, "scale = %g must be positive and at most 2.35e38", (double)scale);
    return FQ_OK;
}

}  // namespace
}  // namespace fq

using namespace fq;

extern "C" {

int fq_kv_append(const void* Q, const void* K, const void* V, int x_dtype, int tokens, int heads_q, int heads_kv, int head_dim,
                 long long ldq, long long ldk, long long ldv, const int32_t* cu_new, const int32_t* past, int batch, int max_new,
                 const float* rope_cos, const float* rope_sin, int rope_rows, int rope_dim, int interleaved,
                 void* Q_out, long long ldqo, void* K_out, long long ldko,
                 int8_t* k_cache, int8_t* v_cache, float* k_scale, float* v_scale, int pages, int page_size,
                 const int32_t* page_table, int table_width, void* stream)
{
    clear_error();
    if (x_dtype != FQ_F32 && x_dtype != FQ_F16 && x_dtype != FQ_BF16) return fail(FQ_ERR_DTYPE, "dtype %d is not F32/F16/BF16", x_dtype);
    int rc = check_heads(heads_q, heads_kv, head_dim);
    if (!rc) rc = check_packed("K", K, x_dtype, tokens, heads_kv, head_dim, ldk);
    if (!rc) rc = check_packed("V", V, x_dtype, tokens, heads_kv, head_dim, ldv);
    if (!rc && Q_out) rc = check_packed("Q", Q, x_dtype, tokens, heads_q, head_dim, ldq);
    if (!rc && Q_out) rc = check_packed("Q_out", Q_out, x_dtype, tokens, heads_q, head_dim, ldqo);
    if (!rc && K_out) rc = check_packed("K_out", K_out, x_dtype, tokens, heads_kv, head_dim, ldko);
    if (!rc) rc = check_batch(batch, "max_new", max_new);
    if (!rc) rc = check_indices("cu_new", cu_new);
    if (!rc) rc = check_indices("past", past);
    if (!rc) rc = check_cache(k_cache, v_cache, k_scale, v_scale, pages, page_size, page_table, table_width);
    if (rc) return rc;
    if (rope_dim < 0 || rope_dim > head_dim || rope_dim % 2 != 0)
        return fail(FQ_ERR_SHAPE, "rope_dim = %d must be even, in 0 .. head_dim = %d", rope_dim, head_dim);
    if (rope_dim > 0) {
        if (!rope_cos || !rope_sin) return fail(FQ_ERR_NULL, "rope_cos or rope_sin is NULL with rope_dim = %d", rope_dim);
        if (!aligned16(rope_cos) || !aligned16(rope_sin)) return fail(FQ_ERR_ALIGN, "rope_cos or rope_sin is not 16-byte aligned");
        if (rope_rows <= 0) return fail(FQ_ERR_SHAPE, "rope_rows = %d must be positive", rope_rows);
    }
    const long long places = append_pages(batch, tokens, max_new, page_size).places * ((Q_out ? 3 : 2) * heads_kv);
    if (!launch_holds(places, append_plan(max_new, page_size, head_dim).threads))
        return fail(FQ_ERR_RANGE, "%d sequences of up to %d new tokens are more than one launch holds", batch, max_new);
    if (tokens == 0) return FQ_OK;
    return launch_kv_append(Q, K, V, x_dtype, tokens, heads_q, heads_kv, head_dim, ldq, ldk, ldv, cu_new, past, batch, max_new, rope_cos, rope_sin,
                            rope_rows, rope_dim, interleaved != 0, Q_out, ldqo, K_out, ldko, k_cache, v_cache, k_scale, v_scale, pages, page_size,
                            page_table, table_width, static_cast<hipStream_t>(stream));
}

size_t fq_attn_cache_workspace_bytes(int batch, int tokens, int max_q, int max_len, int heads_q, int heads_kv, int head_dim)
{
    if (batch <= 0 || tokens < 0 || max_q <= 0 || max_len <= 0 || heads_q <= 0 || heads_kv <= 0 || heads_q < heads_kv || head_dim <= 0) return 16;
    const int splits = cache_plan(batch, tokens, max_q, max_len, heads_q, heads_kv).splits;
    return splits > 1 ? round_up((size_t)tokens * heads_q * splits * (head_dim + 2) * sizeof(float), 16) + 16 : 16;
}

int fq_attn_cache(const void* Q, int x_dtype, int tokens, int heads_q, int heads_kv, int head_dim, long long ldq,
                  const int32_t* cu_q, const int32_t* lens, int batch, int max_q, int max_len,
                  const int8_t* k_cache, const int8_t* v_cache, const float* k_scale, const float* v_scale, int pages, int page_size,
                  const int32_t* page_table, int table_width, float scale, void* Y, long long ldy,
                  void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    int rc = check_attention(x_dtype, scale);
    if (!rc) rc = check_heads(heads_q, heads_kv, head_dim);
    if (!rc) rc = check_packed("Q", Q, x_dtype, tokens, heads_q, head_dim, ldq);
    if (!rc) rc = check_packed("Y", Y, x_dtype, tokens, heads_q, head_dim, ldy);
    if (!rc) rc = check_batch(batch, "max_q", max_q);
    if (!rc) rc = check_indices("cu_q", cu_q);
    if (!rc) rc = check_indices("lens", lens);
    if (!rc) rc = check_cache(k_cache, v_cache, k_scale, v_scale, pages, page_size, page_table, table_width);
    if (rc) return rc;
    if (max_len <= 0) return fail(FQ_ERR_SHAPE, "max_len = %d must be positive", max_len);
    if ((long long)max_q * heads_q >= (1LL << 30)) return fail(FQ_ERR_RANGE, "max_q = %d queries of %d heads: at most 2^30 together", max_q, heads_q);
    if (!cache_holds(cache_plan(batch, tokens, max_q, max_len, heads_q, heads_kv), heads_kv))
        return fail(FQ_ERR_RANGE, "%d sequences of up to %d queries of %d heads are more than one launch holds", batch, max_q, heads_q);
    if (!workspace) return fail(FQ_ERR_NULL, "workspace is NULL");
    if (!aligned16(workspace)) return fail(FQ_ERR_ALIGN, "workspace is not 16-byte aligned");
    const size_t need = fq_attn_cache_workspace_bytes(batch, tokens, max_q, max_len, heads_q, heads_kv, head_dim);
    if (workspace_bytes < need) return fail(FQ_ERR_WORKSPACE, "workspace of %zu bytes < %zu required", workspace_bytes, need);
    if (tokens == 0) return FQ_OK;
    return launch_attn_cache(Q, x_dtype, tokens, heads_q, heads_kv, head_dim, ldq, cu_q, lens, batch, max_q, max_len, k_cache, v_cache, k_scale,
                             v_scale, pages, page_size, page_table, table_width, scale, Y, ldy, workspace,
                             static_cast<hipStream_t>(stream));
}

int fq_attn_prompt(const void* Q, const void* K, const void* V, int x_dtype, int tokens_q, int tokens_k, int heads_q, int heads_kv,
                   int head_dim, long long ldq, long long ldk, long long ldv, const int32_t* cu_q, const int32_t* cu_k, int batch, int max_q,
                   int causal, float scale, void* Y, long long ldy, void* stream)
{
    clear_error();
    int rc = check_attention(x_dtype, scale);
    if (!rc) rc = check_heads(heads_q, heads_kv, head_dim);
    if (!rc) rc = check_packed("Q", Q, x_dtype, tokens_q, heads_q, head_dim, ldq);
    if (!rc) rc = check_packed("K", K, x_dtype, tokens_k, heads_kv, head_dim, ldk);
    if (!rc) rc = check_packed("V", V, x_dtype, tokens_k, heads_kv, head_dim, ldv);
    if (!rc) rc = check_packed("Y", Y, x_dtype, tokens_q, heads_q, head_dim, ldy);
    if (!rc) rc = check_batch(batch, "max_q", max_q);
    if (!rc) rc = check_indices("cu_q", cu_q);
    if (!rc) rc = check_indices("cu_k", cu_k);
    if (rc) return rc;
    const long long places = prompt_workgroups(tokens_q, batch, max_q, heads_q, heads_kv);
    if (places >= (1LL << 31) || !launch_holds(places, PROMPT_THREADS))
        return fail(FQ_ERR_RANGE, "%d sequences of up to %d queries of %d heads are more than one launch holds", batch, max_q, heads_q);
    if (tokens_q == 0) return FQ_OK;
    return launch_attn_prompt(Q, K, V, x_dtype, tokens_q, tokens_k, heads_q, heads_kv, head_dim, ldq, ldk, ldv, cu_q, cu_k, batch, max_q, causal != 0,
                              scale, Y, ldy, static_cast<hipStream_t>(stream));
}

}  // extern "C"
