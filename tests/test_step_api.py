"""The calls around the products and the cache check their arguments on the host before anything is launched (no GPU needed)."""
import pytest
import torch

import paper_2402_17985_amd as fq

P = 0x1000          # aligned, never dereferenced
NULL, SHAPE, DTYPE, RANGE, ALIGN, HIP, WORKSPACE = 1, 2, 3, 4, 5, 6, 7


def norm(**k):
    a = dict(X=P, x_dtype=fq.FQ_BF16, M=4, K=64, ldx=64, R=P, r_dtype=fq.FQ_F32, ldr=64, R_out=P, ldro=64, gamma=P, g_dtype=fq.FQ_F16, eps=1e-5, Y=2 * P,
             y_dtype=fq.FQ_BF16, ldy=64, src_idx=P, rep=P, Kpad=128, bits=8, absmax_in=None, Xq_out=P, s_x_out=P, workspace=P, workspace_bytes=1 << 20, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_rms_norm_quant(*{**a, **k}.values())


def weights(**k):
    a = dict(W=P, w_dtype=fq.FQ_F32, N=8, K=64, ldw=64, group=64, Wq_out=P, S_out=P, B_out=P, s_dtype=fq.FQ_F16, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_group_weights_i4(*{**a, **k}.values())


def product(**k):
    a = dict(X=P, x_dtype=fq.FQ_BF16, M=4, K=64, ldx=64, Wq=P, S=P, B=P, s_dtype=fq.FQ_F16, group=64, N=8, bias=P, Y=P, y_dtype=fq.FQ_F32, ldy=8, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_linear_group_i4(*{**a, **k}.values())


def pages(**k):
    a = dict(k_cache=P, v_cache=P, k_scale=P, v_scale=P, pages=9, heads_kv=2, page_size=64, head_dim=128, src=P, dst=P, count=3, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_kv_copy_pages(*{**a, **k}.values())


@pytest.mark.parametrize("args,code", [
    (dict(X=None), NULL), (dict(X=P + 8), ALIGN), (dict(x_dtype=fq.FQ_I32), DTYPE), (dict(M=0), SHAPE), (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(ldx=60), SHAPE),
    (dict(ldx=68), SHAPE), (dict(R=None), NULL), (dict(R_out=None), NULL), (dict(r_dtype=7), DTYPE), (dict(ldr=65), SHAPE), (dict(ldro=32), SHAPE),
    (dict(R_out=P + 4), ALIGN), (dict(gamma=None), NULL), (dict(gamma=P + 2), ALIGN), (dict(g_dtype=fq.FQ_I32), DTYPE), (dict(eps=0.0), RANGE), (dict(eps=-1e-5), RANGE),
    (dict(eps=float("nan")), RANGE), (dict(eps=float("inf")), RANGE), (dict(Y=None, Xq_out=None), NULL), (dict(y_dtype=fq.FQ_I32), DTYPE), (dict(ldy=63), SHAPE),
    (dict(Y=P), RANGE), (dict(K=32776, ldx=32776, ldr=32776, ldro=32776, ldy=32776), RANGE), (dict(src_idx=None), NULL), (dict(src_idx=P + 4), ALIGN), (dict(rep=None), NULL),
    (dict(rep=P + 2), ALIGN), (dict(Kpad=0), SHAPE), (dict(Kpad=80), SHAPE), (dict(Kpad=131072), RANGE), (dict(bits=5), DTYPE), (dict(bits=6, Kpad=96), SHAPE),
    (dict(Xq_out=P + 8), ALIGN), (dict(s_x_out=None), NULL), (dict(workspace=None), NULL), (dict(workspace=P + 4), ALIGN), (dict(workspace_bytes=100), WORKSPACE)])
def test_norm_refusals(args, code):
    assert norm(**args) == code and fq.lib().fq_last_error_string()


@pytest.mark.parametrize("args,code", [
    (dict(W=None), NULL), (dict(W=P + 8), ALIGN), (dict(w_dtype=fq.FQ_I32), DTYPE), (dict(N=0), SHAPE), (dict(K=48), SHAPE), (dict(K=80, ldw=80), SHAPE), (dict(ldw=32), SHAPE),
    (dict(ldw=66), SHAPE), (dict(group=16), SHAPE), (dict(group=0), SHAPE), (dict(group=256), SHAPE), (dict(Wq_out=None), NULL), (dict(Wq_out=P + 4), ALIGN),
    (dict(S_out=None), NULL), (dict(S_out=P + 2), ALIGN), (dict(B_out=P + 2), ALIGN), (dict(s_dtype=fq.FQ_I32), DTYPE), (dict(N=2**31 - 1), RANGE)])
def test_weights_refusals(args, code):
    assert weights(**args) == code and fq.lib().fq_last_error_string()


@pytest.mark.parametrize("args,code", [
    (dict(X=None), NULL), (dict(X=P + 8), ALIGN), (dict(x_dtype=fq.FQ_F32), DTYPE), (dict(x_dtype=fq.FQ_I32), DTYPE), (dict(M=0), SHAPE), (dict(K=16, ldx=16), SHAPE),
    (dict(K=72, ldx=72), SHAPE), (dict(ldx=56), SHAPE), (dict(ldx=68), SHAPE), (dict(Wq=None), NULL), (dict(Wq=P + 8), ALIGN), (dict(S=None), NULL), (dict(S=P + 2), ALIGN),
    (dict(B=P + 2), ALIGN), (dict(s_dtype=9), DTYPE), (dict(group=96), SHAPE), (dict(N=0), SHAPE), (dict(bias=P + 4), ALIGN), (dict(Y=None), NULL), (dict(Y=P + 4), ALIGN),
    (dict(y_dtype=fq.FQ_I32), DTYPE), (dict(ldy=7), SHAPE), (dict(ldx=2**24 + 8), RANGE), (dict(K=2**24 + 32, ldx=2**25), RANGE), (dict(M=2**31 - 1, N=2**31 - 1, ldy=2**31 - 1), RANGE)])
def test_product_refusals(args, code):
    assert product(**args) == code and fq.lib().fq_last_error_string()


@pytest.mark.parametrize("args,code", [
    (dict(k_cache=None), NULL), (dict(v_cache=P + 8), ALIGN), (dict(k_scale=None), NULL), (dict(v_scale=P + 4), ALIGN), (dict(pages=0), SHAPE), (dict(heads_kv=0), RANGE),
    (dict(heads_kv=20000), RANGE), (dict(page_size=32), SHAPE), (dict(head_dim=72), SHAPE), (dict(count=-1), SHAPE), (dict(src=None), NULL), (dict(dst=None), NULL),
    (dict(src=P + 2), ALIGN), (dict(dst=P + 1), ALIGN), (dict(count=2**31 - 1), RANGE)])
def test_pages_refusals(args, code):
    assert pages(**args) == code and fq.lib().fq_last_error_string()


def test_what_is_not_wanted_may_be_null():
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU: reaching the launch is what comes back as an error")
    for args in (dict(R=None, R_out=None), dict(Y=None), dict(Xq_out=None, s_x_out=None, src_idx=None, rep=None, workspace=None, workspace_bytes=0),
                 dict(absmax_in=P, workspace=None, workspace_bytes=0)):
        assert norm(**args) == HIP
    assert weights(B_out=None) == HIP and product(B=None, bias=None) == HIP
    assert pages(count=0, src=None, dst=None) == 0


def test_a_failing_runtime_comes_back_as_an_error():
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU: the failing runtime is the forced condition")
    for call in (norm, weights, product, pages):
        assert call() == HIP and fq.lib().fq_last_error_string()


def test_workspace_is_checked_against_the_query():
    need = fq.fq_rms_norm_workspace_bytes(4, 64, 128)
    assert norm(workspace_bytes=need - 1) == WORKSPACE
    assert fq.fq_rms_norm_workspace_bytes(0, 64, 128) == 16      # sizes that the call refuses


def test_rows_are_counted_in_32_bits():
    """A workgroup adds their number, up to 4096, to a row's to find its next one."""
    for rows in (2**31 - 1, 2**31 - 4096):
        assert norm(M=rows, absmax_in=P) == RANGE and norm(M=rows, workspace_bytes=1 << 40) == RANGE
    if not torch.cuda.is_available():
        assert norm(M=2**31 - 4097, absmax_in=P) == HIP
