"""The attention entry points check their arguments on the host before anything is launched (no GPU needed)."""
import pytest
import torch

import paper_2402_17985_amd as fq

P = 0x1000          # aligned, never dereferenced
NULL, SHAPE, DTYPE, RANGE, ALIGN, HIP, WORKSPACE = 1, 2, 3, 4, 5, 6, 7


def append(**k):
    a = dict(Q=P, K=P, V=P, x_dtype=fq.FQ_BF16, tokens=4, heads_q=8, heads_kv=2, head_dim=64, ldq=512, ldk=128, ldv=128, cu_new=P, past=P, batch=2, max_new=2,
             rope_cos=P, rope_sin=P, rope_rows=100, rope_dim=64, interleaved=0, Q_out=P, ldqo=512, K_out=P, ldko=128, k_cache=P, v_cache=P, k_scale=P,
             v_scale=P, pages=4, page_size=64, page_table=P, table_width=2, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_kv_append(*{**a, **k}.values())


def cache(**k):
    a = dict(Q=P, x_dtype=fq.FQ_BF16, tokens=4, heads_q=8, heads_kv=2, head_dim=64, ldq=512, cu_q=P, lens=P, batch=2, max_q=2, max_len=128, k_cache=P, v_cache=P,
             k_scale=P, v_scale=P, pages=4, page_size=64, page_table=P, table_width=2, scale=0.125, Y=P, ldy=512, workspace=P, workspace_bytes=1 << 24,
             stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_attn_cache(*{**a, **k}.values())


def prompt(**k):
    a = dict(Q=P, K=P, V=P, x_dtype=fq.FQ_F16, tokens_q=4, tokens_k=4, heads_q=8, heads_kv=2, head_dim=64, ldq=512, ldk=128, ldv=128, cu_q=P, cu_k=P, batch=2,
             max_q=2, causal=1, scale=0.125, Y=P, ldy=512, stream=None)
    assert set(k) <= set(a)
    return fq.lib().fq_attn_prompt(*{**a, **k}.values())


@pytest.mark.parametrize("call", [append, cache, prompt])
@pytest.mark.parametrize("args,code", [
    (dict(heads_q=0), SHAPE), (dict(heads_kv=0), SHAPE), (dict(heads_q=9), SHAPE), (dict(heads_q=-8), SHAPE), (dict(heads_q=16386), RANGE),
    (dict(head_dim=32), SHAPE), (dict(head_dim=72), SHAPE), (dict(head_dim=256), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(batch=0), RANGE), (dict(batch=65536), RANGE), (dict(x_dtype=fq.FQ_I32), DTYPE), (dict(x_dtype=9), DTYPE),
    (dict(ldq=504), SHAPE), (dict(ldq=516), SHAPE), (dict(ldq=1 << 23), RANGE), (dict(Q=None), NULL), (dict(Q=P + 8), ALIGN)])
def test_shared_refusals(call, args, code):
    assert call(**args) == code
    assert fq.lib().fq_last_error_string()


@pytest.mark.parametrize("args,code", [
    (dict(K=None), NULL), (dict(V=None), NULL), (dict(ldk=64), SHAPE), (dict(ldv=130), SHAPE), (dict(ldk=(1 << 22) + 8), RANGE), (dict(ldqo=511), SHAPE),
    (dict(ldko=0), SHAPE), (dict(K_out=P + 4), ALIGN), (dict(Q_out=P + 4), ALIGN), (dict(tokens=-1), SHAPE), (dict(max_new=0), SHAPE), (dict(cu_new=None), NULL),
    (dict(past=None), NULL), (dict(past=P + 2), ALIGN), (dict(rope_dim=63), SHAPE), (dict(rope_dim=66), SHAPE), (dict(rope_dim=-2), SHAPE),
    (dict(rope_cos=None), NULL), (dict(rope_sin=P + 8), ALIGN), (dict(rope_rows=0), SHAPE), (dict(k_cache=None), NULL), (dict(v_cache=P + 8), ALIGN),
    (dict(k_scale=None), NULL), (dict(v_scale=P + 4), ALIGN), (dict(pages=0), SHAPE), (dict(page_size=32), SHAPE), (dict(page_size=96), SHAPE),
    (dict(page_size=256), SHAPE), (dict(page_table=None), NULL), (dict(table_width=0), SHAPE), (dict(table_width=(1 << 24) + 1), RANGE),
    (dict(batch=65535, max_new=2**31 - 1, tokens=2**31 - 1), RANGE)])
def test_append_refusals(args, code):
    assert append(**args) == code


@pytest.mark.parametrize("args,code", [
    (dict(x_dtype=fq.FQ_F32), DTYPE), (dict(scale=0.0), RANGE), (dict(scale=-1.0), RANGE), (dict(scale=float("nan")), RANGE), (dict(scale=float("inf")), RANGE),
    (dict(Y=None), NULL), (dict(ldy=8), SHAPE), (dict(cu_q=None), NULL), (dict(lens=None), NULL), (dict(lens=P + 1), ALIGN), (dict(max_q=0), SHAPE),
    (dict(max_len=0), SHAPE), (dict(max_len=-5), SHAPE), (dict(max_q=1 << 27), RANGE), (dict(k_scale=P + 4), ALIGN), (dict(pages=-1), SHAPE),
    (dict(page_size=16), SHAPE), (dict(table_width=1 << 30), RANGE), (dict(workspace=None), NULL), (dict(workspace=P + 8), ALIGN), (dict(workspace_bytes=15), WORKSPACE),
    (dict(batch=65535, max_q=100000, tokens=(1 << 31) - 1), RANGE)])
def test_cache_attention_refusals(args, code):
    assert cache(**args) == code


@pytest.mark.parametrize("args,code", [
    (dict(x_dtype=fq.FQ_F32), DTYPE), (dict(scale=0.0), RANGE), (dict(scale=float("inf")), RANGE), (dict(K=None), NULL), (dict(V=P + 2), ALIGN), (dict(ldk=1 << 23), RANGE),
    (dict(ldv=100), SHAPE), (dict(Y=None), NULL), (dict(ldy=513), SHAPE), (dict(cu_q=None), NULL), (dict(cu_k=P + 3), ALIGN), (dict(max_q=0), SHAPE),
    (dict(tokens_k=-1), SHAPE), (dict(batch=65535, max_q=2**31 - 1, tokens_q=2**31 - 1), RANGE)])
def test_prompt_attention_refusals(args, code):
    assert prompt(**args) == code


def test_workspace_is_checked_against_the_query():
    need = fq.fq_attn_cache_workspace_bytes(1, 1, 1, 100000, 8, 8, 128)
    assert need > 1000
    args = dict(tokens=1, heads_q=8, heads_kv=8, head_dim=128, ldq=1024, ldy=1024, batch=1, max_q=1, max_len=100000, table_width=2000, pages=2000)
    assert cache(**args, workspace_bytes=need - 1) == WORKSPACE
    assert fq.fq_attn_cache_workspace_bytes(0, 1, 1, 1, 1, 1, 64) == 16     # sizes that the call refuses


def test_no_tokens_are_no_work():
    """Arrays of no rows may have no memory either; nothing is launched."""
    assert append(tokens=0, Q=None, K=None, V=None, Q_out=None, K_out=None) == 0
    assert cache(tokens=0, Q=None, Y=None) == 0
    assert prompt(tokens_q=0, Q=None, Y=None) == 0
    assert prompt(tokens_q=0, tokens_k=0, Q=None, K=None, V=None, Y=None) == 0


def test_queries_may_be_left_out():
    assert append(Q=None, Q_out=None, tokens=0) == 0
    assert append(Q=None, Q_out=P) == NULL
    assert append(rope_dim=0, rope_cos=None, rope_sin=None, rope_rows=0, tokens=0) == 0


def test_a_failing_runtime_comes_back_as_an_error():
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU: the failing runtime is the forced condition")
    for call in (append, cache, prompt):
        assert call() == HIP
        assert fq.lib().fq_last_error_string()


def test_cache_bookkeeping_rejects_tables_shorter_than_its_sequences():
    with pytest.raises(ValueError, match="rope_cos"):
        fq.FqKvCache(4, 1, 200, 1, 64, rope_cos=torch.zeros(100, 32), rope_sin=torch.zeros(100, 32), device="cpu")
    c = fq.FqKvCache(3, 2, 128, 1, 64, device="cpu")
    c.reserve(0, 65)
    with pytest.raises(RuntimeError, match="free"):
        c.reserve(1, 128)
    with pytest.raises(ValueError, match="128"):
        c.reserve(1, 129)
    c.reserve(1, 64)
    assert sorted(c.held[0] + c.held[1]) == [0, 1, 2] and c.page_table.tolist() == [c.held[0], c.held[1] + [-1]]
    c.release(0)
    assert c.held[0] == [] and c.page_table[0].tolist() == [-1, -1]
    c.reserve(1, 128)
    assert len(c.held[1]) == 2
