"""The attention calls on the GPU against their plain forms: cache codes, scales and rotated rows bit for bit, attention within
bounds that follow from the roundings."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import attention as A
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def _angles(rng, rows, rope):
    if not rope:
        return None, None
    at = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rope, 2) / rope)
    return np.cos(at).astype(np.float32), np.sin(at).astype(np.float32)


def _append_both(rng, x, dim, page, heads_q, heads_kv, past, new, rope, interleaved, pad=16, scale=1.0, in_place=False, spare_rows=0, table=None, pool=None):
    tokens = int(sum(new)) + spare_rows
    q, qn = U.packed(rng, tokens, heads_q, dim, x, pad=pad, scale=scale)
    k, kn = U.packed(rng, tokens, heads_kv, dim, x, pad=pad, scale=scale)
    v, vn = U.packed(rng, tokens, heads_kv, dim, x, pad=2 * pad, scale=scale)
    counts = [-(-(p + n) // page) for p, n in zip(past, new)]
    if table is None:
        table, pages = U.page_tables(rng, counts)
    else:
        pages = pool
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads_kv, page, dim)
    cos, sin = _angles(rng, max(p + n for p, n in zip(past, new)) + 1, rope)
    dev = U.to_dev(kc, vc, ks, vs)
    cosd, sind = (None, None) if cos is None else U.to_dev(cos, sin)
    q_out = q if in_place else torch.full((tokens, heads_q, dim), 9.0, dtype=q.dtype, device=U.DEV)
    k_out = k if in_place else torch.full((tokens, heads_kv, dim), 9.0, dtype=k.dtype, device=U.DEV)
    cu = U.offsets(new)
    print(f"[append] {x} dim={dim} page={page} heads={heads_q}/{heads_kv} past={past} new={new} rope={rope} interleaved={interleaved}", flush=True)
    fq.fq_kv_append(q, k, v, U.i32(cu), U.i32(past), max(1, max(new)), *dev, U.i32(table), rope_cos=cosd, rope_sin=sind, interleaved=interleaved,
                    Q_out=q_out, K_out=k_out)
    torch.cuda.synchronize()
    want_q, want_k = A.append(qn, kn, vn, cu, past, table, kc, vc, ks, vs, cos, sin, interleaved)
    for got, want, name in zip(dev, (kc, vc, ks, vs), ("k_cache", "v_cache", "k_scale", "v_scale")):
        assert np.array_equal(got.cpu().numpy(), want), name
    n = int(sum(new))
    reach = np.zeros(tokens, bool)
    for b, p in enumerate(past):
        reach[cu[b]:cu[b + 1]] = p + np.arange(new[b]) < min(table.shape[1] * page, 1 << 30 if cos is None else len(cos))
    for got, want, inp in ((q_out, want_q, qn), (k_out, want_k, kn)):
        want = torch.from_numpy(want).to(got.dtype).float().numpy()
        left = inp if in_place else np.full_like(want, 9.0)
        assert np.array_equal(got.float().cpu().numpy(), np.where(reach[:, None, None], want, left))
    assert n <= tokens


@pytest.mark.parametrize("x", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,page", [(64, 64), (80, 128), (96, 64), (128, 64), (128, 128)])
@pytest.mark.parametrize("past,new", [([0], [1]), ([64, 5, 63], [1, 1, 1]), ([0, 5, 64, 127, 200], [64, 130, 0, 65, 3]), ([15, 16, 17], [17, 1, 300])])
def test_append_stores_what_the_definition_says(x, dim, page, past, new):
    rng = np.random.default_rng(dim + page + len(past))
    _append_both(rng, x, dim, page, 6, 2, past, new, dim, False)


@pytest.mark.parametrize("x,dim,rope,interleaved", [("bf16", 128, 0, False), ("bf16", 128, 64, False), ("f16", 128, 64, True), ("f32", 80, 80, True),
                                                    ("bf16", 80, 40, False), ("f32", 96, 6, False), ("f16", 64, 6, True), ("bf16", 64, 2, True),
                                                    ("f32", 128, 126, False), ("f32", 128, 124, True)])
def test_append_rotations(x, dim, rope, interleaved):
    rng = np.random.default_rng(rope + dim)
    _append_both(rng, x, dim, 64, 4, 4, [0, 70], [33, 70], rope, interleaved)
    _append_both(rng, x, dim, 64, 5, 1, [3, 0], [1, 1], rope, interleaved, in_place=True)


def test_append_in_place_spare_rows_and_long_groups():
    rng = np.random.default_rng(1)
    _append_both(rng, "bf16", 80, 64, 35, 5, [7, 130, 0], [100, 0, 9], 80, False, in_place=True, spare_rows=5)
    _append_both(rng, "f16", 128, 128, 64, 1, [127, 1], [2, 250], 128, True, spare_rows=130)


@pytest.mark.parametrize("batch,page", [(20, 64), (64, 128), (65, 64), (200, 64)])
def test_append_of_a_long_prompt_beside_single_tokens(batch, page):
    rng = np.random.default_rng(batch)
    past, new = [int(n) for n in rng.integers(0, 150, batch)], [int(n) for n in rng.integers(0, 3, batch)]
    new[batch // 2], new[-1] = 8 * page + 30, page + 1
    _append_both(rng, "bf16", 64, page, 2, 1, past, new, 64, False, spare_rows=3)
    _append_both(rng, "f16", 64, page, 2, 2, [0] * batch, new[::-1], 0, False)


@pytest.mark.parametrize("scale", [0.0, 1e-39, 1e-20, 1e4])
def test_append_of_tiny_huge_and_zero_values(scale):
    _append_both(np.random.default_rng(2), "f32", 64, 64, 2, 2, [0, 10, 64], [70, 3, 1], 64, False, scale=scale)


def test_append_leaves_out_what_has_no_page_and_no_position():
    rng = np.random.default_rng(3)
    table = np.array([[0, 1, -1], [9, 3, 4], [5, 2, 6]], np.int32)      # 7 pages: -1 and 9 are none
    _append_both(rng, "bf16", 64, 64, 4, 2, [60, 0, 150], [100, 130, 80], 64, False, table=table, pool=7)   # 230 > 3 pages
    _append_both(rng, "bf16", 64, 64, 4, 2, [60, 0, 192], [100, 130, 5], 0, False, table=table, pool=7)


def test_append_token_by_token_grows_the_scales():
    rng = np.random.default_rng(4)
    dim, page, heads = 64, 64, 3
    table, pages = U.page_tables(rng, [3, 2])
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads, page, dim)
    dev, tab = U.to_dev(kc, vc, ks, vs), U.i32(table)
    past = np.array([0, 60], np.int32)
    for step in range(70):
        k, kn = U.packed(rng, 2, heads, dim, "bf16", scale=1.0 + 0.3 * (step % 23))
        v, vn = U.packed(rng, 2, heads, dim, "bf16", scale=3.0 - 0.04 * step)
        fq.fq_kv_append(None, k, v, U.i32([0, 1, 2]), U.i32(past), 1, *dev, tab)
        A.append(kn, kn, vn, [0, 1, 2], past, table, kc, vc, ks, vs)
        past += 1
    torch.cuda.synchronize()
    for got, want, name in zip(dev, (kc, vc, ks, vs), ("k_cache", "v_cache", "k_scale", "v_scale")):
        assert np.array_equal(got.cpu().numpy(), want), name


# ------------------------------------------------------------------------------------------------
def _cache_both(rng, x, dim, page, heads_q, heads_kv, lens, queries, scale=None, max_len=None, spare_rows=0, bad=(), stream=None, q_scale=1.0, max_q=None):
    scale = dim ** -0.5 if scale is None else scale
    tokens = int(sum(queries)) + spare_rows
    q, qn = U.packed(rng, tokens, heads_q, dim, x, pad=32, scale=q_scale)
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    for b, i, p in bad:
        table[b, i] = p if p < 0 else pages + p
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads_kv, page, dim)
    used = table[(table >= 0) & (table < pages)]
    idle = np.setdiff1d(np.arange(pages), used)
    ks[idle], vs[idle] = np.nan, np.inf
    cu, max_len, max_q = U.offsets(queries), max_len or max(1, max(lens)), max_q or max(queries)
    y = torch.full((tokens, heads_q, dim), 7.0, dtype=q.dtype, device=U.DEV)
    ws = torch.full((fq.fq_attn_cache_workspace_bytes(len(lens), tokens, max_q, max_len, heads_q, heads_kv, dim),), 0xFF, dtype=torch.uint8, device=U.DEV)
    print(f"[cache] {x} dim={dim} page={page} heads={heads_q}/{heads_kv} lens={lens} queries={queries} ws={ws.numel()}", flush=True)
    fq.fq_attn_cache(q, U.i32(cu), U.i32(lens), max_q, max_len, *U.to_dev(kc, vc, ks, vs), U.i32(table), scale, y, ws)
    torch.cuda.synchronize()
    ks[idle], vs[idle] = 0.0, 0.0
    exact, bound = U.cache_case(qn, cu, lens, table, kc, vc, ks, vs, scale, x, max_q)
    n = int(sum(queries))
    U.check(y[:n], exact[:n], bound[:n], "cache")
    assert (y[n:] == 7.0).all()


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page", [(64, 64), (80, 64), (96, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (10, 2)])
def test_cache_attention_of_single_tokens(x, dim, page, heads):
    rng = np.random.default_rng(dim + page + heads[0])
    _cache_both(rng, x, dim, page, *heads, [1, 0, 63, 64, 65, 300, 128], [1] * 7)


@pytest.mark.parametrize("x,dim,page,heads,lens,queries", [
    ("bf16", 128, 64, (8, 1), [40, 200], [2, 2]),             # 16 columns
    ("f16", 128, 64, (8, 2), [40, 200, 5], [5, 3, 5]),        # 20 columns
    ("bf16", 64, 128, (7, 1), [130, 9], [9, 9]),              # 63 columns, all of a sequence at once
    ("f16", 96, 64, (5, 5), [300, 70], [33, 70]),             # every token of a sequence is a query
    ("bf16", 80, 64, (14, 2), [90, 3], [20, 6]),              # more queries than tokens: some see none
    ("bf16", 128, 64, (16, 1), [200], [30]),
    ("f16", 64, 64, (32, 1), [70, 0, 130], [1, 2, 1]),
    ("f16", 128, 128, (8, 2), [128, 300, 64, 63], [128, 100, 5, 0]),
    ("bf16", 96, 64, (3, 3), [200, 0, 400], [129, 40, 33]),
    ("bf16", 80, 128, (4, 1), [500], [70]), ("f16", 64, 64, (2, 1), [260, 65], [150, 66])])
def test_cache_attention_of_several_tokens(x, dim, page, heads, lens, queries):
    _cache_both(np.random.default_rng(sum(lens)), x, dim, page, *heads, lens, queries, spare_rows=3)
    _cache_both(np.random.default_rng(sum(lens)), x, dim, page, *heads, lens, queries, max_len=1 << 20)     # tiles of 128 from 65 columns on


@pytest.mark.parametrize("x,dim,page", [("bf16", 64, 128), ("f16", 80, 64), ("bf16", 96, 64), ("f16", 96, 128), ("bf16", 128, 64), ("f16", 128, 128), ("bf16", 80, 128)])
@pytest.mark.parametrize("batch,heads,most,shared", [(50, (16, 8), 32, False), (49, (8, 8), 40, False), (13, (24, 8), 139, "some"), (20, (24, 8), 139, False)])
def test_cache_attention_of_many_columns_in_many_workgroups(x, dim, page, batch, heads, most, shared):
    """Tiles of 128 columns, mostly with keys that are not shared out: 64 columns, 40, and several tiles."""
    rng = np.random.default_rng(batch + dim)
    lens = [int(n) for n in rng.integers(0, 180, batch)]
    queries = [int(rng.integers(0, min(n, most) + 1)) for n in lens]
    lens[3], queries[3] = max(190, most), most
    assert shared or fq.fq_attn_cache_workspace_bytes(batch, sum(queries), most, 5000, *heads, dim) == 16
    _cache_both(rng, x, dim, page, *heads, lens, queries, max_len=5000)


@pytest.mark.parametrize("x,dim,page,heads,lens,queries", [
    ("bf16", 128, 64, (2, 1), [3000], [1]), ("f16", 64, 128, (4, 2), [5000, 1, 0, 2100], [1, 1, 1, 1]),
    ("bf16", 80, 64, (2, 2), [257, 1025], [3, 1]), ("f16", 128, 64, (12, 1), [1500, 20], [3, 40]),
    ("bf16", 64, 64, (4, 1), [1100, 600], [70, 9]), ("f16", 96, 128, (6, 2), [2100], [25])])
def test_cache_attention_split_over_the_keys(x, dim, page, heads, lens, queries):
    rng = np.random.default_rng(sum(lens))
    tokens = sum(queries)
    assert fq.fq_attn_cache_workspace_bytes(len(lens), tokens, max(queries), max(lens), *heads, dim) > 16
    _cache_both(rng, x, dim, page, *heads, lens, queries)
    _cache_both(rng, x, dim, page, *heads, lens, queries, max_len=60000)     # a bound far above the lengths


@pytest.mark.parametrize("x,dim,page,heads,lens", [
    ("bf16", 128, 64, (8, 1), [5000]), ("f16", 64, 128, (16, 2), [900, 0, 2100, 1, 130]), ("bf16", 96, 64, (5, 5), [200] * 33), ("f16", 80, 128, (9, 3), [400, 64, 65])])
def test_cache_attention_in_long_shares(x, dim, page, heads, lens):
    """A bound of lengths that makes the shares long: workgroups of two waves."""
    _cache_both(np.random.default_rng(sum(lens)), x, dim, page, *heads, lens, [1] * len(lens), max_len=1 << 20, spare_rows=1)


@pytest.mark.parametrize("batch,heads", [(64, 5), (33, 12), (9, 64), (64, 16)])
def test_cache_attention_of_many_uneven_sequences(batch, heads):
    """Enough work for an order by length: longest first, or folded (at most two workgroups per CU)."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 200, batch)]
    lens[batch // 2], lens[0] = 200, 200
    _cache_both(rng, "bf16", 64, 64, heads, heads, lens, [1] * batch, max_len=1024)


@pytest.mark.parametrize("batch,heads", [(3, (8, 1)), (40, (4, 2)), (64, (12, 3)), (65, (8, 8)), (150, (5, 1))])
def test_cache_attention_of_pieces_beside_single_tokens(batch, heads):
    """Some sequences with many new tokens, most with one, some with none: up to 64 go by their length, more as they come."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 150, batch)]
    queries = [min(1, n) for n in lens]
    lens[batch // 2], queries[batch // 2] = 400, 300
    lens[-1], queries[-1] = 130, 67
    _cache_both(rng, "bf16", 64, 64, *heads, lens, queries, spare_rows=2)
    _cache_both(rng, "f16", 64, 64, *heads, lens, queries, max_len=1 << 20)


def test_cache_attention_with_a_bound_of_queries_far_above_them():
    rng = np.random.default_rng(31)
    _cache_both(rng, "f16", 64, 64, 4, 2, [1500, 80], [1, 1], spare_rows=200, max_q=100000)      # in shares, too
    _cache_both(rng, "f16", 64, 64, 4, 2, [80] * 70, [1] * 70, max_q=100000)


@pytest.mark.parametrize("spread", [1.0, 12.0, 30.0])
def test_cache_attention_of_many_columns_over_pages_of_very_different_scales(spread):
    """Values' scales up to a factor e^60 apart between neighbouring pages, and pages of zeros."""
    rng, real = np.random.default_rng(9), U.filled_cache
    def filled(*shape):
        k, v, ks, vs = real(*shape)
        vs = np.exp(rng.uniform(-spread, spread, vs.shape)).astype(np.float32)
        vs[::4], ks[1::5] = 0.0, 0.0
        return k, v, ks, vs
    try:
        U.filled_cache = filled
        _cache_both(rng, "bf16", 64, 64, 4, 2, [1000, 300], [40, 20], max_len=1 << 20)
        _cache_both(rng, "bf16", 64, 64, 4, 2, [1000, 300], [40, 20])
        _cache_both(rng, "f16", 64, 64, 4, 2, [1000, 300], [1, 2])
    finally:
        U.filled_cache = real


def test_cache_attention_leaves_out_pages_that_do_not_exist():
    _cache_both(np.random.default_rng(5), "f16", 128, 64, 4, 2, [200, 64, 400], [50, 20, 21], bad=((0, 1, -1), (1, 0, 0), (2, 6, 1 << 20), (2, 0, -(1 << 31))))
    _cache_both(np.random.default_rng(5), "f16", 128, 64, 4, 2, [200, 64, 400], [50, 20, 21], bad=((0, 1, -1), (1, 0, 0), (2, 6, 1 << 20), (2, 0, -(1 << 31))), max_len=1 << 20)
    _cache_both(np.random.default_rng(5), "bf16", 64, 64, 4, 2, [200, 64, 400], [1, 1, 2], bad=((0, 1, -1), (1, 0, 0), (2, 6, 1 << 20), (2, 0, -(1 << 31))))


@pytest.mark.parametrize("x,q_scale,scale", [("bf16", 1e30, 1e-31), ("bf16", 1e-38, 1e36), ("f16", 100.0, 1e-3), ("bf16", 6.0, 0.4), ("bf16", 0.0, 1.0)])
def test_cache_attention_of_large_and_small_queries(x, q_scale, scale):
    _cache_both(np.random.default_rng(6), x, 64, 64, 4, 2, [200, 64], [1, 2], q_scale=q_scale, scale=scale)


# ------------------------------------------------------------------------------------------------
def _prompt_both(rng, x, dim, heads_q, heads_kv, queries, keys, causal, scale=None, pad=16, spare=3, q_scale=1.0, max_q=None):
    scale = dim ** -0.5 if scale is None else scale
    q, qn = U.packed(rng, int(sum(queries)) + spare, heads_q, dim, x, pad=pad, scale=q_scale)
    k, kn = U.packed(rng, int(sum(keys)) + spare, heads_kv, dim, x, pad=2 * pad)
    v, vn = U.packed(rng, int(sum(keys)) + spare, heads_kv, dim, x, pad=pad)
    cu_q, cu_k = U.offsets(queries), U.offsets(keys)
    k[cu_k[-1]:], v[cu_k[-1]:] = float("nan"), float("inf")       # behind the last sequence
    y = torch.full((q.shape[0], heads_q, dim), 7.0, dtype=q.dtype, device=U.DEV)
    print(f"[prompt] {x} dim={dim} heads={heads_q}/{heads_kv} queries={queries} keys={keys} causal={causal}", flush=True)
    fq.fq_attn_prompt(q, k, v, U.i32(cu_q), U.i32(cu_k), max_q or max(max(queries), 1), scale, y, causal=causal)
    torch.cuda.synchronize()
    n, m = cu_q[-1], cu_k[-1]
    exact, bound = U.prompt_case(qn[:n], kn[:m], vn[:m], cu_q, cu_k, scale, causal, x)
    U.check(y[:n], exact, bound, "prompt")
    assert (y[n:] == 7.0).all()


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[1], [2, 31, 33], [64, 1, 65, 127], [128, 129, 300]])
def test_prompt_attention(x, dim, causal, lens):
    _prompt_both(np.random.default_rng(dim + sum(lens)), x, dim, 4, 2, lens, lens, causal)


@pytest.mark.parametrize("queries,keys", [([5, 40], [70, 200]), ([1, 1], [129, 64]), ([100, 30, 3], [20, 0, 3]), ([0, 7, 0], [5, 7, 0]), ([200, 1], [64, 0])])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_attention_of_some_queries_and_rows_without_keys(queries, keys, causal):
    _prompt_both(np.random.default_rng(sum(keys)), "bf16", 128, 6, 2, queries, keys, causal)


@pytest.mark.parametrize("batch", [64, 65, 130])
def test_prompt_attention_of_many_sequences(batch):
    """Up to 64 go by their length, more as they come."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 50, batch)]
    lens[batch // 3] = 150
    _prompt_both(rng, "bf16", 64, 3, 1, lens, lens, True)
    _prompt_both(rng, "f16", 64, 1, 1, [n // 2 for n in lens], lens, False)


@pytest.mark.parametrize("batch,heads", [(5, (12, 12)), (20, (3, 1)), (70, (2, 2))])
def test_prompt_attention_of_one_long_sequence_among_short_ones(batch, heads):
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 20, batch)]
    lens[1], lens[batch - 2] = 700, 128
    _prompt_both(rng, "bf16", 64, *heads, lens, lens, True, spare=300)
    _prompt_both(rng, "bf16", 64, *heads, lens, [n + 9 for n in lens], True, max_q=1 << 30)
    _prompt_both(rng, "bf16", 64, *heads, [n // 2 for n in lens], lens, False)


@pytest.mark.parametrize("batch", [3, 100])
def test_prompt_attention_of_a_batch_without_queries(batch):
    rng = np.random.default_rng(3)
    q, k = U.packed(rng, 300, 2, 64, "bf16")[0], U.packed(rng, 3 * batch, 1, 64, "bf16")[0]
    y = torch.full_like(q, 7.0)
    fq.fq_attn_prompt(q, k, k, U.i32([0] * (batch + 1)), U.i32([3 * b for b in range(batch + 1)]), 100, 0.1, y)
    torch.cuda.synchronize()
    assert (y == 7.0).all()


@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (5, 5), (16, 8)])
def test_prompt_attention_of_groups(heads):
    _prompt_both(np.random.default_rng(heads[0]), "f16", 64, *heads, [90, 140], [90, 140], True, pad=0)


@pytest.mark.parametrize("x,q_scale,scale", [("bf16", 1.0, 3.0), ("bf16", 1e-3, 1.0), ("f16", 40.0, 0.1), ("bf16", 0.0, 1.0)])
def test_prompt_attention_of_sharp_and_flat_scores(x, q_scale, scale):
    _prompt_both(np.random.default_rng(8), x, 64, 2, 2, [200], [200], True, q_scale=q_scale, scale=scale)
