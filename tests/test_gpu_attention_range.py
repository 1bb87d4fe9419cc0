"""Attention where weights and values' scales are far apart: long caches and prompts under a dominating token, pages whose scales fall or rise by large factors,
queries that are not finite."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def _attend(q, cu, lens, table, arrays, scale, max_q, max_len, one_share=True):
    size = fq.fq_attn_cache_workspace_bytes(len(lens), q.shape[0], max_q, max_len, q.shape[1], arrays[0].shape[1], q.shape[2])
    assert (size == 16) == one_share
    y, ws = torch.full_like(q, 7.0), torch.full((size,), 0xFF, dtype=torch.uint8, device=U.DEV)
    fq.fq_attn_cache(q, U.i32(cu), U.i32(lens), max_q, max_len, *U.to_dev(*arrays), U.i32(table), scale, y, ws)
    torch.cuda.synchronize()
    return y


def _queries(rng, tokens, heads, dim, x):
    """Rows of nearly equal elements, about 1."""
    q = torch.from_numpy((1.0 + 0.01 * rng.standard_normal((tokens, heads, 1)) + 0.002 * rng.standard_normal((tokens, heads, dim))).astype(np.float32)).to(U.TYPES[x])
    return q.to(U.DEV), q.float().numpy()


# ------------------------------------------------------------------------------------------------
def _ladder(rng, dim, page, lens, heads, v_scales, gap):
    """A cache in which every sequence's page i has values' scales v_scales[i % n] and scores that rise by `gap` nats from page to page."""
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads, page, dim)
    vc[:] = rng.integers(20, 100, vc.shape)
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            kc[table[b, i]] = (25 if gap >= 0 else -25) * (i % 5 - 2) + rng.integers(-2, 3, kc[0].shape)
            vs[table[b, i]] = v_scales[i % len(v_scales)]
    ks[:] = (abs(gap) if gap else 1.0) / (25 * dim)
    return table, (kc, vc, ks, vs)


LADDERS = {"down": [2.0**(-59 * i) for i in range(3)], "up": [2.0**(59 * i - 118) for i in range(3)], "down by halves of it": [2.0**(-30 * i) for i in range(5)],
           "zeros between": [1.0, 0.0, 2.0**-59, 0.0, 2.0**-118], "from zero": [0.0, 2.0**-100, 2.0**-40, 2.0**-126, 1.0], "up and down": [2.0**-60, 2.0**60, 2.0**-60, 1.0, 2.0**-59],
           "wide": [2.0**100, 2.0**-20, 2.0**41, 2.0**-79, 2.0**-126]}


@pytest.mark.parametrize("gap", [0.0, 41.0, -41.0])
@pytest.mark.parametrize("ladder", list(LADDERS))
@pytest.mark.parametrize("columns", ["many", "few"])
def test_pages_whose_scales_fall_and_rise_step_by_step(columns, ladder, gap):
    rng = np.random.default_rng(len(ladder))
    dim, page, heads, most = 64, 64, (16, 8), 32 if columns == "many" else 2
    batch = 50
    lens = [int(n) for n in rng.integers(32, 320, batch)]
    lens[:3] = [320, 192, 257]
    queries = [most if b < 4 else 0 for b in range(batch)]
    table, arrays = _ladder(rng, dim, page, lens, heads[1], LADDERS[ladder], gap)
    q, qn = _queries(rng, sum(queries), heads[0], dim, "bf16")
    print(f"[ladder] {columns} {ladder} gap={gap}", flush=True)
    y = _attend(q, U.offsets(queries), lens, table, arrays, 1.0, most, 5000)
    exact, bound = U.cache_rows(qn, U.offsets(queries), lens, table, *arrays, 1.0, "bf16", columns)
    U.check(y, exact, bound, "ladder")


@pytest.mark.parametrize("columns", ["many", "few"])
def test_values_near_the_largest(columns):
    """Values of up to 2^115: what the accumulators hold of 320 of them is still a number."""
    rng = np.random.default_rng(4)
    most, batch = 32 if columns == "many" else 2, 50
    lens, queries = [320, 200, 64] + [0] * (batch - 3), [most] * 3 + [0] * (batch - 3)
    table, arrays = _ladder(rng, 64, 64, lens, 8, [2.0**108, 2.0**107, 2.0**90], 0.0)
    q, qn = _queries(rng, sum(queries), 16, 64, "bf16")
    print(f"[near the largest] {columns}", flush=True)
    y = _attend(q, U.offsets(queries), lens, table, arrays, 1.0, most, 5000)
    exact, bound = U.cache_rows(qn, U.offsets(queries), lens, table, *arrays, 1.0, "bf16", columns)
    U.check(y, exact, bound, "near the largest")


def test_scales_that_fall_across_shares():
    """The same with keys that are shared out: parts of very different units meet."""
    rng = np.random.default_rng(12)
    lens, queries = [1600, 900], [64, 33]
    for name in LADDERS:
        table, arrays = _ladder(rng, 64, 64, lens, 2, LADDERS[name], 20.0)
        q, qn = _queries(rng, sum(queries), 4, 64, "bf16")
        print(f"[ladder in shares] {name}", flush=True)
        y = _attend(q, U.offsets(queries), lens, table, arrays, 1.0, 64, 1 << 20, one_share=False)
        exact, bound = U.cache_rows(qn, U.offsets(queries), lens, table, *arrays, 1.0, "bf16", "many")
        U.check(y, exact, bound, "ladder in shares")


# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [17.0, 17.7])
def test_long_prompts_whose_weights_lie_in_one_token_and_all_others(x, gap):
    """The dominating key's values are 1, all others 0: the sum that divides has to hold what 2^19 weights of e^-gap add up to."""
    rng = np.random.default_rng(int(10 * gap))
    dim, keys, n = 64, 1 << 19, 5
    q, qn = _queries(rng, n, 2, dim, x)
    k = (rng.integers(-20, 21, (keys, 1, dim)) / 100.0).astype(np.float32)
    v = np.zeros((keys, 1, dim), np.float32)
    k[0], v[0] = 1.0, 1.0
    k, v = (torch.from_numpy(a).to(U.TYPES[x]) for a in (k, v))
    y, cu_q, cu_k = torch.full_like(q, 7.0), [0, n], [0, keys]
    print(f"[prompt sum] {x} gap={gap}", flush=True)
    fq.fq_attn_prompt(q, k.to(U.DEV), v.to(U.DEV), U.i32(cu_q), U.i32(cu_k), n, gap / dim, y)
    torch.cuda.synchronize()
    exact, bound = U.prompt_rows(qn, k.float().numpy(), v.float().numpy(), cu_q, cu_k, gap / dim, True, x)
    U.check(y, exact, bound, "prompt sum")


# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("columns", ["few", "many"])
@pytest.mark.parametrize("gap,spread", [(17.0, 20), (17.7, 20), (17.7, 0)])
def test_long_caches_under_a_dominating_token(x, columns, gap, spread):
    """One key holds nearly all the weight and its values are zero: the result is what the many others add up to, each of e^-gap."""
    rng = np.random.default_rng(int(10 * gap) + spread)
    dim, page, heads, batch, most = 64, 64, (8, 1), 300, 1 if columns == "few" else 16
    lens = [131072, 70001] + [0] * (batch - 2)
    queries = [most, most] + [0] * (batch - 2)
    kc, vc, ks, vs = U.filled_cache(rng, 8, 1, page, dim)
    kc[:] = rng.integers(-spread, spread + 1, kc.shape)
    vc[:] = rng.integers(20, 61, vc.shape)
    kc[0, 0, 0], vc[0, 0, :, 0] = 100, 0
    ks[:], vs[:] = gap / (100 * dim), 1.0 / 64
    table = np.full((batch, 2048), -1, np.int32)
    for b in range(2):
        table[b, 0], table[b, 1:] = 0, rng.integers(1, 8, 2047)
    q, qn = _queries(rng, sum(queries), heads[0], dim, x)
    print(f"[sink] {x} {columns} gap={gap} spread={spread}", flush=True)
    y = _attend(q, U.offsets(queries), lens, table, (kc, vc, ks, vs), 1.0, most, 131072)
    exact, bound = U.cache_rows(qn, U.offsets(queries), lens, table, kc, vc, ks, vs, 1.0, x, columns)
    assert (bound < 0.1 * np.abs(exact)).all()
    U.check(y, exact, bound, "sink")


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [17.0, 17.7])
def test_long_prompts_under_a_dominating_token(x, gap):
    rng = np.random.default_rng(int(10 * gap))
    dim, keys, n = 64, 131072, 5
    q, qn = _queries(rng, n, 2, dim, x)
    k = (rng.integers(-20, 21, (keys, 1, dim)) / 100.0).astype(np.float32)
    v = rng.integers(20, 61, (keys, 1, dim)).astype(np.float32) / np.float32(64.0)
    k[0], v[0] = 1.0, 0.0
    k, v = (torch.from_numpy(a.astype(np.float32)).to(U.TYPES[x]) for a in (k, v))
    y, cu_q, cu_k = torch.full_like(q, 7.0), [0, n], [0, keys]
    print(f"[prompt sink] {x} gap={gap}", flush=True)
    fq.fq_attn_prompt(q, k.to(U.DEV), v.to(U.DEV), U.i32(cu_q), U.i32(cu_k), n, gap / dim, y)
    torch.cuda.synchronize()
    exact, bound = U.prompt_rows(qn, k.float().numpy(), v.float().numpy(), cu_q, cu_k, gap / dim, True, x)
    assert (bound < 0.1 * np.abs(exact)).all()
    U.check(y, exact, bound, "prompt sink")


# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("queries,max_len", [([1, 1, 1, 1], 700), ([4, 2, 3, 0], 700), ([40, 33, 5, 0], 1 << 20), ([1, 1, 1, 1], 60000)])
def test_queries_that_are_not_finite_show_and_stay_alone(x, bad, queries, max_len):
    """A query with an element that is not finite gives no finite result (a plausible one would hide it), and leaves all other rows and heads as they
    are; where it sees no key the result is 0 as ever."""
    rng = np.random.default_rng(sum(queries))
    lens, heads, dim = [600, 130, 200, 0], (8, 2), 128
    table, pages = U.page_tables(rng, [-(-n // 64) for n in lens])
    arrays, cu = U.filled_cache(rng, pages, heads[1], 64, dim), U.offsets(queries)
    q, _ = U.packed(rng, sum(queries), heads[0], dim, x)
    size = fq.fq_attn_cache_workspace_bytes(4, q.shape[0], max(queries), max_len, *heads, dim)
    dev, ws, tab, cud, ln = U.to_dev(*arrays), torch.empty(size, dtype=torch.uint8, device=U.DEV), U.i32(table), U.i32(cu), U.i32(lens)

    def call(rows):
        y = torch.full(q.shape, 7.0, dtype=q.dtype, device=U.DEV)
        fq.fq_attn_cache(rows, cud, ln, max(queries), max_len, *dev, tab, 0.09, y, ws)
        torch.cuda.synchronize()
        return y
    print(f"[not finite] {x} {bad} queries={queries} max_len={max_len}", flush=True)
    want, spoiled = call(q), q.clone()
    at = [(0, 3, 5), (int(cu[1]), 0, 127), (int(cu[2]), 7, 64)] + ([(int(cu[3]), 1, 0)] if queries[3] else [])
    for row, head, d in at:
        spoiled[row, head, d] = bad
    got = call(spoiled)
    for row, head, _ in at[:3]:
        assert not torch.isfinite(got[row, head]).any(), (row, head)
    if queries[3]:
        assert (got[int(cu[3])] == 0).all()
    same = torch.ones(q.shape[:2], dtype=torch.bool, device=U.DEV)
    for row, head, _ in at:
        same[row, head] = False
    assert torch.equal(got[same], want[same])


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("columns", ["many", "few", "shares"])
@pytest.mark.parametrize("nats", [-300.0, -100000.0])
def test_pages_that_do_not_exist_beside_scores_far_below_zero(x, columns, nats):
    """A page that is left out has scales of 0; it must not pass for scores of 0."""
    rng = np.random.default_rng(int(-nats))
    dim, heads = 64, (8, 2)
    batch, most = (2, 40) if columns == "shares" else (200, 20 if columns == "many" else 1)
    lens, queries = [700, 300] + [0] * (batch - 2), [most, min(most, 33)] + [0] * (batch - 2)
    table, pages = U.page_tables(rng, [-(-n // 64) for n in lens])
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads[1], 64, dim)
    kc[:] = rng.integers(-101, -99, kc.shape)
    ks[:] = -nats / (100 * dim)
    for b, i in ((0, 0), (0, 5), (0, 10), (1, 4)):
        table[b, i] = -1
    cu = U.offsets(queries)
    q, qn = _queries(rng, sum(queries), heads[0], dim, x)
    print(f"[missing pages] {x} {columns} {nats}", flush=True)
    y = _attend(q, cu, lens, table, (kc, vc, ks, vs), 1.0, most, 1 << 20 if columns == "shares" else 700, one_share=columns != "shares")
    assert torch.isfinite(y).all()
    for b in range(2):
        there = np.repeat(table[b, :-(-lens[b] // 64)] >= 0, 64)[:lens[b]]
        for head in (0, 3, 5):
            at, h = np.maximum(table[b, :-(-lens[b] // 64)], 0), head // 4
            k = kc[at, h].reshape(-1, dim)[:lens[b]].astype(np.float64) * ks[0, 0]
            v = (vc[at, h].transpose(0, 2, 1) * vs[at, h][:, None, None].astype(np.float64)).reshape(-1, dim)[:lens[b]]
            for i in range(queries[b]):
                row = int(cu[b]) + i
                seen = there & (np.arange(lens[b]) <= lens[b] - queries[b] + i)
                s = k[seen] @ qn[row, head].astype(np.float64)
                assert s.max() < nats / 2
                got, size = y[row, head].float().cpu().numpy(), np.abs(v[seen]).max(0)
                if nats == -300.0:      # a score's sums and the fused exponent are off by 2^-15 of it at most (1152 is nine times the codes): 1 % of a weight
                    w = np.exp(s - s.max())
                    assert (np.abs(got - w @ v[seen] / w.sum()) <= 0.03 * (w @ np.abs(v[seen]) / w.sum()) + U.HALF_STEP[x] * size).all()
                assert np.abs(got).max() > 0 and (np.abs(got) <= 1.01 * size).all()
