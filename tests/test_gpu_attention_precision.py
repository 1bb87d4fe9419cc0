"""How exact the attention calls are on ordinary inputs: the root mean square of their errors against 64 bits, in units of what rounding the exact result
to the output's type alone gives.

What adds to that rounding, as independent errors of the weights: half a step of the type that probabilities are rounded to, 1 for the output's own type
(sqrt 2 in all) and 2^-3 or less for fp16 probabilities of bf16 calls (1.01); with few columns of fp16 probabilities as two values (0) and queries as integers
of 1 / 32512 of the largest: on these inputs 3e-5 of a weight where fp16 rounds by 2e-4 (1.02), and the 1152 that a step's products carry, 2e-7 of 1152 times
a step's weight, 4e-5 (1.02).  1.1 and 1.5 leave room for the inputs' chance."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def _cache_ratio(rng, x, dim, page, heads, lens, queries, max_len, one_share, columns):
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    arrays = U.ordinary_cache(rng, pages, heads[1], page, dim)
    cu, most = U.offsets(queries), max(queries)
    q, qn = U.packed(rng, sum(queries), heads[0], dim, x)
    size = fq.fq_attn_cache_workspace_bytes(len(lens), q.shape[0], most, max_len, *heads, dim)
    assert (size == 16) == one_share
    y, ws = torch.empty(q.shape, dtype=q.dtype, device=U.DEV), torch.empty(size, dtype=torch.uint8, device=U.DEV)
    print(f"[precision] {x} dim={dim} heads={heads} lens={lens[:3]} queries={queries[:3]} max_len={max_len}", flush=True)
    fq.fq_attn_cache(q, U.i32(cu), U.i32(lens), most, max_len, *U.to_dev(*arrays), U.i32(table), dim**-0.5, y, ws)
    torch.cuda.synchronize()
    exact, bound = U.cache_rows(qn, cu, lens, table, *arrays, dim**-0.5, x, columns)
    U.check(y, exact, bound, "precision")
    ratio = U.error_ratio(y, exact, x)
    print(f"  {ratio:.3f} times a rounding's error", flush=True)
    return ratio


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page,heads,lens,queries", [(128, 64, (16, 2), [1001, 130, 700, 64], [1, 1, 1, 1]), (80, 128, (8, 8), [500, 77, 2000], [5, 5, 5]),
                                                         (64, 64, (8, 2), [900, 300], [8, 3])])
@pytest.mark.parametrize("max_len", [2000, 1 << 20])
def test_few_columns_are_as_exact_as_their_output(x, dim, page, heads, lens, queries, max_len):
    assert _cache_ratio(np.random.default_rng(dim), x, dim, page, heads, lens, queries, max_len, False, "few") < 1.1


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_few_columns_of_whole_sequences_are_as_exact_as_their_output(x, dim):
    rng = np.random.default_rng(dim + 1)
    lens = [int(n) for n in rng.integers(50, 600, 40)]
    assert _cache_ratio(rng, x, dim, 64, (16, 8), lens, [1] * 40, 600, True, "few") < 1.1


@pytest.mark.parametrize("x,limit", [("bf16", 1.1), ("f16", 1.5)])
@pytest.mark.parametrize("dim,page", [(64, 64), (96, 128), (128, 64)])
@pytest.mark.parametrize("one_share", [True, False])
def test_many_columns(x, limit, dim, page, one_share):
    rng = np.random.default_rng(dim + 2)
    if one_share:
        assert _cache_ratio(rng, x, dim, page, (16, 8), [200] * 20 + [333] * 30, [32] * 2 + [1] * 48, 5000, True, "many") < limit
    else:
        assert _cache_ratio(rng, x, dim, page, (8, 2), [900, 500], [70, 33], 1 << 20, False, "many") < limit


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(x, dim, causal):
    rng = np.random.default_rng(dim + 3)
    lens = [300, 64, 700]
    q, k, v = (U.packed(rng, sum(lens), h, dim, x) for h in (4, 2, 2))
    cu, y = U.offsets(lens), torch.empty((sum(lens), 4, dim), dtype=U.TYPES[x], device=U.DEV)
    print(f"[precision] prompt {x} dim={dim} causal={causal}", flush=True)
    fq.fq_attn_prompt(q[0], k[0], v[0], U.i32(cu), U.i32(cu), max(lens), dim**-0.5, y, causal=causal)
    torch.cuda.synchronize()
    exact, bound = U.prompt_rows(q[1], k[1], v[1], cu, cu, dim**-0.5, causal, x)
    U.check(y, exact, bound, "precision")
    ratio = U.error_ratio(y, exact, x)
    print(f"  {ratio:.3f} times a rounding's error", flush=True)
    assert ratio < 1.5
