"""Scores far beyond what their differences need: the softmax is all but one key's, and the result that key's values, whatever the size."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def _check(y, q, k, v, scale, hidden, x, half_p, where):
    """One head: rows whose largest score is the largest by far more than any rounding (1e-4 of the sizes that make it up, and 40) are that key's values, but
    for the output's rounding and, as the weight need not be a power of two, half_p, the weight's; all rows are finite and within the values' range.
    Returns how many rows were looked at."""
    s = np.where(hidden, -np.inf, scale * (q @ k.T))
    size = scale * (np.abs(q) @ np.abs(k).T).max(1)
    order = np.argsort(s, axis=1)
    rows = np.arange(len(q))
    clear = s[rows, order[:, -1]] - s[rows, order[:, -2]] > 40 + 1e-4 * size
    got, want = y.float().cpu().numpy().astype(np.float64), v[order[:, -1]]
    assert np.isfinite(got).all(), f"{where}: not finite"
    assert (np.abs(got) <= np.abs(v).max() * 1.01).all(), where
    assert (np.abs(got - want)[clear] <= (U.HALF_STEP[x] + half_p) * 1.01 * np.abs(want)[clear] + 1e-6 * np.abs(v).max()).all(), where
    return clear.sum()


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("columns", ["few", "many"])
@pytest.mark.parametrize("scale", [1.0, 1e2, 1e4, 1e6, 1e9, 1e14])
def test_cache_attention_of_huge_scores(x, columns, scale):
    rng = np.random.default_rng(int(np.log10(scale)))
    dim, page, heads, batch, most = 64, 64, (8, 2), 200, 1 if columns == "few" else 20
    lens, queries = [500, 300] + [0] * (batch - 2), [most, most] + [0] * (batch - 2)
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads[1], page, dim)
    cu = U.offsets(queries)
    q, qn = U.packed(rng, sum(queries), heads[0], dim, x, scale=30.0)
    size = fq.fq_attn_cache_workspace_bytes(batch, sum(queries), most, 500, *heads, dim)
    assert size == 16
    y, ws = torch.full_like(q, 7.0), torch.empty(size, dtype=torch.uint8, device=U.DEV)
    print(f"[huge] {x} {columns} scale={scale}", flush=True)
    fq.fq_attn_cache(q, U.i32(cu), U.i32(lens), most, 500, *U.to_dev(kc, vc, ks, vs), U.i32(table), scale, y, ws)
    torch.cuda.synchronize()
    clear = 0
    for b in range(2):
        at = table[b, :-(-lens[b] // page)]
        for head in range(heads[0]):
            h = head // 4
            k = (kc[at, h].astype(np.float64) * ks[at, h, None, None].astype(np.float64)).reshape(-1, dim)[:lens[b]]
            v = (vc[at, h].astype(np.float64) * vs[at, h, None, None].astype(np.float64)).transpose(0, 2, 1).reshape(-1, dim)[:lens[b]]
            hidden = np.arange(lens[b])[None] > lens[b] - most + np.arange(most)[:, None]
            clear += _check(y[cu[b]:cu[b + 1], head], qn[cu[b]:cu[b + 1], head].astype(np.float64), k, v, scale, hidden, x, 0.0 if columns == "few" else 2.0**-11,
                            f"{b} {head}")
    assert clear >= 4


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [1.0, 1e2, 1e4, 1e6, 1e9, 1e14])
def test_prompt_attention_of_huge_scores(x, dim, scale):
    rng = np.random.default_rng(dim + int(np.log10(scale)))
    lens = [300, 70]
    (q, qn), (k, kn), (v, vn) = (U.packed(rng, sum(lens), h, dim, x, scale=c) for h, c in ((4, 30.0), (2, 30.0), (2, 1.0)))
    cu, y = U.offsets(lens), torch.full_like(q, 7.0)
    print(f"[huge prompt] {x} dim={dim} scale={scale}", flush=True)
    fq.fq_attn_prompt(q, k, v, U.i32(cu), U.i32(cu), 300, scale, y)
    torch.cuda.synchronize()
    clear = 0
    for b, n in enumerate(lens):
        rows = slice(cu[b] + 1, cu[b + 1])      # (a first row sees one key only)
        for head in range(4):
            clear += _check(y[rows, head], qn[rows, head].astype(np.float64), kn[cu[b]:cu[b + 1], head // 2].astype(np.float64), vn[cu[b]:cu[b + 1], head // 2].astype(np.float64), scale,
                            np.arange(n)[None] > 1 + np.arange(n - 1)[:, None], x, U.HALF_STEP[x], f"{b} {head}")
    assert clear >= 100


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("columns", ["few", "many"])
def test_scores_that_grow_by_single_steps_of_fp32(x, columns):
    """Pages whose keys' scales are neighbours in fp32: scores of 2^24 to 2^31 that differ by one step, which may be less, as much or more than what the running
    maximum may lag behind."""
    rng = np.random.default_rng(3)
    dim, page, heads, batch, most = 64, 64, (32, 4), 130, 1 if columns == "few" else 5
    lens, queries = [1500] * 8 + [0] * (batch - 8), [most] * 8 + [0] * (batch - 8)
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    kc, vc, ks, vs = U.filled_cache(rng, pages, heads[1], page, dim)
    kc[:], vs[:] = 100, 1.0
    one = np.float32(0.01)
    for b in range(8):
        for i in range(-(-lens[b] // page)):
            ks[table[b, i]] = (one.view(np.int32) + i // 4).view(np.float32)
    q, _ = U.packed(rng, sum(queries), heads[0], dim, x)
    q = q.abs()
    y, ws = torch.full_like(q, 7.0), torch.empty(16, dtype=torch.uint8, device=U.DEV)
    for power in range(24, 32):
        print(f"[single steps] {x} {columns} 2^{power}", flush=True)
        fq.fq_attn_cache(q, U.i32(U.offsets(queries)), U.i32(lens), most, 1500, *U.to_dev(kc, vc, ks, vs), U.i32(table), 2.0**power / 70.0, y, ws)
        torch.cuda.synchronize()
        n = sum(queries)
        assert torch.isfinite(y[:n]).all() and (y[:n].abs() <= 129).all()
