"""That the checks of precision see what they are for: the arithmetic of the cache's attention with few columns, followed in NumPy, passes them as it is and
fails them with coarser queries or fewer bits of the probabilities."""
import numpy as np
import pytest
import torch

from tests import attn_util as U


def few_columns(q, codes, k_scale, v_codes, v_scale, scale, x, steps, limbs):
    """One head: q [n, dim], codes and v_codes [keys, dim], scales [keys].  Queries as integers of 1 / steps of their largest magnitude, probabilities as
    the sum of `limbs` fp16 values: 2^7 times them, against the largest of all or, 64 keys that are 2^8 below it, of their own."""
    top = np.abs(q).max(1, keepdims=True)
    s = np.rint(q / top * steps) @ codes.T * (top / steps) * scale * np.log2(np.e) * k_scale
    y, total, best = np.zeros(q.shape), np.zeros((len(q), 1)), np.max(s, 1, keepdims=True)
    for at in range(0, s.shape[1], 64):
        part = s[:, at:at + 64]
        m = part.max(1, keepdims=True)
        below = np.where(m < best - 8, m - best, 0.0)
        w, p = np.exp2(part - best - below + 7), 0.0
        for _ in range(limbs):
            p = p + (w - p).astype(np.float16).astype(np.float64)
        weight = np.exp2(below)
        y += p @ (v_codes[at:at + 64] * v_scale[at:at + 64, None]) * weight
        total += p.sum(1, keepdims=True) * weight
    return torch.from_numpy(y / total).to(U.TYPES[x]).double().numpy()


def _case(x, dim, keys, steps, limbs, seed=0):
    rng = np.random.default_rng(seed)
    n, page = 64, 64
    q = torch.from_numpy(rng.standard_normal((n, 1, dim)).astype(np.float32)).to(U.TYPES[x]).float().numpy()
    kc, vc, ks, vs = U.ordinary_cache(rng, -(-keys // page), 1, page, dim)
    table = np.arange(len(ks), dtype=np.int32)[None]
    results = []
    for i in range(n):                      # one sequence a query: all of them see all keys
        exact, bound = U.cache_rows(q[i:i + 1], [0, 1], [keys], table, kc, vc, ks, vs, dim**-0.5, x, "few")
        got = few_columns(q[i].astype(np.float64), kc[:, 0].reshape(-1, dim)[:keys].astype(np.float64), np.repeat(ks[:, 0].astype(np.float64), page)[:keys],
                          vc[:, 0].transpose(0, 2, 1).reshape(-1, dim)[:keys].astype(np.float64), np.repeat(vs[:, 0].astype(np.float64), page)[:keys], dim**-0.5, x, steps, limbs)
        results.append((got, exact[0], bound[0]))
    got, exact, bound = (np.concatenate(a) for a in zip(*results))
    return U.error_ratio(got, exact, x), np.abs(got - exact) / bound


@pytest.mark.parametrize("x,limbs", [("bf16", 1), ("f16", 2)])
@pytest.mark.parametrize("dim,keys", [(128, 1001), (64, 300)])
def test_the_arithmetic_as_it_is_passes(x, limbs, dim, keys):
    ratio, off = _case(x, dim, keys, 32512, limbs)
    assert ratio < 1.1 and off.max() <= 1.0


@pytest.mark.parametrize("x,steps,limbs", [("bf16", 508, 1), ("f16", 508, 2), ("f16", 4064, 2), ("f16", 32512, 1)])
@pytest.mark.parametrize("dim,keys", [(128, 1001), (64, 300)])
def test_coarser_queries_and_fewer_bits_fail(x, steps, limbs, dim, keys):
    assert _case(x, dim, keys, steps, limbs)[0] > 1.15


@pytest.mark.parametrize("x", ["bf16", "f16"])
def test_rounding_alone_counts_as_one(x):
    exact = np.random.default_rng(1).standard_normal(20000)
    assert U.error_ratio(torch.from_numpy(exact).to(U.TYPES[x]), exact, x) == 1.0
