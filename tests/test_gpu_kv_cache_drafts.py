"""Drafted tokens in an FqKvCache: appended together, checked together, the rejected ones dropped."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from tests import attn_util as U
from tests.test_gpu_attention_use import Reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("past,kept", [([62, 10], [1, 5]), ([60, 126], [0, 2]), ([64, 127], [4, 1])])
def test_rejected_drafts_are_dropped_by_their_lengths(past, kept):
    """Five drafts a sequence, of which `kept` stay (across and at the ends of pages); the next tokens take the places of the others."""
    rng = np.random.default_rng(past[0] + kept[0])
    heads, dim, scale = (4, 2), 64, 0.125
    cache = fq.FqKvCache(10, 2, 300, heads[1], dim)
    for t in (cache.k_cache, cache.v_cache):
        t.fill_(77)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(0.5)
    ref = Reference(cache)

    def step(new, x=1.0):
        before = list(cache.lengths)
        q, qn = U.packed(rng, sum(new), heads[0], dim, "bf16")
        (k, kn), (v, vn) = (U.packed(rng, sum(new), heads[1], dim, "bf16", scale=x) for _ in range(2))
        cache.append(None, k, v, new)
        torch.cuda.synchronize()
        ref.append(kn, kn, vn, new, before, None, None, False)
        ref.same()
        y = cache.attend(q, new, scale)
        torch.cuda.synchronize()
        cu, table = U.offsets(new), cache.page_table.cpu().numpy()
        exact, bound = U.cache_rows(qn, cu, cache.lengths, table, *ref.arrays, scale, "bf16", "few" if max(new) * 2 <= 32 else "many")
        U.check(y, exact, bound, f"step {new}")
    step(past)
    step([5, 5], 3.0)
    cache.lengths = [p + k for p, k in zip(past, kept)]
    step([1, 1])
    step([5, 0])
