"""FqKvCache on several streams at once."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def test_attentions_on_two_streams_at_once():
    """Both split their keys and join the shares; the larger workspace comes while the smaller is in use."""
    rng = np.random.default_rng(0)
    cache = fq.FqKvCache(200, 2, 6000, 1, 64)
    k, v = (U.packed(rng, 6000 + 3000, 1, 64, "bf16")[0] for _ in range(2))
    cache.append(None, k, v, [6000, 3000])
    ones = [(U.packed(rng, sum(n), 4, 64, "bf16")[0], n) for n in ([1, 0], [2, 2], [0, 1], [3, 1])]
    want = [cache.attend(q, n, 0.125) for q, n in ones]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(10):
        for i, (q, n) in enumerate(ones):
            print(f"[two streams] turn {turn} call {i}", flush=True)
            with torch.cuda.stream(streams[(turn + i) % 2]):
                got.append((i, cache.attend(q, n, 0.125)))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i, y in got)
