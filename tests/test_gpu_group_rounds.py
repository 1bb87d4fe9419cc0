"""fq_linear_group_i4 where its kernels go round more than once: more outputs than 2^31, workgroups with several tiles, rings of stages whose places are used again.

Bounds are counted from the roundings, as in test_gpu_group.py; codes that enter as they are (fp16 activations without offsets) count as such."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import step as S
from tests import step_util as T

pytestmark = pytest.mark.gpu


def operands(rng, M, N, K, group, x, s, offsets):
    X = T.values(rng, (M, K), x)
    q = rng.integers(-8, 8, (N, K)).astype(np.int8)
    groups = -(-K // group)
    scale = S.round_to(np.exp(0.5 * rng.standard_normal((N, groups))).astype(np.float32) / np.float32(4.6 * np.sqrt(K)), s)
    return X, q, scale, S.round_to((scale * rng.standard_normal((N, groups))).astype(np.float32), s) if offsets else None


def device(a, t):
    return None if a is None else torch.from_numpy(a).to(T.TYPES[t]).to(T.DEV)


@pytest.mark.parametrize("group", [32, 128])
def test_more_outputs_than_2_31(group):
    """524291 rows of 4104 columns: launches hold them, as their tiles are of 64 x 128 outputs or more."""
    rng = np.random.default_rng(group)
    M, N, K = 524291, 4104, 160
    X, q, scale, _ = operands(rng, M, N, K, group, "f16", "f32", False)
    Y = torch.full((M, N), float("nan"), dtype=torch.float16, device=T.DEV)
    fq.fq_linear_group_i4(T.strided(X, "f16"), torch.from_numpy(S.pack(q)).to(T.DEV), device(scale, "f32"), group, Y)
    rows = np.unique(np.concatenate([np.arange(70), M - 1 - np.arange(70), rng.integers(0, M, 200)]))
    want, size = S.linear_group(X[rows], q, scale, None, group)
    got = Y[torch.from_numpy(rows).to(T.DEV)].double().cpu().numpy()
    steps = 4 * 33 + 3 * (K // 128 + 4) + 10
    assert np.all(np.abs(got - want) <= steps * 2.0**-24 * size + T.HALF["f16"] * (np.abs(want) + steps * 2.0**-24 * size) + 2.0**-25)
    assert not any(torch.isnan(part).any() for part in Y.split(1 << 16))
