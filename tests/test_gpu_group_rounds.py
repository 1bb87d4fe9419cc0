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


def check(M, N, K, group, x, s, y, offsets, bias, ldy):
    rng = np.random.default_rng(M + N + K + group)
    X, q, scale, offset = operands(rng, M, N, K, group, x, s, offsets)
    add = rng.standard_normal(N).astype(np.float32) if bias else None
    out = torch.full((M, N + ldy), float("nan"), dtype=T.TYPES[y], device=T.DEV)
    fq.fq_linear_group_i4(T.strided(X, x, 8), torch.from_numpy(S.pack(q)).to(T.DEV), device(scale, s), group, out[:, :N], B=device(offset, s), bias=device(add, "f32"))
    want, size = S.linear_group(X, q, scale, offset, group, add, surplus=24 if offsets or x == "bf16" else 0)
    got = out[:, :N].double().cpu().numpy()
    assert torch.isnan(out[:, N:].float()).all()
    # as in test_gpu_group.py: at most 33 roundings in each of a group's four matrix products, three a step for scale and offset, sixteen joins and the bias
    steps = 4 * 33 + 3 * (K // 128 + 4) + 18
    bound = steps * 2.0**-24 * size + T.HALF[y] * (np.abs(want) + steps * 2.0**-24 * size) + (2.0**-25 if y == "f16" else 0.0)
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)
    # On the whole: the sums over groups, at most 32 in a row here, are rounded twice for each group, by 0.58 of half a step, at a magnitude that is at most the
    # result's; that is 1.44 size / sqrt(K) where codes are uniform and activations normal, so 2^-24 * 0.58 * sqrt(64) * 1.44 = 2^-21.3 of size / sqrt(K).
    rms = np.sqrt(np.mean((got - want) ** 2))
    assert rms <= np.sqrt(np.mean((0.58 * T.HALF[y] * want) ** 2) + np.mean((2.0**-20 * size / np.sqrt(K)) ** 2)) * 1.1 + (2.0**-25 if y == "f16" else 0.0)


FORMS = [("f16", "f32", "f32", False, False, 0), ("f16", "f16", "f16", True, True, 3), ("bf16", "f32", "f32", True, False, 5), ("bf16", "bf16", "bf16", False, True, 1)]


@pytest.mark.parametrize("x,s,y,offsets,bias,ldy", FORMS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 8200, 160), (1, 17000, 1056), (7, 8250, 1056), (2, 8250, 4256), (16, 9000, 2080), (13, 4130, 3616), (16, 4130, 4480)])
def test_workgroups_of_several_tiles(M, N, K, group, x, s, y, offsets, bias, ldy):
    """Up to 16 rows: more tiles of 16 columns than two workgroups for each of 256 compute units take (8 waves: activations of up to 64 KiB), or than one (16 waves).  Among them
    stretches of two, four and six steps, waves without any, one to four rounds, a last tile of 2 to 10 columns."""
    check(M, N, K, group, x, s, y, offsets, bias, ldy)


@pytest.mark.parametrize("x,s,y,offsets,bias,ldy", FORMS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(16, 50, 4640), (16, 4130, 4640), (20, 250, 4256), (20, 4130, 3232), (20, 8200, 1184), (40, 8200, 1184), (20, 16500, 1184), (300, 6700, 1184), (600, 6700, 992)])
def test_rings_that_go_round(M, N, K, group, x, s, y, offsets, bias, ldy):
    """Every tile that a device of 256 compute units takes, 16 x 16 to 64 x 256, with more stages along the reduction than the ring in LDS has places, the last of them a part of one."""
    check(M, N, K, group, x, s, y, offsets, bias, ldy)


@pytest.mark.parametrize("x", ["f16", "bf16"])
def test_all_rows_of_few_and_many_agree(x):
    """The same rows through the kernels for one token, a few and many, every one of them: results differ by the roundings of two sums."""
    rng = np.random.default_rng(1)
    X, q, scale, offset = operands(rng, 300, 530, 1184, 64, x, "f32", True)
    size = torch.from_numpy(S.linear_group(X, q, scale, offset, 64)[1]).to(T.DEV)
    X, wq, s, b = T.strided(X, x), torch.from_numpy(S.pack(q)).to(T.DEV), device(scale, "f32"), device(offset, "f32")
    out = {}
    for rows in (300, 1, 7, 16, 20, 45, 60):
        out[rows] = torch.full((rows, 530), float("nan"), device=T.DEV)
        fq.fq_linear_group_i4(X[:rows], wq, s, 64, out[rows], B=b)
        steps = 2 * (4 * 33 + 3 * (1184 // 128 + 4) + 18)
        assert ((out[rows].double() - out[300][:rows].double()).abs() <= steps * 2.0**-24 * size[:rows]).all(), rows
