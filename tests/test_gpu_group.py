"""fq_group_weights_i4 (bit for bit) and fq_linear_group_i4 (within bounds counted from its roundings) against the oracle."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import step as S
from tests import step_util as T

pytestmark = pytest.mark.gpu


def make(W, w_dtype, group, s_dtype, offsets, extra=0):
    N, K = W.shape
    groups = -(-K // group)
    dw = T.strided(W, w_dtype, extra)
    wq = torch.full((N, K // 2), 0x5A, dtype=torch.uint8, device=T.DEV)
    s, b = (torch.full((N, groups), float("nan"), dtype=T.TYPES[s_dtype], device=T.DEV) for _ in range(2))
    fq.fq_group_weights_i4(dw, group, wq, s, B_out=b if offsets else None)
    return wq, s, b if offsets else None


def check_weights(W, w_dtype, group, s_dtype, offsets, extra=0):
    wq, s, b = make(W, w_dtype, group, s_dtype, offsets, extra)
    q, ws, wb = S.group_weights(W, group, s_dtype, offsets)
    assert np.array_equal(s.float().cpu().numpy(), ws)
    assert b is None or np.array_equal(b.float().cpu().numpy(), wb)
    assert np.array_equal(wq.cpu().numpy(), S.pack(q))


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 32), (3, 64), (17, 96), (5, 160), (64, 128), (33, 4000), (130, 1376), (2, 22016)])
def test_weights_sizes(N, K, group, offsets):
    rng = np.random.default_rng(N + K + group)
    check_weights(T.values(rng, (N, K), "bf16"), "bf16", group, "bf16", offsets, extra=8)


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("s_dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("w_dtype", ["f32", "f16", "bf16"])
def test_weights_types(w_dtype, s_dtype, offsets):
    rng = np.random.default_rng(7)
    check_weights(T.values(rng, (21, 352), w_dtype, 0.02), w_dtype, 64, s_dtype, offsets)


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("s_dtype", ["f32", "f16", "bf16"])
def test_weights_far_from_one(s_dtype, offsets):
    """Rows of zeros, of one value, of one sign, scales that vanish or overflow in 16 bits, subnormal weights."""
    rng = np.random.default_rng(8)
    W = rng.standard_normal((16, 256)).astype(np.float32)
    W[0], W[1], W[2] = 0, 3.25, -0.1
    W[3], W[4] = np.abs(W[3]), -np.abs(W[4])
    W[5] *= np.float32(1e-8)
    W[6] *= np.float32(1e-30)
    W[7] *= np.float32(1e-38)
    W[8] *= np.float32(1e-40)
    W[9] *= np.float32(1e6)
    W[10] *= np.float32(1e30)
    W[11] = np.clip(W[11], -1, 1) * np.float32(1.6e38)
    W[12, ::2], W[13, 5] = 0, 1000
    W[14] = 7 * np.sign(W[14])
    W[15] = np.arange(256) % 16 - 8
    check_weights(W, "f32", 64, s_dtype, offsets)


def product(M, N, K, group, x="bf16", s="bf16", offsets=False, bias=False, y="bf16", seed=0, extra=0, mean=0.0, ldy=0, scale=1.0):
    rng = np.random.default_rng(seed)
    X = S.round_to(T.values(rng, (M, K), x, scale) + np.float32(mean), x)
    groups = -(-K // group)
    q = rng.integers(-8, 8, (N, K)).astype(np.int8)
    sc = S.round_to(np.exp(0.5 * rng.standard_normal((N, groups))).astype(np.float32) / np.float32(4.6 * np.sqrt(K)), s)
    of = S.round_to((sc * rng.standard_normal((N, groups))).astype(np.float32), s) if offsets else None
    bi = rng.standard_normal(N).astype(np.float32) if bias else None
    want, size = S.linear_group(X, q, sc, of, group, bi)
    dev = lambda a, t: None if a is None else torch.from_numpy(a).to(T.TYPES[t]).to(T.DEV)  # noqa: E731
    out = torch.full((M, N + ldy), float("nan"), dtype=T.TYPES[y], device=T.DEV)
    Y = out[:, :N]
    fq.fq_linear_group_i4(T.strided(X, x, extra), torch.from_numpy(S.pack(q)).to(T.DEV), dev(sc, s), group, Y, B=dev(of, s), bias=dev(bi, "f32"))
    got = Y.double().cpu().numpy()
    assert torch.isnan(out[:, N:].float()).all()
    # roundings of fp32 on the way of one product into the sum: at most 33 in each of a group's four matrix products, two for the scale, those of
    # the steps that a wave adds up, eight joins and the bias; then half a step of the output's type
    steps = 4 * 33 + 3 * (K // 128 + 4) + 10
    bound = steps * 2.0**-24 * size + T.HALF[y] * (np.abs(want) + steps * 2.0**-24 * size) + (2.0**-25 if y == "f16" else 0.0)
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)
    # and on the whole: a rounding's error is at most half a step, uniform at worst, so its root mean square is under 0.58 of it; fp32 sums of this
    # length add under 2^-20 of the summands' root mean square, which is at most size / sqrt(K)
    rms = np.sqrt(np.mean((got - want) ** 2))
    assert rms <= np.sqrt(np.mean((0.58 * T.HALF[y] * want) ** 2) + np.mean((2.0**-20 * size / np.sqrt(K)) ** 2)) * 1.1 + (2.0**-25 if y == "f16" else 0.0)
    return Y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (1, 16, 64), (1, 4096, 4096), (2, 17, 96), (1, 100, 11008), (5, 33, 160), (16, 64, 128), (17, 80, 352), (4, 250, 2080),
                                   (31, 31, 1056), (33, 16, 4000), (64, 130, 512), (65, 48, 640), (200, 300, 288), (130, 129, 2048), (3, 40, 22016)])
def test_product_sizes(M, N, K, group):
    product(M, N, K, group, seed=M + N + K)


@pytest.mark.parametrize("y", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("s", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("x", ["f16", "bf16"])
def test_product_types(x, offsets, s, y):
    for M in (1, 20, 70, 140):
        product(M, 70, 736, 64, x, s, offsets, bias=M != 20, y=y, seed=M, extra=24, ldy=3)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("x", ["f16", "bf16"])
@pytest.mark.parametrize("offsets", [False, True])
def test_product_groups(x, group, offsets):
    for M in (1, 18, 100, 260):
        product(M, 144, 992, group, x, "f32", offsets, y="f32", seed=M)


@pytest.mark.parametrize("x", ["f16", "bf16"])
def test_activations_of_one_sign(x):
    """What bf16 codes carry too much, 24 times the sum of the activations, is then many times the result."""
    for M in (1, 40, 150):
        product(M, 64, 2048, 128, x, "f32", y="f32", mean=4.0)


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("x,scale", [("f16", 2.0**-18), ("f16", 2.0**12), ("bf16", 2.0**-100), ("bf16", 2.0**100)])
def test_magnitudes(x, scale, offsets):
    """Among them activations that are subnormal in fp16: most of the first case's."""
    for M in (1, 12, 40, 150):
        product(M, 48, 1024, 64, x, "f32", offsets, y="f32", scale=scale, seed=M)


@pytest.mark.parametrize("x,dt", [("f16", torch.float16), ("bf16", torch.bfloat16)])
def test_few_and_many_rows_agree(x, dt):
    """The same rows through the kernels for one token, a few and many: the sums differ by their order only."""
    X = torch.randn(300, 1184, device=T.DEV).to(dt)
    wq = torch.randint(0, 256, (530, 592), dtype=torch.uint8, device=T.DEV)
    s, b = torch.rand(530, 19, device=T.DEV), torch.randn(530, 19, device=T.DEV)
    out = []
    for rows in (1, 7, 16, 20, 45, 60, 300):
        y = torch.empty(rows, 530, device=T.DEV)
        fq.fq_linear_group_i4(X[:rows], wq, s, 64, y, B=b)
        out.append(y)
    size = X[:1].float().abs() @ (8 * s + b.abs()).repeat_interleave(64, 1)[:, :1184].t() * 4
    for y in out[:-1]:
        assert ((y[0] - out[-1][0]).abs() <= 300 * 2.0**-24 * size[0]).all()
        assert torch.allclose(y, out[-1][:len(y)], rtol=1e-3, atol=1e-2 * float(size.mean()))


def test_each_code_at_each_place():
    """One activation a row, so that a result is one weight: any code or column in the wrong place shows, exactly."""
    K, N = 256, 16
    q = ((np.arange(K)[None, :] * 7 + np.arange(N)[:, None] * 3) % 16 - 8).astype(np.int8)
    for x, dt in (("f16", torch.float16), ("bf16", torch.bfloat16)):
        for group in (32, 64, 128):
            s = (2.0 ** (np.arange(-(-K // group))[None, :] + np.arange(N)[:, None] % 3)).astype(np.float32)
            Y = torch.empty(K, N, device=T.DEV)
            fq.fq_linear_group_i4(torch.eye(K, device=T.DEV, dtype=dt), torch.from_numpy(S.pack(q)).to(T.DEV), torch.from_numpy(s).to(T.DEV), group, Y)
            assert np.array_equal(Y.cpu().numpy().T, S.weights_of(q, s, None, group))
            one = torch.empty(1, N, device=T.DEV)
            for k in (0, 1, 37, 130, 255):
                fq.fq_linear_group_i4(torch.eye(K, device=T.DEV, dtype=dt)[k:k + 1], torch.from_numpy(S.pack(q)).to(T.DEV), torch.from_numpy(s).to(T.DEV), group, one)
                assert np.array_equal(one.cpu().numpy()[0], S.weights_of(q, s, None, group)[:, k])


@pytest.mark.parametrize("M", [1, 3, 40, 300])
def test_results_do_not_change(M):
    a, b = product(M, 200, 1312, 64, y="f32", offsets=True), product(M, 200, 1312, 64, y="f32", offsets=True)
    assert torch.equal(a, b)


def test_a_row_does_not_go_by_its_neighbours():
    """Infinities and NaN in one row of activations, or in one row's scales, stay there."""
    X = torch.randn(70, 320, device=T.DEV).to(torch.bfloat16)
    wq = torch.randint(0, 256, (50, 160), dtype=torch.uint8, device=T.DEV)
    s = torch.rand(50, 5, device=T.DEV)
    want = torch.empty(70, 50, device=T.DEV)
    fq.fq_linear_group_i4(X, wq, s, 64, want)
    X[7, 5], X[69, 319], s[11, 2] = float("inf"), float("nan"), float("inf")
    got = torch.empty_like(want)
    fq.fq_linear_group_i4(X, wq, s, 64, got)
    rows, cols = [i for i in range(70) if i not in (7, 69)], [j for j in range(50) if j != 11]
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])
    assert not torch.isfinite(got[7]).any() and not torch.isfinite(got[69]).any() and not torch.isfinite(got[:, 11]).any()


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(15, 50, 9248), (16, 4130, 5152), (20, 4130, 800), (33, 2070, 1440), (20, 8200, 416), (40, 8200, 544), (20, 16500, 288), (70, 10000, 672),
                                   (70, 16500, 416), (130, 9000, 1184), (70, 33000, 160)])
def test_product_tiles(M, N, K, group, offsets):
    """Numbers of tiles that take each of the kernels' tiles on a device of 256 compute units, both sides of every rule."""
    product(M, N, K, group, offsets=offsets, seed=M + N + K)
