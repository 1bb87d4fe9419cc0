"""The oracle of the calls around the products and the cache, pinned by hand cases and by the definitions written a second way."""
import numpy as np
import pytest

from oracle import fq_oracle as O
from oracle import step as S

F = np.float32


def test_norm_by_hand():
    """Row (3, 4): mean of squares 12.5; eps 12.5 makes the root 5, so t = 0.2."""
    h, y = S.rms_norm(np.array([[3, 4]], F), np.array([1, 10], F), 12.5)
    assert h.tolist() == [[3, 4]] and np.array_equal(y, np.array([[F(3) * F(0.2), F(4) * F(0.2) * F(10)]], F))
    h, y = S.rms_norm(np.array([[1, 256]], F), np.ones(2, F), 1e-5, r=np.array([[2, 1]], F), r_dtype="bf16")
    assert h.tolist() == [[3, 256]]                 # 257 is halfway between 256 and 258 in bf16: to even


def test_norm_codes_by_hand():
    """All elements alike: y = 1, every code 127; a channel split in two holds half of it."""
    x, g = np.full((2, 4), 7, F), np.array([1, 1, 2, 1], F)
    src, rep, kp, kpad = O.plan(np.array([1, 1, 2, 1], F), 1.0, 32)
    h, y, q, s = S.rms_norm_quant(x, g, 1e-30, src, rep, 8)
    assert np.array_equal(y, np.array([[1, 1, 2, 1]] * 2, F)) and s == F(1 / 127)
    assert q[:, :5].tolist() == [[127] * 5] * 2 and not q[:, 5:].any() and src[4] == 2


def test_norm_is_scale_free():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 50)).astype(F)
    y = S.rms_norm(x, np.ones(50, F), 1e-30)[1]
    assert np.array_equal(S.rms_norm(x * F(1024), np.ones(50, F), 1e-30)[1], y)
    assert np.allclose((y.astype(np.float64) ** 2).mean(1), 1, atol=1e-6)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_roundings(dtype):
    torch = pytest.importorskip("torch")
    x = (np.random.default_rng(1).standard_normal(10000) * 10.0 ** np.arange(-5, 5).repeat(1000)).astype(F)
    want = torch.from_numpy(x).to({"f16": torch.float16, "bf16": torch.bfloat16}[dtype]).float().numpy()
    assert np.array_equal(S.round_to(x, dtype), want)


def test_weights_by_hand():
    w = np.zeros((2, 32), F)
    w[0, :4] = [7, -7, 3.5, -3.4]                   # s = 1; 3.5 rounds to even
    w[1] = np.arange(32) % 16                       # offsets: lo 0, hi 15, s = 1, b = 8
    q, s, b = S.group_weights(w, 32, "f32", False)
    assert s[0, 0] == 1 and q[0, :5].tolist() == [7, -7, 4, -3, 0] and b is None
    q, s, b = S.group_weights(w, 32, "f32", True)
    assert s[1, 0] == 1 and b[1, 0] == 8 and q[1].tolist() == [i % 16 - 8 for i in range(32)]
    assert np.array_equal(S.weights_of(q, s, b, 32)[1], w[1])


def test_weights_of_nothing_and_of_one_value():
    w = np.stack([np.zeros(64, F), np.full(64, 2.5, F)])
    for offsets in (False, True):
        q, s, b = S.group_weights(w, 64, "f16", offsets)
        assert s[0, 0] == 0 and not q[0].any()
    assert s[1, 0] == 0 and b[1, 0] == 2.5 and not q[1].any()


@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_weights_are_within_half_a_step(group, offsets):
    """At most half a step of the scale off, but for what the scale's and the offset's own rounding adds; a short last group counts by itself."""
    rng = np.random.default_rng(2)
    w = rng.standard_normal((7, 224)).astype(F)
    q, s, b = S.group_weights(w, group, "bf16", offsets)
    step = np.repeat(s, group, 1)[:, :224]
    # the end codes lie where the rounded scale puts them: 8 steps times 2^-8, and the offset's 2^-8 of it
    slack = 0.5 * step + (8 * step * 2.0**-7 + (np.repeat(np.abs(b), group, 1)[:, :224] * 2.0**-7 if offsets else 0))
    assert np.all(np.abs(S.weights_of(q, s, b, group) - w) <= slack)
    assert s.shape == (7, -(-224 // group)) and q.min() >= -8 and q.max() <= 7
    last = S.group_weights(w[:, (s.shape[1] - 1) * group:], group, "bf16", offsets)
    assert np.array_equal(last[1][:, 0], s[:, -1])


def test_packing():
    q = np.array([[-8, 7, 0, -1]], np.int8)
    assert S.pack(q).tolist() == [[0x78, 0xF0]] and np.array_equal(O.unpack_i4(S.pack(q)), q)


def test_product_two_ways():
    rng = np.random.default_rng(3)
    x, q = rng.standard_normal((3, 96)).astype(F), rng.integers(-8, 8, (5, 96)).astype(np.int8)
    s, b, bias = rng.random((5, 2)).astype(F), rng.standard_normal((5, 2)).astype(F), rng.standard_normal(5).astype(F)
    y, size = S.linear_group(x, q, s, b, 64, bias)
    for i in range(3):
        for n in range(5):
            want = float(bias[n])
            for k in range(96):
                want += float(x[i, k]) * (float(s[n, k // 64]) * int(q[n, k]) + float(b[n, k // 64]))
            assert abs(y[i, n] - want) < 1e-9 and size[i, n] > abs(want)


def test_copies():
    a = [np.arange(5), np.arange(10).reshape(5, 2)]
    S.copy_pages(a, [0, 4, 7, -1], [2, 1, 3, 0])
    assert a[0].tolist() == [0, 4, 0, 3, 4] and a[1].tolist() == [[0, 1], [8, 9], [0, 1], [6, 7], [8, 9]]
