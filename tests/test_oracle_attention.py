"""What the plain forms of the attention calls (oracle/attention.py) are held by: hand cases, and PyTorch in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import attention as A


def test_rotation_hand_cases():
    x = np.array([[1, 2, 3, 4, 5, 6]], np.float32)
    c, s = np.array([0, 1], np.float32), np.array([1, 0], np.float32)      # a quarter turn, none
    assert A.rotate(x, c, s, False).tolist() == [[-3, 2, 1, 4, 5, 6]]
    assert A.rotate(x, c, s, True).tolist() == [[-2, 1, 3, 4, 5, 6]]


def test_rotation_keeps_products_of_equal_distance():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 64)).astype(np.float32)
    at = np.arange(60)[:, None] * 10000.0 ** (-np.arange(0, 64, 2) / 64)
    c, s = np.cos(at).astype(np.float32), np.sin(at).astype(np.float32)
    for inter in (False, True):
        dots = [float(A.rotate(q, c[p + 7], s[p + 7], inter)[0].astype(np.float64) @ A.rotate(k, c[p], s[p], inter)[0]) for p in (0, 11, 50)]
        assert np.ptp(dots) < 1e-5


def _empty(pages=2, heads=1, page=4, dim=2):
    return (np.zeros((pages, heads, page, dim), np.int8), np.zeros((pages, heads, dim, page), np.int8), np.full((pages, heads), np.nan, np.float32),
            np.full((pages, heads), np.nan, np.float32))


def test_append_hand_case():
    kc, vc, ks, vs = _empty()
    kv = np.array([[[127.0, -1.0]], [[63.5, 0.0]], [[0.4, 0.5]], [[1.5, 2.5]], [[254.0, 3.0]]], np.float32)
    table = np.array([[1, 0]], np.int32)
    A.append(kv, kv, 2 * kv, [0, 3], [0], table, kc, vc, ks, vs)
    assert ks[1, 0] == 1.0 and vs[1, 0] == 2.0 and np.isnan(ks[0, 0])
    assert kc[1, 0].tolist() == [[127, -1], [64, 0], [0, 0], [0, 0]]              # 63.5, 0.5 to even
    assert vc[1, 0].tolist() == [[127, 64, 0, 0], [-1, 0, 0, 0]]
    # two more: the first page's scale stays, the second page starts anew
    A.append(kv[3:], kv[3:], kv[3:], [0, 2], [3], table, kc, vc, ks, vs)
    assert ks[1, 0] == 1.0 and ks[0, 0] == 2.0 and kc[1, 0, 3].tolist() == [2, 2] and kc[0, 0, 0].tolist() == [127, 2]


def test_append_growing_scale_hand_case():
    kc, vc, ks, vs = _empty(1)
    first, second = np.array([[[127.0, 3.0]]], np.float32), np.array([[[254.0, -5.0]]], np.float32)
    table = np.zeros((1, 1), np.int32)
    A.append(first, first, first, [0, 1], [0], table, kc, vc, ks, vs)
    A.append(second, second, second, [0, 1], [1], table, kc, vc, ks, vs)
    assert ks[0, 0] == 2.0 and kc[0, 0, :2].tolist() == [[64, 2], [127, -2]]      # 127 / 2, 3 / 2, -5 / 2: to even
    assert (vc[0, 0].T == kc[0, 0]).all()


def test_append_bounds_every_element_by_half_a_step_and_zeros_stay():
    rng = np.random.default_rng(1)
    kc, vc, ks, vs = _empty(3, 2, 64, 64)
    x = rng.standard_normal((100, 2, 64)).astype(np.float32)
    A.append(x, x, 0 * x, [0, 100], [0], np.array([[2, 0, 1]], np.int32), kc, vc, ks, vs)
    for page, rows in ((2, x[:64]), (0, x[64:])):
        back = kc[page, :, :len(rows)].astype(np.float64) * ks[page][:, None, None]
        assert np.abs(back - rows.transpose(1, 0, 2)).max() <= 0.5000001 * ks[page].max()
        assert np.abs(kc[page]).max() == 127 and vs[page].tolist() == [0, 0] and not vc[page].any()
    assert np.isnan(ks[1]).all()


@pytest.mark.parametrize("causal", [True, False])
def test_attention_against_torch(causal):
    rng = np.random.default_rng(2)
    cu_q, cu_k = [0, 3, 3, 10], [0, 5, 9, 16]
    q, k, v = rng.standard_normal((10, 4, 8)), rng.standard_normal((16, 2, 8)), rng.standard_normal((16, 2, 8))
    y = A.prompt(q, k, v, cu_q, cu_k, 0.3, causal)
    for b in range(3):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        for h in range(4):
            s = torch.from_numpy(q[cu_q[b]:cu_q[b + 1], h]) @ torch.from_numpy(k[cu_k[b]:cu_k[b + 1], h // 2]).T * 0.3
            if causal:
                s = s.masked_fill(torch.ones(n, m, dtype=torch.bool).triu(m - n + 1), -np.inf)
            want = torch.softmax(s, -1) @ torch.from_numpy(v[cu_k[b]:cu_k[b + 1], h // 2])
            np.testing.assert_allclose(y[cu_q[b]:cu_q[b + 1], h], want.numpy(), rtol=1e-12, atol=1e-13)


def test_rows_without_keys_are_zero():
    y = A.prompt(np.ones((3, 1, 4)), np.ones((1, 1, 4)), np.ones((1, 1, 4)), [0, 3], [0, 1], 1.0, True)
    assert y[:, 0, 0].tolist() == [0, 0, 1]
    assert not A.prompt(np.ones((3, 1, 4)), np.ones((0, 1, 4)), np.ones((0, 1, 4)), [0, 3], [0, 0], 1.0, False).any()


def test_cache_attention_is_prompt_attention_of_what_the_codes_stand_for():
    rng = np.random.default_rng(3)
    page, heads, dim = 4, 2, 8
    kc, vc = rng.integers(-128, 128, (5, heads, page, dim), dtype=np.int8), rng.integers(-128, 128, (5, heads, dim, page), dtype=np.int8)
    ks, vs = rng.uniform(0.01, 0.02, (2, 5, heads)).astype(np.float32)
    table, lens, cu = np.array([[3, 1, 9], [4, 0, -1]], np.int32), [7, 6], [0, 2, 5]
    q = rng.standard_normal((5, 4, dim))
    y = A.cache(q, cu, lens, table, kc, vc, ks, vs, 0.2)
    for b in range(2):
        k = np.concatenate([kc[p] * ks[p].astype(np.float64)[:, None, None] for p in table[b, :2]], 1)[:, :lens[b]].transpose(1, 0, 2)
        v = np.concatenate([vc[p].transpose(0, 2, 1) * vs[p].astype(np.float64)[:, None, None] for p in table[b, :2]], 1)[:, :lens[b]].transpose(1, 0, 2)
        want = A.prompt(q[cu[b]:cu[b + 1]], k, v, [0, cu[b + 1] - cu[b]], [0, lens[b]], 0.2, True)
        np.testing.assert_allclose(y[cu[b]:cu[b + 1]], want, rtol=1e-12)
    # a page that does not exist is left out: the second sequence's last two tokens
    table[1, 1] = 7
    y2 = A.cache(q, cu, lens, table, kc, vc, ks, vs, 0.2)
    k = (kc[4] * ks[4].astype(np.float64)[:, None, None]).transpose(1, 0, 2)
    v = (vc[4].transpose(0, 2, 1) * vs[4].astype(np.float64)[:, None, None]).transpose(1, 0, 2)
    want = A.prompt(q[2:5], np.concatenate([k, np.zeros((2, heads, dim))]), np.concatenate([v, np.zeros((2, heads, dim))]), [0, 3], [0, 6], 0.2, True)
    np.testing.assert_allclose(y2[2], want[0], rtol=1e-12)          # sees tokens 0 .. 3
    assert not np.allclose(y2[3], want[1])                          # would see tokens 4 as a zero key; left out it is not seen at all
