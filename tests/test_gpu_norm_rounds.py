"""fq_rms_norm_quant with more rows than workgroups: the next row's prefetch, what lies in LDS from one row to the next, maxima kept over rows."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import step as S
from tests import step_util as T
from tests.test_gpu_norm import EPS, run

pytestmark = pytest.mark.gpu

# On 256 compute units there are at most 4096 workgroups of 64 threads (264 channels), 2048 of 128 (2048), 768 of 320 (5003), 256 of 576, 704 and 1024 (8200, 11008, 20000):
# each of these has two rows for a workgroup at least, and three for some
SIZES = [(9001, 264), (4500, 2048), (1700, 5003), (600, 8200), (530, 11008), (520, 20000)]


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("x,r,g,y,bits", [("bf16", "bf16", "bf16", None, 8), ("bf16", "f32", "f32", "bf16", 4), ("f16", None, "f16", None, 6), ("f32", "f32", "f32", "f32", 8)])
@pytest.mark.parametrize("M,K", SIZES)
def test_more_rows_than_workgroups(M, K, x, r, g, y, bits, dynamic):
    run(M, K, x, r, g, bits, dynamic, y, share=0.05, seed=M)


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", [(9001, 264), (1700, 5003), (520, 20000)])
def test_maps_out_of_order(M, K, bits, dynamic):
    """No slot at its channel's place; copies with counts of their own, more of them than a thread keeps in registers."""
    rng = np.random.default_rng(M)
    Kpad = -(-K * 5 // 4 // 128) * 128
    src = np.concatenate([rng.permutation(K), rng.integers(0, K, Kpad - K)]).astype(np.int32)
    rep = rng.choice([1, 1, 1, 2, 3, 300], Kpad).astype(np.int32)
    src[7], rep[7] = -1, 0
    run(M, K, "bf16", "bf16", bits=bits, dynamic=dynamic, src=src, rep=rep, seed=M)


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("r_out,y", [("R", "X"), ("X", "R"), (None, "X")])
@pytest.mark.parametrize("M,K", [(9001, 264), (1700, 5003), (520, 20000)])
def test_in_place(M, K, r_out, y, dynamic):
    """A row is fetched while the one before it is written over."""
    rng = np.random.default_rng(K)
    X, R = T.values(rng, (M, K), "bf16"), T.values(rng, (M, K), "bf16")
    gamma = T.values(rng, K, "f32")
    src, rep, _, Kpad = T.plan(rng, K, 0.05)
    h, yy, q, s = S.rms_norm_quant(X, gamma, EPS, src, rep, 8, None if dynamic else 2.0, R, "bf16")
    dev = dict(X=T.strided(X, "bf16", 8), R=T.strided(R, "bf16", 8))
    d_out = dev.get(r_out, T.strided(np.zeros((M, K)), "bf16"))
    out, s_x = T.out_codes(8, M, Kpad), torch.zeros(1, device=T.DEV)
    fq.fq_rms_norm_quant(dev["X"], torch.from_numpy(gamma).to(T.DEV), EPS, R=dev["R"], R_out=d_out, Y=dev[y], src_idx=torch.from_numpy(src).to(T.DEV),
                         rep=torch.from_numpy(rep).to(T.DEV), Xq_out=out, s_x_out=s_x, workspace=T.norm_workspace(M, K, Kpad),
                         absmax_in=None if dynamic else torch.tensor([2.0], device=T.DEV))
    assert T.same_values(d_out, h, "bf16") and T.same_values(dev[y], yy, "bf16") and s_x.item() == s and T.same_codes(out, q, 8)


@pytest.mark.parametrize("K", [16392, 20480, 32768])
@pytest.mark.parametrize("x,r,y,bits", [("bf16", "bf16", None, 8), ("f32", None, "f16", 4), ("f16", "f32", "f16", 6)])
def test_one_wide_row(K, x, r, y, bits):
    """One workgroup finds the bound of a row that registers do not hold, and quantizes it."""
    run(1, K, x, r, "f32", bits, True, y, share=0.02, seed=K)


def test_the_bound_lies_in_a_late_row():
    """A workgroup's second or third row holds the largest element, or one that is large only in a copied channel."""
    for at in (4100, 8999):
        def spike(X, R, at=at):
            X[at, 100] = 60.0
            return X, R
        run(9001, 264, "bf16", None, dynamic=True, share=0.1, seed=at, shape=spike)
