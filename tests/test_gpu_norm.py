"""fq_rms_norm_quant against the oracle, bit for bit: residual sums, normalised rows, codes and scales."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import fq_oracle as O
from oracle import step as S
from tests import step_util as T

pytestmark = pytest.mark.gpu
EPS = 1e-5


def run(M, K, x="bf16", r=None, g="bf16", bits=8, dynamic=True, y=None, share=0.1, seed=0, extra=0, src=None, rep=None, scale=1.0, align=128, shape=None):
    rng = np.random.default_rng(seed)
    X = T.values(rng, (M, K), x, scale)
    R = T.values(rng, (M, K), r, 2.0 * scale) if r else None
    gamma = T.values(rng, K, g, 0.3) + np.float32(1.0)
    gamma = S.round_to(gamma, g)
    if shape is not None:
        X, R = shape(X, R)
    if src is None:
        src, rep, _, _ = T.plan(rng, K, share, align)
    Kpad = len(src)
    bound = None if dynamic else 2.5
    h, want_y, want_q, want_s = S.rms_norm_quant(X, gamma, EPS, src, rep, 4 if bits == 6 else bits, bound, R, r or "f32")
    dx = T.strided(X, x, extra)
    dr = T.strided(R, r, 2 * extra) if r else None
    d_out = T.strided(np.zeros((M, K)), r, extra) if r else None
    dy = T.strided(np.zeros((M, K)), y, 3 * extra) if y else None
    out, s_x = T.out_codes(bits, M, Kpad), torch.full((1,), -1.0, device=T.DEV)
    fq.fq_rms_norm_quant(dx, torch.from_numpy(gamma).to(T.TYPES[g]).to(T.DEV), EPS, R=dr, R_out=d_out, Y=dy, src_idx=torch.from_numpy(src).to(T.DEV),
                         rep=torch.from_numpy(rep).to(T.DEV), bits=bits, Xq_out=out, s_x_out=s_x, workspace=T.norm_workspace(M, K, Kpad) if dynamic else None,
                         absmax_in=None if dynamic else torch.tensor([bound], device=T.DEV))
    torch.cuda.synchronize()
    if r:
        assert T.same_values(d_out, h, r)
        base = d_out._base if d_out._base is not None else d_out
        assert torch.isnan(base[:, K:].float()).all()                     # what is between the rows is left alone
    if y:
        assert T.same_values(dy, want_y, y)
        base = dy._base if dy._base is not None else dy
        assert torch.isnan(base[:, K:].float()).all()
    assert s_x.cpu().numpy()[0] == want_s
    assert T.same_codes(out, want_q, bits)


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 16), (1, 4096), (2, 17), (3, 31), (5, 1000), (7, 1025), (16, 5120), (33, 2048), (65, 5003), (300, 129), (1500, 250),
                                 (2, 11008), (3, 16384)])
def test_sizes(M, K, dynamic):
    run(M, K, r="bf16", dynamic=dynamic, y="bf16", seed=M + K)


@pytest.mark.parametrize("K", [16385, 20480, 32768])
@pytest.mark.parametrize("dynamic", [True, False])
def test_wide_rows(K, dynamic):
    run(3, K, x="f16", r="f32", g="f32", dynamic=dynamic, y="f32", share=0.02, seed=K)


@pytest.mark.parametrize("x", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("r", [None, "f32", "f16", "bf16"])
@pytest.mark.parametrize("g,y,bits,dynamic", [("f32", "f16", 8, True), ("f16", "f32", 4, False), ("bf16", None, 6, True), ("bf16", "bf16", 4, True), ("f32", "bf16", 6, False)])
def test_types(x, r, g, y, bits, dynamic):
    run(19, 700, x, r, g, bits, dynamic, y, seed=3, extra=16)


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("share,align", [(0.0, 32), (0.0, 128), (1.0, 32), (0.5, 64)])
def test_plans(share, align, dynamic):
    """Nothing split, everything split (up to five copies a channel), padding of less than a group."""
    for K in (64, 333, 2000):
        run(9, K, dynamic=dynamic, share=share, align=align, bits=8)
        run(9, K, dynamic=dynamic, share=share, align=align, bits=4)


@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("bits", [8, 4])
def test_maps_that_no_plan_makes(bits, dynamic):
    """Channels out of order, twice with different copy counts, left out, numbers outside the row, counts of 0, 255 to 2^30."""
    rng = np.random.default_rng(5)
    K, Kpad = 500, 1504
    src = rng.integers(-3, K + 3, Kpad).astype(np.int32)
    rep = rng.choice([0, 1, 2, 3, 254, 255, 256, 257, 1000, 2**24 + 1, 2**30], Kpad).astype(np.int32)
    src[:64], rep[:64] = np.arange(64), rng.choice([1, 2, 2**24 + 1], 64)
    src[-1], src[-2] = 2**31 - 1, -2**31
    used = (src >= 0) & (src < K) & (rep > 0)
    run(11, K, bits=bits, dynamic=dynamic, src=np.where(used, src, -1).astype(np.int32), rep=np.where(used, rep, 0).astype(np.int32))
    few = np.full(32, 7, np.int32)
    run(4, K, bits=bits, dynamic=dynamic, src=few, rep=np.full(32, 3, np.int32))


def test_bad_map_entries_are_padding():
    rng = np.random.default_rng(6)
    K, Kpad, M = 100, 128, 3
    src, rep = np.arange(Kpad, dtype=np.int32), np.ones(Kpad, np.int32)
    src[:5], rep[5:8] = [-1, K, 2**31 - 1, -2**31, 10**6], [0, -1, -2**31]
    ok = (src >= 0) & (src < K) & (rep > 0)
    X = T.values(rng, (M, K), "f32")
    g = np.ones(K, np.float32)
    for dynamic in (True, False):
        _, _, q, s = S.rms_norm_quant(X, g, EPS, np.where(ok, src, -1).astype(np.int32), np.where(ok, rep, 0).astype(np.int32), 8, None if dynamic else 1.5)
        out, s_x = T.out_codes(8, M, Kpad), torch.zeros(1, device=T.DEV)
        fq.fq_rms_norm_quant(T.strided(X, "f32"), torch.from_numpy(g).to(T.DEV), EPS, src_idx=torch.from_numpy(src).to(T.DEV), rep=torch.from_numpy(rep).to(T.DEV),
                             Xq_out=out, s_x_out=s_x, workspace=T.norm_workspace(M, K, Kpad), absmax_in=None if dynamic else torch.tensor([1.5], device=T.DEV))
        assert s_x.item() == s and T.same_codes(out, q, 8)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("dynamic", [True, False])
def test_magnitudes(scale, dynamic):
    """Squares that fp32 cannot hold, rows far below eps."""
    run(6, 640, x="f32", r="f32", g="f32", y="f32", dynamic=dynamic, scale=scale)


@pytest.mark.parametrize("dynamic", [True, False])
def test_rows_of_zeros(dynamic):
    """All rows, and some of them: y = 0, and with nothing but zeros the scale is 1."""
    def zeros(X, R):
        return np.zeros_like(X), np.zeros_like(R)

    def some(X, R):
        X[::2] = 0
        return X, -X * (np.arange(len(X)) % 3 == 0)[:, None].astype(np.float32)

    run(8, 200, r="bf16", y="f16", dynamic=dynamic, shape=zeros)
    run(8, 200, r="bf16", y="f16", dynamic=dynamic, shape=some)


@pytest.mark.parametrize("bound", [0.0, -1.0, float("nan"), float("inf")])
def test_static_bounds_that_are_none(bound):
    """As in fq_flatten_quant_act: codes 0, scale 1."""
    x = torch.randn(4, 64, device=T.DEV)
    out, s_x = T.out_codes(8, 4, 64), torch.zeros(1, device=T.DEV)
    idx = torch.arange(64, dtype=torch.int32, device=T.DEV)
    fq.fq_rms_norm_quant(x, torch.ones(64, device=T.DEV), EPS, src_idx=idx, rep=torch.ones_like(idx), Xq_out=out, s_x_out=s_x, absmax_in=torch.tensor([bound], device=T.DEV))
    assert s_x.item() == 1.0 and not out.any()


@pytest.mark.parametrize("M", [1, 2, 40])
@pytest.mark.parametrize("dynamic", [True, False])
@pytest.mark.parametrize("r_out,y", [("R", None), ("X", None), ("R", "X"), ("X", "R"), (None, "X"), (None, "R")])
def test_in_place(r_out, y, dynamic, M):
    rng = np.random.default_rng(8)
    K = 1000
    X, R = T.values(rng, (M, K), "bf16"), T.values(rng, (M, K), "bf16")
    gamma = np.ones(K, np.float32)
    src, rep, _, Kpad = T.plan(rng, K, 0.2)
    h, yy, q, s = S.rms_norm_quant(X, gamma, EPS, src, rep, 8, None if dynamic else 2.0, R, "bf16")
    dev = dict(X=T.strided(X, "bf16", 8), R=T.strided(R, "bf16", 8))
    spare = dict(r=T.strided(np.zeros((M, K)), "bf16"), y=T.strided(np.zeros((M, K)), "bf16"))
    d_out, dy = dev.get(r_out, spare["r"]), dev.get(y, spare["y"])
    out, s_x = T.out_codes(8, M, Kpad), torch.zeros(1, device=T.DEV)
    fq.fq_rms_norm_quant(dev["X"], torch.from_numpy(gamma).to(T.DEV), EPS, R=dev["R"], R_out=d_out, Y=dy, src_idx=torch.from_numpy(src).to(T.DEV),
                         rep=torch.from_numpy(rep).to(T.DEV), Xq_out=out, s_x_out=s_x, workspace=T.norm_workspace(M, K, Kpad),
                         absmax_in=None if dynamic else torch.tensor([2.0], device=T.DEV))
    assert T.same_values(d_out, h, "bf16") and T.same_values(dy, yy, "bf16") and s_x.item() == s and T.same_codes(out, q, 8)


@pytest.mark.parametrize("r", [None, "f16"])
def test_rows_alone(r):
    """No codes wanted: no map, no workspace.  In place without a residual."""
    rng = np.random.default_rng(9)
    X = T.values(rng, (70, 333), "f16")
    R = T.values(rng, (70, 333), "f16") if r else None
    gamma = T.values(rng, 333, "f16")
    h, y = S.rms_norm(X, gamma, EPS, R, "f16")
    dx = T.strided(X, "f16")
    d_out = T.strided(np.zeros((70, 333)), "f16") if r else None
    dy = T.strided(np.zeros((70, 333)), "f16") if r else dx
    fq.fq_rms_norm_quant(dx, torch.from_numpy(gamma).half().to(T.DEV), EPS, R=T.strided(R, "f16") if r else None, R_out=d_out, Y=dy)
    assert T.same_values(dy, y, "f16") and (r is None or T.same_values(d_out, h, "f16"))


@pytest.mark.parametrize("dynamic", [True, False])
def test_the_same_as_norm_then_quantizer(dynamic):
    """The codes are those that fq_flatten_quant_act makes of the fp32 rows."""
    rng = np.random.default_rng(10)
    M, K = 777, 2048
    src, rep, _, Kpad = T.plan(rng, K, 0.15)
    src, rep = torch.from_numpy(src).to(T.DEV), torch.from_numpy(rep).to(T.DEV)
    x = torch.randn(M, K, device=T.DEV).to(torch.bfloat16)
    g = torch.rand(K, device=T.DEV)
    bound = None if dynamic else torch.tensor([1.25], device=T.DEV)
    y = torch.empty(M, K, device=T.DEV)
    out, s_x = T.out_codes(8, M, Kpad), torch.zeros(1, device=T.DEV)
    fq.fq_rms_norm_quant(x, g, EPS, Y=y, src_idx=src, rep=rep, Xq_out=out, s_x_out=s_x, workspace=T.norm_workspace(M, K, Kpad), absmax_in=bound)
    again, s_again = T.out_codes(8, M, Kpad), torch.zeros(1, device=T.DEV)
    fq.fq_flatten_quant_act(y, src, rep, 8, again, s_again, T.U.bytes_ws(fq.fq_act_workspace_bytes(K, Kpad)), absmax_in=bound)
    assert torch.equal(out, again) and torch.equal(s_x, s_again)


def test_a_row_that_ends_with_its_memory():
    """The last row's stride reaches behind the allocation: elements from K on are not read."""
    rng = np.random.default_rng(11)
    M, K, ld = 3, 1001, 1008
    flat = torch.full(((M - 1) * ld + K,), 1.0)
    X = T.values(rng, (M, K), "f32")
    for i in range(M):
        flat[i * ld:i * ld + K] = torch.from_numpy(X[i])
    x = flat.to(T.DEV).as_strided((M, K), (ld, 1))
    y = torch.empty(M, 1008, device=T.DEV)[:, :K]
    fq.fq_rms_norm_quant(x, torch.ones(K, device=T.DEV), EPS, Y=y)
    assert T.same_values(y, S.rms_norm(X, np.ones(K), EPS)[1], "f32")
