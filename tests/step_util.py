"""Helpers for the tests of the calls around the products and the cache."""
import numpy as np
import torch

import paper_2402_17985_amd as fq
from oracle import fq_oracle as O
from oracle import step as S
from tests import gpu_util as U

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}      # half a step of a rounding, relative to the value


def strided(x, dtype, extra=0, fill=float("nan")):
    """fp32 array -> device matrix of that type whose rows lie a multiple of 16 bytes (and `extra` elements) apart; what is between is `fill`."""
    M, K = x.shape
    t = torch.full((M, -(-K // 8) * 8 + extra), fill, dtype=torch.float32)
    t[:, :K] = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return t.to(TYPES[dtype]).to(DEV)[:, :K]


def values(rng, shape, dtype, scale=1.0):
    return S.round_to((scale * rng.standard_normal(shape)).astype(np.float32), dtype)


def plan(rng, K, share, align=128, most=5):
    chmax = np.ones(K, np.float32)
    many = int(share * K)
    if many:
        chmax[rng.choice(K, many, replace=False)] = rng.integers(2, most + 1, many)
    return O.plan(chmax, 1.0, align)


def codes_of(out, bits, M, Kpad):
    """Codes as the oracle has them from the device's storage."""
    b = out.cpu().numpy()
    if bits == 8:
        return b.view(np.int8).reshape(M, Kpad)
    assert bits == 4
    return O.unpack_i4(b.reshape(M, Kpad // 2))


def out_codes(bits, M, Kpad):
    if bits == 6:
        return torch.full((Kpad // 128, M, 96), 0xA5, dtype=torch.uint8, device=DEV)
    return torch.full((M, Kpad if bits == 8 else Kpad // 2), 0x55, dtype=torch.int8 if bits == 8 else torch.uint8, device=DEV)


def same_codes(out, q, bits):
    if bits == 6:
        return np.array_equal(out.cpu().numpy().reshape(-1), O.pack_e3m2_blocked(q).reshape(-1))
    return np.array_equal(codes_of(out, bits, *q.shape), q)


def same_values(t, want, dtype):
    """The device matrix holds exactly these values (fp32, rounded to the type)."""
    return np.array_equal(t.float().cpu().numpy(), S.round_to(want, dtype))


def norm_workspace(M, K, Kpad):
    return U.bytes_ws(fq.fq_rms_norm_workspace_bytes(M, K, Kpad))
