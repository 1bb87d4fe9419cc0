"""The calls around the products and the cache in plain NumPy, written from include/fq.h's definitions: single steps in fp32 (or the
stored type) where the interface fixes them, float64 elsewhere.  Nothing shared with the library."""
import numpy as np

from . import fq_oracle as O

F = np.float32


def round_to(x, dtype):
    """fp32 -> "f32" / "f16" / "bf16" (half to even) and back to fp32."""
    x = np.asarray(x, F)
    if dtype == "f32":
        return x
    if dtype == "f16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).astype(F)
    u = np.ascontiguousarray(x).view(np.uint32).astype(np.uint64)
    out = (((u + ((u >> 16) & 1) + 0x7FFF) >> 16) << 16).astype(np.uint32).view(F)
    return np.where(np.isnan(x), x, out)


def rms_norm(x, gamma, eps, r=None, r_dtype="f32"):
    """x, r fp32 [M, K], gamma fp32 [K].  Returns (h, y), both fp32: the residual sum as stored, and the normalised rows before rounding."""
    h = np.asarray(x, F) if r is None else round_to(np.asarray(x, F) + np.asarray(r, F), r_dtype)
    rms = np.sqrt((h.astype(np.float64) ** 2).sum(1) / h.shape[1] + np.float64(F(eps)))
    t = (1.0 / rms).astype(F)
    return h, (h * t[:, None]) * np.asarray(gamma, F)


def rms_norm_quant(x, gamma, eps, src, rep, bits, bound=None, r=None, r_dtype="f32"):
    """Returns (h, y, codes int8 [M, Kpad], s_x)."""
    h, y = rms_norm(x, gamma, eps, r, r_dtype)
    a = O.act_absmax_dynamic(y, src, rep) if bound is None else F(bound)
    q, s_x = O.flatten_quant_act(y, src, rep, bits, a)
    return h, y, q, s_x


LARGEST = {"f32": np.finfo(F).max, "f16": F(65504.0), "bf16": round_to(F(3.3895314e38), "bf16")}


def group_weights(w, group, s_dtype, offsets):
    """w fp32 [N, K].  Returns (codes int8 [N, K], scales fp32 [N, groups], offsets or None)."""
    N, K = w.shape
    groups = -(-K // group)
    q, s, b = np.zeros((N, K), np.int8), np.zeros((N, groups), F), np.zeros((N, groups), F)
    top = LARGEST[s_dtype]
    with np.errstate(over="ignore"):
        for g in range(groups):
            part = w[:, g * group:(g + 1) * group].astype(F)
            lo, hi = part.min(1), part.max(1)
            step = (hi - lo) / F(15.0) if offsets else np.abs(part).max(1) / F(7.0)
            step = np.minimum(round_to(step, s_dtype), top)
            step = np.where(step < F(2.0**-126), F(0.0), step).astype(F)
            if offsets:
                b[:, g] = np.clip(round_to(lo + F(8.0) * step, s_dtype), -top, top)
            turn = np.where(step > 0, F(1.0) / np.where(step > 0, step, F(1.0)), F(0.0)).astype(F)
            q[:, g * group:(g + 1) * group] = np.rint(np.clip((part - b[:, g, None]) * turn[:, None], F(-8.0), F(7.0)))
            s[:, g] = step
    return q, s, b if offsets else None


def pack(q):
    """int8 codes [N, K] to nibbles, even column in the low one."""
    u = q.astype(np.uint8) & 15
    return u[:, 0::2] | (u[:, 1::2] << 4)


def weights_of(q, s, b, group):
    """float64 [N, K]: s q + b."""
    K = q.shape[1]
    wide = lambda a: np.repeat(a.astype(np.float64), group, axis=1)[:, :K]  # noqa: E731
    return wide(s) * q + (0.0 if b is None else wide(b))


def linear_group(x, q, s, b, group, bias=None, surplus=24):
    """float64: x times the weights' transpose, plus bias; and the sum of the absolute values of what is added up, codes as q + surplus."""
    y = x.astype(np.float64) @ weights_of(q, s, b, group).T
    size = np.abs(x.astype(np.float64)) @ weights_of(np.abs(q.astype(np.int16)) + 2 * surplus, np.abs(s), None if b is None else np.abs(b), group).T
    return (y, size) if bias is None else (y + bias.astype(np.float64), size + np.abs(bias))


def copy_pages(arrays, src, dst):
    """Pages of every array (first axis) copied in place; numbers outside the pool copy nothing."""
    pages = len(arrays[0])
    for a, b in zip(src, dst):
        if 0 <= a < pages and 0 <= b < pages:
            for x in arrays:
                x[b] = x[a]
