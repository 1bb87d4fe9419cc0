"""Inputs and error bounds of the attention tests."""
import numpy as np
import torch

from oracle import attention as A

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def i32(a, dev=DEV):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def packed(rng, tokens, heads, dim, x, dev=DEV, pad=0, scale=1.0):
    """A [tokens, heads, dim] view into wider rows (`pad` elements more), and its values in fp32."""
    rows = torch.from_numpy(rng.standard_normal((tokens, heads * dim + pad)).astype(np.float32) * np.float32(scale)).to(TYPES[x]).to(dev)
    t = rows[:, pad // 2:pad // 2 + heads * dim].unflatten(1, (heads, dim))
    return t, t.float().cpu().numpy()


def page_tables(rng, counts, extra=2):
    """Page numbers for sequences of counts[b] pages, in no order, with a column to spare; unused entries are no pages."""
    total = int(sum(counts)) + extra
    order = rng.permutation(total)
    table, at = np.full((len(counts), max(list(counts) + [1]) + 1), -7, np.int32), 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def filled_cache(rng, pages, heads, page, dim):
    k, v = (rng.integers(-128, 128, s, dtype=np.int8) for s in ((pages, heads, page, dim), (pages, heads, dim, page)))
    ks, vs = (np.exp(rng.standard_normal((pages, heads)) * 0.7).astype(np.float32) / np.float32(60.0) for _ in range(2))
    return k, v, ks, vs


def to_dev(*arrays):
    return [torch.from_numpy(a.copy()).to(DEV) for a in arrays]


def attention_bound(exact, spread, scores, keys, dim, vmax, x, p_half):
    """How far a result may be from `exact`: spread = sum p |v|, scores = a bound of scale * sum |q| |k|.
    The output's rounding; a probability's rounding (p_half); the scores' 32-bit sums, which change a probability and the sum that
    divides it; the second product's 32-bit sum; and what fp16 probabilities lose below their smallest step (2^-25 each)."""
    fp32 = 2.0**-24
    in_p = p_half + 2 * (dim + 16) * fp32 * scores + (keys + 16) * fp32
    off = in_p * spread + (keys * 2.0**-25 * vmax if p_half == HALF_STEP["f16"] else 0.0)
    return HALF_STEP[x] * (np.abs(exact) + off) + off + 2.0**-24 * (x == "f16") + 1e-30


def check(got, exact, bound, where):
    """Within the bound; infinite where the result is surely beyond the type (fp16 rounds 65520 and more to infinity), either between."""
    limit = 65520.0 if got.dtype == torch.float16 else 3.4e38
    got = got.float().cpu().numpy().astype(np.float64)
    surely = np.abs(exact) - bound >= limit
    assert (got[surely] == np.sign(exact[surely]) * np.inf).all(), f"{where}: not infinite where the result is beyond the type"
    fine = np.abs(exact) + bound < limit
    assert np.isfinite(got[fine]).all() and not np.isnan(got).any(), f"{where}: not finite"
    off = np.where(fine, np.abs(np.where(fine, got, 0.0) - exact) / bound, 0.0)
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert off.max() <= 1.0, f"{where}: {off.max():.2f} times the bound at {worst}: {got[worst]} for {exact[worst]}"


def prompt_case(q, k, v, cu_q, cu_k, scale, causal, x):
    exact, spread = A.prompt(q, k, v, cu_q, cu_k, scale, causal), A.prompt(q, k, np.abs(v), cu_q, cu_k, scale, causal)
    g = q.shape[1] // k.shape[1]
    scores = scale * np.abs(q).max() * np.abs(k).sum(-1).max() if len(k) else 0.0
    assert g >= 1
    return exact, attention_bound(exact, spread, scores, int(np.diff(cu_k).max()), q.shape[2], np.abs(v).max() if len(v) else 0.0, x, HALF_STEP[x])


def cache_case(q, cu_q, lens, table, kc, vc, ks, vs, scale, x, max_q=None):
    """Beyond attention_bound's, for up to 32 columns (query tokens times heads of a group): queries are rounded to 1 / 32512 of their
    head's largest magnitude (half a step is 1 / 65024 of it), which moves a score by `scores` / 65024 at most and a probability and the
    sum that divides it by as much each; and a step's product is a sum of 64 p (1152 + v) less 1152 times the sum of p, 16 roundings (two
    products, four lanes' partial sums) of up to 1280 times the sum of p, in codes.
    From 33 columns on either kernel may serve, the one for few columns or the one for many, in which the scores' 32-bit sums are of codes plus 1152, up to 1280
    where `scores` counts 128: the larger of the two bounds."""
    exact, spread = A.cache(q, cu_q, lens, table, kc, vc, ks, vs, scale), A.cache(q, cu_q, lens, table, kc, np.abs(vc.astype(np.int16)), ks, vs, scale)
    scores = scale * np.abs(q).max() * 128 * q.shape[2] * ks.max()
    bound = attention_bound(exact, spread, scores, int(max(lens)), q.shape[2], 128 * vs.max(), x, HALF_STEP["f16"])
    few = 2 * scores / 65024 * spread + 16 * 2.0**-24 * 1280 * vs.max()
    if (max_q or int(np.diff(cu_q).max())) * (q.shape[1] // kc.shape[1]) > 32:
        return exact, bound + np.maximum(few, 2 * (q.shape[2] + 16) * 2.0**-24 * 9 * scores * spread)
    return exact, bound + few


# ------------------------------------------------------------------------------------------------
# bounds row by row and key by key
# ------------------------------------------------------------------------------------------------
def _softmax(s):
    w = np.exp(s - s.max(-1, keepdims=True))
    return w / w.sum(-1, keepdims=True)


def _off(p, y, v, delta, half_p, floor):
    """What weights that are off by `delta` (and by a rounding of half_p each that their sum may or may not see) and the products lose: p [n, keys],
    y [n, dim], v [keys, dim], delta [n, keys] or [n, 1]; floor [n, keys]: what a weight may lose whatever its size."""
    keys = p.shape[1]
    sums = (keys / 64 + 80) * 2.0**-24              # a step's 64 products and sums, then one sum a step
    return (p * (delta + half_p + sums) + floor) @ np.abs(v) + ((p * (delta + half_p + sums)).sum(1, keepdims=True)) * np.abs(y)


def cache_rows(q, cu_q, lens, table, kc, vc, ks, vs, scale, x, columns):
    """Exact results and how far they may be off, for sequences with queries.  columns "few": the kernel for up to 32 columns, whose queries are integers of
    1 / 32512 of their largest, whose second product has 1152 too much in it (16 roundings a step) and whose weights below 2^-24 of a step's largest vanish;
    "many": scores of codes plus 1152, logarithms of the values' scales, and weights times scales that vanish below 2^-36 of their largest."""
    page, pages, dim = kc.shape[2], kc.shape[0], q.shape[2]
    g = q.shape[1] // kc.shape[1]
    exact, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(lens)):
        n, keys = int(cu_q[b + 1] - cu_q[b]), int(lens[b])
        if not n or not keys:
            continue
        at = table[b, :-(-keys // page)]
        assert ((at >= 0) & (at < pages)).all()
        for h in range(kc.shape[1]):
            codes = kc[at, h].reshape(-1, dim)[:keys].astype(np.float64)
            k_scale, v_scale = (np.repeat(s[at, h].astype(np.float64), page)[:keys] for s in (ks, vs))
            v = vc[at, h].transpose(0, 2, 1).reshape(-1, dim)[:keys].astype(np.float64) * v_scale[:, None]
            hidden = np.arange(keys)[None, :] > keys - n + np.arange(n)[:, None]
            for head in range(h * g, (h + 1) * g):
                rows = slice(int(cu_q[b]), int(cu_q[b + 1]))
                qh = q[rows, head].astype(np.float64)
                s = np.where(hidden, -np.inf, scale * (qh @ codes.T) * k_scale)
                seen = ~hidden.all(1)
                p = np.zeros_like(s)
                p[seen] = _softmax(s[seen])
                y = p @ v
                aq, top = np.abs(qh), np.abs(qh).max(1, keepdims=True)
                size = scale * (aq @ (np.abs(codes) + (1152 if columns == "many" else 0)).T) * k_scale
                by_q = scale * top * (np.abs(codes).sum(1) * k_scale)
                fp32 = 2 * (dim + 16) * 2.0**-24 * np.where(hidden, 0.0, size).max(1, keepdims=True) + 2.0**-21
                if columns == "few":
                    delta = fp32 + by_q / 65024
                    floor = np.repeat(np.maximum.reduceat(p, np.arange(0, keys, 64), axis=1), 64, axis=1)[:, :keys] * 2.0**-24
                    more = 16 * 2.0**-24 * 1280 * (p @ v_scale)[:, None]
                    half_p = 2.0**-22 if x == "f16" else 2.0**-11
                else:
                    logs = np.abs(np.log2(v_scale[v_scale > 0])).max() if (v_scale > 0).any() else 0.0
                    delta = fp32 + (by_q * 2.0**-25 if x == "bf16" else 0.0) + 2.0**-22 * (logs + 16)
                    floor = (p * v_scale).max(1, keepdims=True) * 2.0**-36 / np.where(v_scale > 0, v_scale, np.inf)
                    more, half_p = 0.0, 2.0**-11
                off = _off(p, y, v, delta, half_p, np.where(hidden, 0.0, floor)) + more
                exact[rows, head], bound[rows, head] = y, HALF_STEP[x] * (np.abs(y) + off) + off + 2.0**-24 * (x == "f16") + 1e-36
    return exact, bound


def prompt_rows(q, k, v, cu_q, cu_k, scale, causal, x):
    """The same for the prompt's attention: weights rounded to the type; of fp16 those below 2^-36 of the largest vanish."""
    dim, g = q.shape[2], q.shape[1] // k.shape[1]
    exact, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(cu_q) - 1):
        rows, keys = slice(int(cu_q[b]), int(cu_q[b + 1])), slice(int(cu_k[b]), int(cu_k[b + 1]))
        n, m = rows.stop - rows.start, keys.stop - keys.start
        if not n or not m:
            continue
        hidden = causal & (np.arange(m)[None, :] > m - n + np.arange(n)[:, None])
        for head in range(q.shape[1]):
            qh, kh, vh = q[rows, head].astype(np.float64), k[keys, head // g].astype(np.float64), v[keys, head // g].astype(np.float64)
            s = np.where(hidden, -np.inf, scale * (qh @ kh.T))
            seen = ~hidden.all(1)
            p = np.zeros_like(s)
            p[seen] = _softmax(s[seen])
            y = p @ vh
            size = np.where(hidden, 0.0, scale * (np.abs(qh) @ np.abs(kh).T)).max(1, keepdims=True)
            floor = np.where(hidden, 0.0, p.max(1, keepdims=True) * 2.0**-36 * (x == "f16"))
            off = _off(p, y, vh, 2 * (dim + 16) * 2.0**-24 * size + 2.0**-21, HALF_STEP[x], floor)
            exact[rows, head], bound[rows, head] = y, HALF_STEP[x] * (np.abs(y) + off) + off + 2.0**-24 * (x == "f16") + 1e-36
    return exact, bound


def error_ratio(got, exact, x):
    """Root mean square of a result's errors, in units of what rounding the exact result to the type x alone gives."""
    exact = torch.as_tensor(exact, dtype=torch.float64)
    rounded = exact.to(TYPES[x]).double()
    return float(((torch.as_tensor(got).double().cpu() - exact).square().mean() / (rounded - exact).square().mean()).sqrt())


def ordinary_cache(rng, pages, heads, page, dim):
    """Codes and scales as keys and values of about normal distribution give them."""
    k, v = (np.clip(np.rint(rng.standard_normal(s) * 32.0), -127, 127).astype(np.int8) for s in ((pages, heads, page, dim), (pages, heads, dim, page)))
    ks, vs = (np.exp(rng.standard_normal((pages, heads)) * 0.2).astype(np.float32) / np.float32(32.0) for _ in range(2))
    return k, v, ks, vs
