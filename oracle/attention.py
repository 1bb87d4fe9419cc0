"""The attention calls in plain NumPy, written from include/fq.h's definitions: single steps in fp32 where the interface fixes
them (rotation, block scales, codes), float64 elsewhere.  Loops over sequences, heads and pages; nothing shared with the library."""
import numpy as np

F = np.float32


def rotate(x, cos, sin, interleaved):
    """x fp32 [heads, dim] of one token, cos / sin fp32 [rope_dim / 2] of its position."""
    y = x.astype(F).copy()
    h = len(cos)
    for i in range(h):
        u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        y[:, u] = x[:, u] * cos[i] - x[:, w] * sin[i]
        y[:, w] = x[:, w] * cos[i] + x[:, u] * sin[i]
    return y


def _store(x, slot, codes, scale, head):
    """x fp32 [n, dim] of one head at slots slot.. of a page: codes int8 [heads, page, dim], scale fp32 [heads], both of that page."""
    n = len(x)
    step = F(np.abs(x).max() / F(127.0))
    if step < F(2.0**-126):
        step = F(0.0)
    if slot > 0:
        old = scale[head]
        if step > old:
            codes[head, :slot] = np.rint(codes[head, :slot].astype(F) * F(old / step))
        step = max(old, step)
    scale[head] = step
    turn = F(F(1.0) / step) if step > 0 else F(0.0)
    codes[head, slot:slot + n] = np.clip(np.rint(x * turn), F(-127), F(127))


def append(q, k, v, cu, past, table, k_cache, v_cache, k_scale, v_scale, cos=None, sin=None, interleaved=False):
    """q, k, v fp32 [tokens, heads, dim]; caches and scales are updated in place (v_cache transposed within a page).
    Returns the rotated q and k (fp32; rows that have no place keep their input)."""
    page, pages = k_cache.shape[2], k_cache.shape[0]
    q, k = q.astype(F).copy(), k.astype(F).copy()
    reach = table.shape[1] * page if cos is None else min(table.shape[1] * page, len(cos))
    for b in range(len(past)):
        groups = {}
        for t in range(cu[b], cu[b + 1]):
            pos = past[b] + t - cu[b]
            if pos >= reach:
                continue
            if cos is not None:
                q[t], k[t] = rotate(q[t], cos[pos], sin[pos], interleaved), rotate(k[t], cos[pos], sin[pos], interleaved)
            groups.setdefault(pos // page, []).append((t, pos % page))
        for index, tokens in groups.items():
            p = table[b, index]
            if not 0 <= p < pages:
                continue
            rows, slot = [t for t, _ in tokens], tokens[0][1]
            for head in range(k.shape[1]):
                _store(k[rows, head], slot, k_cache[p], k_scale[p], head)
                turned = v_cache[p].transpose(0, 2, 1)
                _store(v[rows, head].astype(F), slot, turned, v_scale[p], head)
    return q, k


def softmax_rows(q, k, v, scale, causal):
    """One head in float64: q [n, dim], k and v [m, dim]; query i sees keys 0 .. m - n + i, or all."""
    n, m = len(q), len(k)
    y = np.zeros((n, v.shape[1]))
    for i in range(n):
        seen = m if not causal else max(0, m - n + i + 1)
        if seen:
            s = k[:seen] @ q[i] * scale
            w = np.exp(s - s.max())
            y[i] = (w / w.sum()) @ v[:seen]
    return y


def prompt(q, k, v, cu_q, cu_k, scale, causal=True):
    """float64 [tokens_q, heads_q, dim] (rows behind the last sequence: 0)."""
    y = np.zeros(q.shape)
    g = q.shape[1] // k.shape[1]
    for b in range(len(cu_q) - 1):
        for h in range(q.shape[1]):
            y[cu_q[b]:cu_q[b + 1], h] = softmax_rows(q[cu_q[b]:cu_q[b + 1], h].astype(np.float64), k[cu_k[b]:cu_k[b + 1], h // g].astype(np.float64),
                                                     v[cu_k[b]:cu_k[b + 1], h // g].astype(np.float64), scale, causal)
    return y


def gather(table_row, length, k_cache, v_cache, k_scale, v_scale):
    """float64 keys and values [n, heads, dim] of one sequence, and which positions they have (keys of pages that do not exist are left out)."""
    page, pages = k_cache.shape[2], k_cache.shape[0]
    k, v, at = [], [], []
    for t in range(length):
        p = table_row[t // page]
        if 0 <= p < pages:
            k.append(k_cache[p, :, t % page].astype(np.float64) * k_scale[p].astype(np.float64)[:, None])
            v.append(v_cache[p, :, :, t % page].astype(np.float64) * v_scale[p].astype(np.float64)[:, None])
            at.append(t)
    shape = (0, k_cache.shape[1], k_cache.shape[3])
    return (np.array(k) if k else np.zeros(shape)), (np.array(v) if v else np.zeros(shape)), np.array(at, np.int64)


def cache(q, cu_q, lens, table, k_cache, v_cache, k_scale, v_scale, scale):
    y = np.zeros(q.shape)
    g = q.shape[1] // k_cache.shape[1]
    for b in range(len(lens)):
        n = cu_q[b + 1] - cu_q[b]
        k, v, at = gather(table[b], lens[b], k_cache, v_cache, k_scale, v_scale)
        for i in range(n):
            seen = at < lens[b] - n + i + 1
            if seen.any():
                for h in range(q.shape[1]):
                    y[cu_q[b] + i, h] = softmax_rows(q[cu_q[b] + i, h].astype(np.float64)[None], k[seen, h // g], v[seen, h // g], scale, False)[0]
    return y
