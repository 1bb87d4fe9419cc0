"""Performance cases of the attention operators beside the quantized linear layer: what a serving program calls between
the QKV projection and the output projection.

Kinds of case (key "kind"):
  append   fq_kv_append: rotate the new queries and keys by their positions, store keys and values in the paged 8-bit
           cache (one scale for each page and head), at the end of what each sequence holds there already.
  cache    fq_attn_cache: the last "queries" tokens of every sequence attend to all that the cache holds of it, causally.
  prompt   fq_attn_prompt: attention over packed sequences of different lengths, straight from the projections' output;
           "fresh" less than 1 makes only that share of a sequence's last tokens queries.

"length" is the longest sequence; the others are drawn by "mix" from "shortest" times it upwards (an append's are the
tokens that the cache holds before the call).  "heads" query heads share "kv" key heads.  Queries, keys and values come out
of one projection: they are views into its rows.

The cache's codes are whole numbers that the interface defines to the bit; they come back as such, beside their scales.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # one new token of one conversation: nothing but latency
        dict(name="append_one", kind="append", batch=1, new=1, heads=32, kv=32, dim=128, length=1000, shortest=1.0, mix=1, page=64,
             rope=128, interleaved=False, x="bf16"),
        # a decoding step of 64 conversations, grouped heads
        dict(name="append_batch64", kind="append", batch=64, new=1, heads=64, kv=8, dim=128, length=4000, shortest=0.02, mix=2, page=64,
             rope=128, interleaved=False, x="bf16"),
        # four prompts of 2048 tokens of a 40-head model, part of each head rotated, pairs side by side
        dict(name="append_prompts", kind="append", batch=4, new=2048, heads=40, kv=40, dim=128, length=0, shortest=1.0, mix=3, page=64,
             rope=64, interleaved=True, x="f16"),
        # the next token of one conversation of an ordinary length, as many key heads as query heads
        dict(name="decode_one", kind="cache", batch=1, queries=1, heads=32, kv=32, dim=128, length=1001, shortest=1.0, mix=4, page=64, x="bf16"),
        # a decoding step of 64 conversations of very different lengths, grouped heads
        dict(name="decode_batch64", kind="cache", batch=64, queries=1, heads=64, kv=8, dim=128, length=8192, shortest=0.02, mix=5, page=64,
             x="bf16"),
        # two long documents, grouped heads: the cache is split among the compute units
        dict(name="decode_long", kind="cache", batch=2, queries=1, heads=64, kv=8, dim=128, length=131072, shortest=1.0, mix=6, page=128,
             x="f16"),
        # five proposed tokens a sequence are checked at once; heads of 80
        dict(name="verify_five", kind="cache", batch=16, queries=5, heads=32, kv=32, dim=80, length=2048, shortest=0.1, mix=7, page=64, x="f16"),
        # a further piece of 512 tokens of a prompt that is in the cache already
        dict(name="chunk512", kind="cache", batch=1, queries=512, heads=64, kv=8, dim=128, length=8192, shortest=1.0, mix=8, page=64, x="bf16"),
        # eight prompts of 256 tokens, 32 heads
        dict(name="prompt_8x256", kind="prompt", batch=8, heads=32, kv=32, dim=128, length=256, shortest=1.0, mix=9, fresh=1.0, causal=True,
             x="bf16"),
        # a batch of uneven prompts of a 40-head model
        dict(name="prompt_ragged", kind="prompt", batch=8, heads=40, kv=40, dim=128, length=2048, shortest=0.01, mix=10, fresh=1.0,
             causal=True, x="f16"),
        # one long prompt, grouped heads
        dict(name="prompt_8192", kind="prompt", batch=1, heads=64, kv=8, dim=128, length=8192, shortest=1.0, mix=11, fresh=1.0, causal=True,
             x="bf16"),
        # an encoder's batch: every token sees every other, heads of 64
        dict(name="encode_16x512", kind="prompt", batch=16, heads=16, kv=16, dim=64, length=512, shortest=0.3, mix=12, fresh=1.0,
             causal=False, x="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "cache", "cache", "prompt", "prompt"])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 32, 40])
    groups = [g for g in (1, 2, 4, 5, 7, 8, 16) if g * kv <= 64]
    case = dict(kind=kind, heads=kv * rng.choice(groups), kv=kv, dim=rng.choice([64, 80, 96, 128, 128, 128]), mix=rng.randrange(1 << 20),
                shortest=rng.choice([1.0, 0.5, 0.1, 0.01]))
    if kind == "append":
        rope = rng.choice([0, case["dim"], case["dim"], case["dim"] // 2])
        case |= dict(page=rng.choice([64, 64, 128]), rope=rope, interleaved=rng.random() < 0.5, x=rng.choice(["bf16", "bf16", "f16", "f32"]))
        while True:
            case |= dict(batch=_log_int(rng, 1, 256), new=rng.choice([1, 1, _log_int(rng, 1, 4096)]), length=rng.choice([0, _log_int(rng, 1, 8192)]))
            if case["batch"] * case["new"] * (case["heads"] + 2 * kv) <= 8192 * 120 and _cells(case) <= 1 << 27:
                return case
    case["x"] = rng.choice(["bf16", "bf16", "f16"])
    if kind == "cache":
        case["page"] = rng.choice([64, 64, 128])
        while True:
            case |= dict(batch=_log_int(rng, 1, 128), length=_log_int(rng, 1, 131072), queries=rng.choice([1, 1, 1, 2, 8, _log_int(rng, 1, 512)]))
            case["queries"] = min(case["queries"], case["length"])
            pairs = case["batch"] * case["length"] * case["queries"] * case["heads"] * case["dim"]
            if _cells(case) <= 2 * 131072 * 8 * 128 and pairs <= 512 * 8192 * 64 * 128:
                return case
    case |= dict(fresh=rng.choice([1.0, 1.0, 1.0, 0.3]), causal=rng.random() < 0.8)
    while True:
        case |= dict(batch=_log_int(rng, 1, 32), length=_log_int(rng, 1, 8192))
        if case["batch"] * case["length"] ** 2 * case["heads"] * case["dim"] * (1 if case["causal"] else 2) <= 64 * 8192**2 * 128:
            return case


def _cells(case):
    return case["batch"] * (case["length"] + case.get("new", 0)) * case["kv"] * case["dim"]


def _lengths(case):
    """Tokens of each sequence: the longest is the case's, the others lie between its shortest and that."""
    r = random.Random(case["mix"])
    full = [case["length"]] + [int(case["length"] * r.uniform(case["shortest"], 1.0)) for _ in range(case["batch"] - 1)]
    r.shuffle(full)
    return [max(n, case.get("queries", 0), 1 if case["kind"] == "prompt" else 0) for n in full]


def _queries(case):
    """Query tokens of each sequence."""
    if case["kind"] == "cache":
        return [case["queries"]] * case["batch"]
    return [max(1, int(n * case["fresh"])) for n in _lengths(case)]


def _new(case):
    """New tokens of each sequence of an append; prompts differ as the lengths do."""
    r = random.Random(case["mix"] + 1)
    return [max(1, int(case["new"] * r.uniform(case["shortest"], 1.0))) if i else case["new"] for i in range(case["batch"])]


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _projected(g, tokens, case):
    """Rows of a fused QKV projection, and the views of queries, keys and values in it."""
    Hq, Hkv, D = case["heads"], case["kv"], case["dim"]
    rows = torch.randn((tokens, (Hq + 2 * Hkv) * D), dtype=torch.float32, device=DEV, generator=g).to(DTYPES[case["x"]])
    q, k, v = rows.split([Hq * D, Hkv * D, Hkv * D], dim=1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


def _offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device=DEV)


def _pages(g, lengths, case):
    """A pool of pages with what the sequences hold, and their page tables: any page can come anywhere."""
    P, Hkv, D = case["page"], case["kv"], case["dim"]
    counts = [-(-n // P) for n in lengths]
    width, used = max(1, max(counts)), sum(counts)
    pool = used + 3
    order = torch.randperm(pool, device=DEV, generator=g).to(torch.int32)
    table = torch.zeros((len(lengths), width), dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV)[None, :] < torch.tensor(counts, device=DEV)[:, None]
    table[held] = order[:used]
    s = dict(page_table=table)
    for name, shape in (("k", (pool, Hkv, P, D)), ("v", (pool, Hkv, D, P))):
        codes = torch.empty(shape, dtype=torch.int8, device=DEV)
        for part in codes.split(max(1, (1 << 27) // (Hkv * P * D))):
            part.copy_(torch.randn(part.shape, dtype=torch.float32, device=DEV, generator=g).mul_(32.0).round_().clamp_(-127, 127))
        s[name + "_cache"] = codes
        s[name + "_scale"] = torch.exp(0.2 * torch.randn((pool, Hkv), dtype=torch.float32, device=DEV, generator=g)) / 32.0
    return s


def _angles(rows, dim):
    """Cosines and sines of position times frequency, in 64 bits, rounded once."""
    at = torch.arange(rows, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEV) / dim)
    return at.cos().float(), at.sin().float()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case, scale=case["dim"] ** -0.5)
    if case["kind"] == "append":
        past, new = _lengths(case), _new(case)
        s |= _pages(g, [p + n for p, n in zip(past, new)], case)
        s["q"], s["k"], s["v"] = _projected(g, sum(new), case)
        s |= dict(cu_new=_offsets(new), past=torch.tensor(past, dtype=torch.int32, device=DEV), max_new=max(new))
        s["cos"], s["sin"] = _angles(max(p + n for p, n in zip(past, new)), case["rope"]) if case["rope"] else (None, None)
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
        s["k_out"] = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEV)
    elif case["kind"] == "cache":
        lengths, queries = _lengths(case), _queries(case)
        s |= _pages(g, lengths, case)
        s["q"] = _projected(g, sum(queries), case)[0]
        s |= dict(cu_q=_offsets(queries), lens=torch.tensor(lengths, dtype=torch.int32, device=DEV), max_q=max(queries), max_len=max(lengths))
        s["y"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
    else:
        lengths, queries = _lengths(case), _queries(case)
        q, k, v = _projected(g, sum(lengths), case)
        if case["fresh"] < 1.0:  # only the queries of the last tokens of each sequence
            ends = np.cumsum(lengths)
            q = q[torch.from_numpy(np.concatenate([np.arange(e - n, e) for e, n in zip(ends, queries)])).to(DEV)]
        s |= dict(q=q, k=k, v=v, cu_q=_offsets(queries), cu_k=_offsets(lengths), max_q=max(queries), max_k=max(lengths))
        s["y"] = torch.empty(q.shape, dtype=q.dtype, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _rotated(x, cos, sin, interleaved):
    """Pairs of the first 2 * cos.shape[-1] elements of each head turned by their angles; products and sums rounded one by one."""
    x = x.float()
    if cos is None:
        return x
    h = cos.shape[-1]
    a, b, rest = (x[..., 0 : 2 * h : 2], x[..., 1 : 2 * h : 2], x[..., 2 * h :]) if interleaved else (x[..., :h], x[..., h : 2 * h], x[..., 2 * h :])
    c, s = cos[:, None, :], sin[:, None, :]
    u, w = a * c - b * s, b * c + a * s
    return torch.cat([torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1), rest], -1)


def _store(x, codes, scales, seq, pos, past, table, page):
    """x [tokens, heads, dim] (32 bits) into codes [pages, heads, page, dim]: each page's scale grows to hold its new tokens."""
    pages, heads = scales.shape
    at = table[seq, pos // page].long()
    top = torch.zeros((pages, heads), dtype=torch.float32, device=DEV).index_reduce_(0, at, x.abs().amax(-1), "amax")
    wanted = top / torch.full_like(top, 127.0)
    wanted = torch.where(wanted < 2.0**-126, 0.0, wanted)
    # one place more than there are pages, for what has no page
    touched, begun = (torch.zeros(pages + 1, dtype=torch.bool, device=DEV) for _ in range(2))
    touched[at] = True
    begun[torch.where(pos % page == 0, at, pages)] = True
    touched, begun = touched[:pages, None], begun[:pages, None]
    old = torch.where(begun, 0.0, scales)
    scale = torch.where(touched, torch.maximum(old, wanted), scales)
    # codes that the pages held before, in the new scale
    held = torch.zeros(pages + 1, dtype=torch.int64, device=DEV)
    rows = torch.arange(past.numel(), device=DEV)
    held[torch.where(past % page != 0, table[rows, torch.clamp(past // page, max=table.shape[1] - 1)].long(), pages)] = past % page
    grown = ((scale > old) & touched & ~begun)[:, :, None, None] & (torch.arange(page, device=DEV)[:, None] < held[:pages, None, None, None])
    again = torch.round(codes * (old / torch.where(scale > 0, scale, 1.0))[:, :, None, None]).to(torch.int8)
    codes = torch.where(grown, again, codes)
    turn = torch.where(scale > 0, torch.ones_like(scale) / scale, 0.0)
    codes[at, :, pos % page] = torch.round(x * turn[at][:, :, None]).clamp(-127, 127).to(torch.int8)
    return codes, scale


def _append(s):
    case = s["case"]
    new = (s["cu_new"][1:] - s["cu_new"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), new, output_size=s["k"].shape[0])
    pos = s["past"].long()[seq] + torch.arange(seq.numel(), device=DEV) - s["cu_new"].long()[seq]
    cos, sin = (None, None) if s["cos"] is None else (s["cos"][pos], s["sin"][pos])
    q, k = (_rotated(s[n], cos, sin, case["interleaved"]) for n in ("q", "k"))
    s["q_out"].copy_(q)
    s["k_out"].copy_(k)
    args = seq, pos, s["past"].long(), s["page_table"], case["page"]
    codes, scale = _store(k, s["k_cache"], s["k_scale"], *args)
    s["k_cache"].copy_(codes)
    s["k_scale"].copy_(scale)
    codes, scale = _store(s["v"].float(), s["v_cache"].transpose(2, 3), s["v_scale"], *args)
    s["v_cache"].copy_(codes.transpose(2, 3))
    s["v_scale"].copy_(scale)


def _attention(q, k, v, hidden, scale):
    """q [batch, kv, rows, dim], k and v [batch, kv, keys, dim] in 32 bits; hidden [batch, 1, rows, keys]."""
    w = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(hidden, -math.inf)
    top = w.amax(-1, keepdim=True)
    w = w.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(-1, keepdim=True)
    return torch.matmul(w, v) / torch.where(total > 0, total, 1.0)


def _padded(x, cu, most):
    """[tokens, heads, dim] packed -> [batch, heads, most, dim], and the lengths."""
    n = (cu[1:] - cu[:-1]).long()
    at = cu[:-1].long()[:, None] + torch.minimum(torch.arange(most, device=DEV)[None, :], n[:, None] - 1)
    return x[at].float().transpose(1, 2), n


def _attend(s, k, v, keys):
    """k, v [batch, kv, most, dim], of which each sequence has `keys`."""
    case = s["case"]
    G, D = case["heads"] // case["kv"], case["dim"]
    q, nq = _padded(s["q"], s["cu_q"], s["max_q"])
    B, _, most_q, _ = q.shape
    row, col = torch.arange(most_q, device=DEV), torch.arange(k.shape[2], device=DEV)
    last = keys[:, None] - nq[:, None] + row[None, :] if case.get("causal", True) else (keys[:, None] - 1).expand(-1, most_q)
    hidden = col[None, None, :] > last[:, :, None]
    q = q.reshape(B, case["kv"], G * most_q, D)
    y = _attention(q, k, v, hidden[:, None].repeat(1, 1, G, 1), s["scale"])
    y = y.reshape(B, case["heads"], most_q, D).transpose(1, 2)
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), nq, output_size=s["y"].shape[0])
    s["y"].copy_(y.flatten(0, 1)[seq * most_q + torch.arange(seq.numel(), device=DEV) - s["cu_q"].long()[seq]])


def _cache(s):
    B, W = s["page_table"].shape
    kv, D = s["case"]["kv"], s["case"]["dim"]
    at = s["page_table"].long()
    k = s["k_cache"][at] * s["k_scale"][at][..., None, None]
    v = (s["v_cache"][at] * s["v_scale"][at][..., None, None]).transpose(3, 4)
    k, v = (x.transpose(1, 2).reshape(B, kv, -1, D) for x in (k, v))
    _attend(s, k, v, s["lens"].long())


def _prompt(s):
    k, n = _padded(s["k"], s["cu_k"], s["max_k"])
    _attend(s, k, _padded(s["v"], s["cu_k"], s["max_k"])[0], n)


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        import paper_2402_17985_amd as fq

        if kind == "append":
            fq.fq_kv_append(s["q"], s["k"], s["v"], s["cu_new"], s["past"], s["max_new"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                            s["page_table"], rope_cos=s["cos"], rope_sin=s["sin"], interleaved=s["case"]["interleaved"], Q_out=s["q_out"], K_out=s["k_out"])
        elif kind == "cache":
            if "workspace" not in s:
                c = s["case"]
                size = fq.fq_attn_cache_workspace_bytes(c["batch"], s["q"].shape[0], s["max_q"], s["max_len"], c["heads"], c["kv"], c["dim"])
                s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
            fq.fq_attn_cache(s["q"], s["cu_q"], s["lens"], s["max_q"], s["max_len"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                             s["page_table"], s["scale"], s["y"], s["workspace"])
        else:
            fq.fq_attn_prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["max_q"], s["scale"], s["y"], causal=s["case"]["causal"])
    else:
        _append(s) if kind == "append" else _cache(s) if kind == "cache" else _prompt(s)
    if kind == "append":
        return {n: s[n] for n in ("q_out", "k_out", "k_cache", "v_cache", "k_scale", "v_scale")}
    return s["y"]


def _pairs(case):
    """(query, key) pairs that see each other, over the sequences, for one head."""
    total = 0
    for nk, nq in zip(_lengths(case), _queries(case)):
        total += nq * nk if not case.get("causal", True) else sum(range(nk - nq + 1, nk + 1))
    return total


def work(case):
    Hq, Hkv, D, e = case["heads"], case["kv"], case["dim"], SIZE[case["x"]]
    if case["kind"] == "append":
        new = _new(case)
        t = sum(new)
        return {"bytes": t * D * ((Hq + 2 * Hkv) * e + (Hq + Hkv) * e + 2 * Hkv) + 4 * t * case["rope"], "flops": 3 * t * case["rope"] * (Hq + Hkv) + 4 * t * Hkv * D}
    q = sum(_queries(case))
    flops = 4 * _pairs(case) * Hq * D
    if case["kind"] == "cache":
        pages = sum(-(-n // case["page"]) for n in _lengths(case))
        return {"bytes": 2 * sum(_lengths(case)) * Hkv * D + 12 * pages * Hkv + 2 * q * Hq * D * e, "flops": flops}
    return {"bytes": 2 * q * Hq * D * e + 2 * sum(_lengths(case)) * Hkv * D * e, "flops": flops}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits: sequence by sequence, head by head
# ------------------------------------------------------------------------------------------------
def _exact_rows(q, k, v, scale, causal):
    """One head: q [nq, dim], k, v [nk, dim] in 64 bits."""
    nq, nk = q.shape[0], k.shape[0]
    out = []
    for lo in range(0, nq, 2048):
        hi = min(nq, lo + 2048)
        w = q[lo:hi] @ k.t() * scale
        if causal:
            w += torch.triu(torch.full((hi - lo, nk), -math.inf, dtype=torch.float64, device=DEV), diagonal=nk - nq + lo + 1)
        out.append(torch.softmax(w, dim=1) @ v)
    return torch.cat(out)


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, D = case["heads"], case["kv"], case["dim"]
    if case["kind"] == "append":
        got = {}
        for name in ("q", "k"):
            parts = []
            for b, (past, lo) in enumerate(zip(s["past"].tolist(), s["cu_new"].tolist()[:-1])):
                n = s["cu_new"].tolist()[b + 1] - lo
                z = s[name][lo : lo + n].double()
                if case["rope"]:
                    h = case["rope"] // 2
                    i = torch.arange(h, device=DEV)
                    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + h)
                    turn = torch.complex(s["cos"][past : past + n].double(), s["sin"][past : past + n].double())[:, None]
                    moved = torch.complex(z[..., first], z[..., second]) * turn
                    z[..., first], z[..., second] = moved.real, moved.imag
                parts.append(z)
            got[name + "_out"] = torch.cat(parts)
        values = {"k": got["k_out"], "v": s["v"].double()}
        for name, x in values.items():
            scale = s[name + "_scale"].double()
            for b, (past, lo) in enumerate(zip(s["past"].tolist(), s["cu_new"].tolist()[:-1])):
                n = s["cu_new"].tolist()[b + 1] - lo
                for j in range(past // case["page"], (past + n - 1) // case["page"] + 1):
                    begin = max(past, j * case["page"]) - past
                    peak = x[lo + begin : lo + min(n, (j + 1) * case["page"] - past)].abs().amax((0, 2)) / 127.0
                    page = s["page_table"][b, j].long()
                    scale[page] = peak if past <= j * case["page"] else torch.maximum(scale[page], peak)
            got[name + "_scale"] = scale
        return got | {"k_cache": None, "v_cache": None}
    if 4 * _pairs(case) * Hq * D > 4e12 or case["batch"] * Hq > 4096:
        return None
    cq = s["cu_q"].tolist()
    y = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, nk in enumerate(_lengths(case)):
        if case["kind"] == "cache":
            pages = s["page_table"][b, : -(-nk // case["page"])].long()
            k = (s["k_cache"][pages].double() * s["k_scale"][pages].double()[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :nk]
            v = (s["v_cache"][pages].double() * s["v_scale"][pages].double()[:, :, None, None]).permute(1, 0, 3, 2).flatten(1, 2)[:, :nk]
        else:
            lo = s["cu_k"].tolist()[b]
            k, v = (s[n][lo : lo + nk].double().transpose(0, 1) for n in ("k", "v"))
        for h in range(Hq):
            q = s["q"][cq[b] : cq[b + 1], h].double()
            y[cq[b] : cq[b + 1], h] = _exact_rows(q, k[h // (Hq // Hkv)].contiguous(), v[h // (Hq // Hkv)].contiguous(), s["scale"], case.get("causal", True))
    return y
