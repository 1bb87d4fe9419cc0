"""The attention calls as a serving program uses them: together with the quantized layer, through FqKvCache, from captured graphs, on
other streams, in place, with far offsets, and what the binding refuses."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import attention as A
from tests import attn_util as U

pytestmark = pytest.mark.gpu


def _angles(rows, dim):
    at = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, dim, 2) / dim)
    return np.cos(at).astype(np.float32), np.sin(at).astype(np.float32)


def _projection(rng, out, inp, bits=8):
    w = torch.from_numpy((rng.standard_normal((out, inp)) / np.sqrt(inp)).astype(np.float32)).to(torch.bfloat16).to(U.DEV)
    return fq.FqLinear(w, np.full(inp, 4.0, np.float32), 4.5, bits)


class Reference:
    """A cache in plain arrays beside an FqKvCache, stepped with the same calls."""

    def __init__(self, cache):
        self.cache = cache
        self.arrays = [t.cpu().numpy().copy() for t in (cache.k_cache, cache.v_cache, cache.k_scale, cache.v_scale)]

    def append(self, q, k, v, new, past, cos, sin, interleaved):
        table = self.cache.page_table.cpu().numpy()
        return A.append(q, k, v, U.offsets(new), past, table, *self.arrays, cos, sin, interleaved)

    def same(self):
        used = sorted(p for held in self.cache.held for p in held)
        for got, want in zip((self.cache.k_cache, self.cache.v_cache, self.cache.k_scale, self.cache.v_scale), self.arrays):
            assert np.array_equal(got.cpu().numpy()[used], want[used])


def test_prompt_then_decoding_between_quantized_projections():
    """Two uneven prompts through QKV projection, cache append, prompt attention and output projection; then a joint step, a third
    sequence's prompt while the others decode, and the end of one whose pages the next takes over."""
    rng = np.random.default_rng(0)
    hidden, hq, hkv, dim, page = 256, 4, 2, 64, 64
    qkv, out = _projection(rng, (hq + 2 * hkv) * dim, hidden), _projection(rng, hidden, hq * dim)
    cos, sin = _angles(400, dim)
    cache = fq.FqKvCache(12, 3, 400, hkv, dim, page, *U.to_dev(cos, sin))
    ref = Reference(cache)
    for t in (cache.k_cache, cache.v_cache):
        t.fill_(99)
    ref.arrays = [np.full_like(a, 99) if a.dtype == np.int8 else a for a in ref.arrays]

    def step(new, fresh):
        past, n = list(cache.lengths), sum(new)
        x = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(torch.bfloat16).to(U.DEV)
        rows = qkv.forward(x)
        q, k, v = (t.unflatten(1, (-1, dim)) for t in rows.split([hq * dim, hkv * dim, hkv * dim], 1))
        raw = [t.float().cpu().numpy() for t in (q, k, v)]
        cache.append(q, k, v, new, Q_out=q, K_out=k)               # rotated where they lie
        torch.cuda.synchronize()
        want_q, want_k = ref.append(*raw, new, past, cos, sin, False)
        ref.same()
        as_stored = lambda a: torch.from_numpy(a).to(torch.bfloat16).float().numpy()  # noqa: E731
        assert np.array_equal(q.float().cpu().numpy(), as_stored(want_q)) and np.array_equal(k.float().cpu().numpy(), as_stored(want_k))
        cu, scale = U.offsets(new), dim ** -0.5
        if fresh:
            y = torch.empty((n, hq, dim), dtype=torch.bfloat16, device=U.DEV)
            fq.fq_attn_prompt(q, k, v, U.i32(cu), U.i32(cu), max(new), scale, y)
            exact, bound = U.prompt_case(as_stored(want_q), as_stored(want_k), raw[2], cu, cu, scale, True, "bf16")
        else:
            y = cache.attend(q, new, scale)
            exact, bound = U.cache_case(as_stored(want_q), cu, cache.lengths, cache.page_table.cpu().numpy(), *ref.arrays, scale, "bf16")
        U.check(y, exact, bound, f"step {new}")
        z = out.forward(y.flatten(1))
        assert torch.isfinite(z).all() and z.shape == (n, hidden)

    step([70, 130, 0], True)
    for _ in range(3):
        step([1, 1, 0], False)
    step([1, 1, 100], False)           # the third one's prompt is a piece like any other
    step([2, 0, 5], False)
    cache.release(1)
    assert cache.lengths == [76, 0, 105]
    step([0, 200, 1], False)
    with pytest.raises(RuntimeError, match="pages wanted"):
        step([390 - 76, 0, 390 - 106], False)
    assert cache.lengths == [76, 200, 106]
    step([1, 1, 1], False)


def _decode_inputs(rng, lens, queries, hq=8, hkv=2, dim=128, page=64, x="bf16"):
    q, qn = U.packed(rng, sum(queries), hq, dim, x)
    table, pages = U.page_tables(rng, [-(-n // page) for n in lens])
    arrays = U.filled_cache(rng, pages, hkv, page, dim)
    return q, qn, table, arrays


@pytest.mark.parametrize("lens,queries", [([900, 300], [1, 1]), ([700, 500], [30, 20])])
def test_captured_cache_attention_follows_lengths_and_cache(lens, queries):
    """One capture, replayed with other lengths, queries, pages and codes, with eager calls between; each replay against the plain form."""
    rng = np.random.default_rng(1)
    q, qn, table, arrays = _decode_inputs(rng, lens, queries)
    dev, tab, cu, ln = U.to_dev(*arrays), U.i32(table), U.i32(U.offsets(queries)), U.i32(lens)
    y, scale = torch.empty_like(q), 0.09
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, q.shape[0], max(queries), 1000, 8, 2, 128), dtype=torch.uint8, device=U.DEV)
    call = lambda out: fq.fq_attn_cache(q, cu, ln, max(queries), 1000, *dev, tab, scale, out, ws)  # noqa: E731
    call(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(y)
    for turn in range(4):
        now = [max(0, n - 211 * turn) for n in lens]
        ln.copy_(U.i32(now))
        q.copy_(q.roll(1, 2))
        dev[1].copy_(dev[1].roll(turn, 2))
        arrays = (arrays[0], dev[1].cpu().numpy(), arrays[2], arrays[3])
        ws.fill_(0xFF)
        y.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        exact, bound = U.cache_case(q.float().cpu().numpy(), U.offsets(queries), now, table, *arrays, scale, "bf16")
        U.check(y, exact, bound, f"replay {turn}")
        eager = torch.empty_like(q)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, y)


@pytest.mark.parametrize("batch", [12, 70])
def test_captured_calls_follow_how_the_rows_are_dealt_out(batch):
    """An append, a prompt's attention and attention of pieces, captured once and replayed with the rows dealt out otherwise among the sequences."""
    rng = np.random.default_rng(batch)
    rows, hq, hkv, dim, page, longest, scale = 700, 4, 2, 64, 64, 520, 0.11
    (q, qn), (k, kn), (v, vn) = (U.packed(rng, rows, h, dim, "bf16") for h in (hq, hkv, hkv))
    table, pages = U.page_tables(rng, [-(-longest // page)] * batch)
    start = U.filled_cache(rng, pages, hkv, page, dim)
    dev, tab, cu, none, ln = U.to_dev(*start), U.i32(table), U.i32([0] * (batch + 1)), U.i32([0] * batch), U.i32([0] * batch)
    k_out, y, z = torch.empty_like(k), torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(batch, rows, longest, longest, hq, hkv, dim), dtype=torch.uint8, device=U.DEV)

    def calls():
        fq.fq_kv_append(None, k, v, cu, none, longest, *dev, tab, K_out=k_out)
        fq.fq_attn_prompt(q, k_out, v, cu, cu, longest, scale, y)
        fq.fq_attn_cache(q, cu, ln, longest, longest, *dev, tab, scale, z, ws)
    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    deals = [[rows // batch] * batch, [longest] + [2] * (batch - 1), [1] * (batch - 1) + [longest], [0, 300] + [0] * (batch - 3) + [400]]
    for turn, lens in enumerate(deals):
        at = U.offsets(lens)
        n = at[-1]
        assert n <= rows
        cu.copy_(U.i32(at)), ln.copy_(U.i32(lens))
        for have, value in zip(dev, U.to_dev(*start)):
            have.copy_(value)
        ws.fill_(0xFF), y.fill_(5.0), z.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        want = [a.copy() for a in start]
        A.append(qn, kn, vn, at, [0] * batch, table, *want, None, None, False)
        for got, w in zip(dev, want):
            assert np.array_equal(got.cpu().numpy(), w), turn
        U.check(y[:n], *U.prompt_case(qn[:n], kn[:n], vn[:n], at, at, scale, True, "bf16"), f"prompt {turn}")
        exact, bound = U.cache_case(qn, at, lens, table, *want, scale, "bf16", longest)
        U.check(z[:n], exact[:n], bound[:n], f"pieces {turn}")
        assert (y[n:] == 5.0).all() and (z[n:] == 5.0).all()


def test_captured_decoding_steps_share_cache_and_workspace():
    """A graph of a decoding step (append, then attention) and one of another batch's, both on one workspace, replayed in turn."""
    rng = np.random.default_rng(2)
    dim, hq, hkv, page = 64, 4, 2, 64
    cos, sin = _angles(300, dim)
    cosd, sind = U.to_dev(cos, sin)
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, 2, 1, 4000, hq, hkv, dim), dtype=torch.uint8, device=U.DEV)
    assert ws.numel() > 16
    steps = []
    for past in ([10, 63], [150, 200]):
        table, pages = U.page_tables(rng, [4, 4])
        arrays = U.filled_cache(rng, pages, hkv, page, dim)
        s = dict(past=np.array(past, np.int32), table=table, arrays=arrays, dev=U.to_dev(*arrays), tab=U.i32(table), pd=U.i32(past), ld=U.i32(np.array(past) + 1), cu=U.i32([0, 1, 2]))
        s["rows"] = torch.empty((2, (hq + 2 * hkv) * dim), dtype=torch.float16, device=U.DEV)
        s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, dim)) for t in s["rows"].split([hq * dim, hkv * dim, hkv * dim], 1))
        s["qo"], s["y"] = (torch.empty((2, hq, dim), dtype=torch.float16, device=U.DEV) for _ in range(2))

        def run(s=s):
            fq.fq_kv_append(s["q"], s["k"], s["v"], s["cu"], s["pd"], 1, *s["dev"], s["tab"], rope_cos=cosd, rope_sin=sind, Q_out=s["qo"])
            fq.fq_attn_cache(s["qo"], s["cu"], s["ld"], 1, 4000, *s["dev"], s["tab"], 0.125, s["y"], ws)
            s["pd"].add_(1)
            s["ld"].add_(1)
        s["rows"].zero_()
        saved = [t.clone() for t in s["dev"]]
        run()
        for t, u in zip(s["dev"], saved):
            t.copy_(u)
        s["pd"].copy_(U.i32(past))
        s["ld"].copy_(U.i32(np.array(past) + 1))
        s["g"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["g"]):
            run()
        steps.append(s)
    for turn in range(4):
        for s in steps:
            values = rng.standard_normal(s["rows"].shape).astype(np.float32) * (1 + turn)
            s["rows"].copy_(torch.from_numpy(values))
            s["g"].replay()
        torch.cuda.synchronize()
        for s in steps:
            q, k, v = (t.float().cpu().numpy() for t in (s["q"], s["k"], s["v"]))
            rq, _ = A.append(q, k, v, [0, 1, 2], s["past"], s["table"], *s["arrays"], cos, sin, False)
            s["past"] += 1
            for got, want in zip(s["dev"], s["arrays"]):
                assert np.array_equal(got.cpu().numpy(), want)
            rq = torch.from_numpy(rq).half().float().numpy()
            exact, bound = U.cache_case(rq, [0, 1, 2], s["past"], s["table"], *s["arrays"], 0.125, "f16")
            U.check(s["y"], exact, bound, f"turn {turn}")


def test_calls_go_to_the_stream_that_is_current_or_given():
    rng = np.random.default_rng(3)
    lens = [400, 90]
    q, k, v = (U.packed(rng, sum(lens), h, 64, "bf16")[0] for h in (4, 2, 2))
    cu = U.i32(U.offsets(lens))
    want, got = torch.empty_like(q), [torch.zeros_like(q) for _ in range(2)]
    fq.fq_attn_prompt(q, k, v, cu, cu, 400, 0.125, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=U.DEV)
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-4                               # keeps the side stream busy
        late = q + 0 * big[0, 0].to(q.dtype).nan_to_num(0.0, 0.0, 0.0)
        fq.fq_attn_prompt(late, k, v, cu, cu, 400, 0.125, got[0])
    fq.fq_attn_prompt(late, k, v, cu, cu, 400, 0.125, got[1], stream=side)
    side.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want)


def test_two_streams_at_once_with_workspaces_of_their_own():
    rng = np.random.default_rng(4)
    jobs = []
    for lens in ([3000], [2500]):
        q, qn, table, arrays = _decode_inputs(rng, lens, [1], hq=4, hkv=1, dim=64)
        ws = torch.empty(fq.fq_attn_cache_workspace_bytes(1, 1, 1, 3000, 4, 1, 64), dtype=torch.uint8, device=U.DEV)
        jobs.append((q, U.i32([0, 1]), U.i32(lens), U.to_dev(*arrays), U.i32(table), ws, torch.cuda.Stream()))
    call = lambda j, y: fq.fq_attn_cache(j[0], j[1], j[2], 1, 3000, *j[3], j[4], 0.125, y, j[5])  # noqa: E731
    want = [torch.empty_like(j[0]) for j in jobs]
    for j, y in zip(jobs, want):
        call(j, y)
    torch.cuda.synchronize()
    got = [[torch.empty_like(j[0]) for _ in range(20)] for j in jobs]
    for i in range(20):
        for j, ys in zip(jobs, got):
            with torch.cuda.stream(j[6]):
                call(j, ys[i])
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)


@pytest.mark.parametrize("lens,queries", [([130, 64], [130, 64]), ([3000, 2000], [1, 1]), ([500, 90], [40, 3])])
def test_output_in_the_place_of_the_queries(lens, queries):
    rng = np.random.default_rng(5)
    q, qn, table, arrays = _decode_inputs(rng, lens, queries, dim=80)
    cu, ln = U.i32(U.offsets(queries)), U.i32(lens)
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, q.shape[0], max(queries), max(lens), 8, 2, 80), dtype=torch.uint8, device=U.DEV)
    args = (cu, ln, max(queries), max(lens), *U.to_dev(*arrays), U.i32(table), 0.1)
    y = torch.empty_like(q)
    fq.fq_attn_cache(q, *args, y, ws)
    own = q.clone()
    fq.fq_attn_cache(own, *args, own, ws)
    k, v = (U.packed(rng, sum(lens), 2, 80, "bf16")[0] for _ in range(2))
    cu_k = U.i32(U.offsets(lens))
    z, own_z = torch.empty_like(q), q.clone()
    fq.fq_attn_prompt(q, k, v, cu, cu_k, max(queries), 0.1, z)
    fq.fq_attn_prompt(own_z, k, v, cu, cu_k, max(queries), 0.1, own_z)
    torch.cuda.synchronize()
    assert torch.equal(y, own) and torch.equal(z, own_z)


def test_pages_beyond_four_gigabytes():
    """Page numbers whose codes lie beyond 2^32 bytes: as the same pages at the pool's begin."""
    rng = np.random.default_rng(6)
    hkv, dim, page, far = 8, 128, 64, 70000                      # 65536 bytes a page: 4.6 GB of keys
    low = np.array([[3, 0, 2], [1, 4, -1]], np.int32)
    pools = [(torch.empty((n, hkv, page, dim), dtype=torch.int8, device=U.DEV), torch.empty((n, hkv, dim, page), dtype=torch.int8, device=U.DEV),
              torch.empty((n, hkv), device=U.DEV), torch.empty((n, hkv), device=U.DEV)) for n in (5, far + 5)]
    for pool in pools:                                           # slots behind the last token keep what memory held
        pool[0][-5:], pool[1][-5:] = 11, 12
    tables = [low, np.where(low >= 0, low + far, low).astype(np.int32)]
    q = U.packed(rng, 150 + 70, 8, dim, "bf16")[0]
    k, v = (U.packed(rng, 150 + 70, hkv, dim, "bf16")[0] for _ in range(2))
    one = U.packed(rng, 2, 8, dim, "bf16")[0]
    results = []
    for pool, table in zip(pools, tables):
        tab = U.i32(table)
        fq.fq_kv_append(None, k, v, U.i32([0, 150, 220]), U.i32([0, 0]), 150, *pool, tab)
        fq.fq_kv_append(None, k[:5] * 3, v[:5] * 3, U.i32([0, 3, 5]), U.i32([150, 70]), 3, *pool, tab)
        ys = []
        for qs, n in ((one, [1, 1]), (q, [150, 70])):
            y = torch.empty_like(qs)
            ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, qs.shape[0], max(n), 192, 8, hkv, dim), dtype=torch.uint8, device=U.DEV)
            fq.fq_attn_cache(qs, U.i32(U.offsets(n)), U.i32([153, 72]), max(n), 192, *pool, tab, 0.09, y, ws)
            ys.append(y)
        torch.cuda.synchronize()
        results.append((*ys, pool[0][-5:].clone(), pool[1][-5:].clone(), pool[2][-5:].clone(), pool[3][-5:].clone()))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_rows_beyond_two_to_the_32_elements():
    """Token strides of 2^22 elements, the largest allowed: the last rows lie beyond 2^32 elements."""
    rng = np.random.default_rng(7)
    tokens, ld, dim = 1100, 1 << 22, 64
    small = [U.packed(rng, tokens, h, dim, "bf16", pad=0)[0] for h in (2, 1, 1)]
    wide = torch.empty(tokens * ld, dtype=torch.bfloat16, device=U.DEV)
    far, at = [], 0
    for t in small:
        h = t.shape[1]
        view = wide.as_strided((tokens, h, dim), (ld, dim, 1), at)
        view.copy_(t)
        far.append(view)
        at += h * dim
    out = wide.as_strided((tokens, 2, dim), (ld, dim, 1), at)
    cu = U.i32([0, 40, tokens])
    want = torch.empty_like(small[0])
    fq.fq_attn_prompt(*small, cu, cu, tokens, 0.125, want)
    fq.fq_attn_prompt(*far, cu, cu, tokens, 0.125, out)
    table = U.i32(np.arange(20).reshape(1, 20))
    caches = []
    for q, k, v in (small, far):
        c = [torch.zeros((20, 1, 64, dim), dtype=torch.int8, device=U.DEV), torch.zeros((20, 1, dim, 64), dtype=torch.int8, device=U.DEV),
             torch.zeros((20, 1), device=U.DEV), torch.zeros((20, 1), device=U.DEV)]
        fq.fq_kv_append(None, k, v, U.i32([0, tokens]), U.i32([0]), tokens, *c, table)
        caches.append(c)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert all(torch.equal(a, b) for a, b in zip(*caches))


def test_lengths_beyond_the_bounds_of_the_call_are_cut():
    """max_len, the page table, max_q and max_new bound what a call does, whatever stands on the device."""
    rng = np.random.default_rng(8)
    q, qn, table, arrays = _decode_inputs(rng, [256, 256], [1, 1])
    table = table[:, :4].copy()
    dev = U.to_dev(*arrays)
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, 2, 1, 100000, 8, 2, 128), dtype=torch.uint8, device=U.DEV)
    for lens, max_len, used in (([2**31 - 1, 2**30], 100000, [256, 256]), ([300, -5], 200, [200, 0])):
        y = torch.full_like(q, 3.0)
        fq.fq_attn_cache(q, U.i32([0, 1, 2]), U.i32(lens), 1, max_len, *dev, U.i32(table), 0.1, y, ws)
        torch.cuda.synchronize()
        exact, bound = U.cache_case(qn, [0, 1, 2], used, table, *arrays, 0.1, "bf16")
        U.check(y, exact, bound, f"lens {lens}")
    for cu in ([-7, 1, 9], [0, 1 << 30, -(1 << 31)], [2, 2, 2]):
        y = torch.full_like(q, 3.0)
        fq.fq_attn_cache(q, U.i32(cu), U.i32([256, 256]), 1, 256, *dev, U.i32(table), 0.1, y, ws)
        fq.fq_attn_prompt(q, q[:, :2], q[:, :2], U.i32(cu), U.i32(cu), 1, 0.1, y)
        fq.fq_kv_append(None, q[:, :2], q[:, :2], U.i32(cu), U.i32([2**31 - 1, -9]), 1, *U.to_dev(*arrays), U.i32(table))
        torch.cuda.synchronize()


def test_index_arrays_need_no_alignment_beyond_their_type():
    rng = np.random.default_rng(9)
    lens, queries = [300, 70], [1, 1]
    q, qn, table, arrays = _decode_inputs(rng, lens, queries)
    shifted = lambda a: torch.cat([U.i32([7]), U.i32(a).flatten()])[1:].view(np.shape(a))  # noqa: E731
    y = torch.empty_like(q)
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(2, 2, 1, 300, 8, 2, 128), dtype=torch.uint8, device=U.DEV)
    fq.fq_attn_cache(q, shifted([0, 1, 2]), shifted(lens), 1, 300, *U.to_dev(*arrays), shifted(table), 0.1, y, ws)
    torch.cuda.synchronize()
    exact, bound = U.cache_case(qn, [0, 1, 2], lens, table, *arrays, 0.1, "bf16")
    U.check(y, exact, bound, "shifted")


def test_results_do_not_change_from_run_to_run():
    rng = np.random.default_rng(10)
    q, qn, table, arrays = _decode_inputs(rng, [5000, 33, 1200], [2, 1, 3])
    dev, tab, cu, ln = U.to_dev(*arrays), U.i32(table), U.i32([0, 2, 3, 6]), U.i32([5000, 33, 1200])
    ws = torch.empty(fq.fq_attn_cache_workspace_bytes(3, 6, 3, 5000, 8, 2, 128), dtype=torch.uint8, device=U.DEV)
    ys = [torch.empty_like(q) for _ in range(5)]
    for y in ys:
        ws.random_()
        fq.fq_attn_cache(q, cu, ln, 3, 5000, *dev, tab, 0.1, y, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(ys[0], y) for y in ys)


def test_binding_refuses_what_does_not_fit_together():
    q = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device=U.DEV)
    k, f32 = q[:, :2], q.float()
    cu, ln = U.i32([0, 2, 4]), U.i32([5, 6])
    cache = [torch.zeros((4, 2, 64, 64), dtype=torch.int8, device=U.DEV), torch.zeros((4, 2, 64, 64), dtype=torch.int8, device=U.DEV),
             torch.zeros((4, 2), device=U.DEV), torch.zeros((4, 2), device=U.DEV)]
    tab, y, ws = U.i32([[0, 1], [2, 3]]), torch.empty_like(q), torch.empty(1 << 20, dtype=torch.uint8, device=U.DEV)
    cos = torch.zeros((128, 32), device=U.DEV)
    with pytest.raises(ValueError, match="on cpu"):
        fq.fq_attn_prompt(q.cpu(), k, k, cu, cu, 2, 0.1, y)
    with pytest.raises(ValueError, match="dense heads"):
        fq.fq_attn_prompt(q.transpose(0, 1).contiguous().transpose(0, 1), k, k, cu, cu, 2, 0.1, y)
    with pytest.raises(ValueError, match="shape and type"):
        fq.fq_attn_prompt(q, k, k.float(), cu, cu, 2, 0.1, y)
    with pytest.raises(ValueError, match="shape and type"):
        fq.fq_attn_prompt(q, k, k, cu, cu, 2, 0.1, y[:3])
    with pytest.raises(ValueError, match="cu_k"):
        fq.fq_attn_prompt(q, k, k, cu, U.i32([0, 4]), 2, 0.1, y)
    with pytest.raises(ValueError, match="cu_q"):
        fq.fq_attn_prompt(q, k, k, cu.long(), cu, 2, 0.1, y)
    with pytest.raises(fq.FqError, match="FQ_ERR_DTYPE"):
        fq.fq_attn_prompt(f32, f32[:, :2], f32[:, :2], cu, cu, 2, 0.1, f32)
    with pytest.raises(ValueError, match="v_cache"):
        fq.fq_attn_cache(q, cu, ln, 2, 6, cache[0], cache[1][:, :1], *cache[2:], tab, 0.1, y, ws)
    with pytest.raises(ValueError, match="k_scale"):
        fq.fq_attn_cache(q, cu, ln, 2, 6, cache[0], cache[1], cache[2].half(), cache[3], tab, 0.1, y, ws)
    with pytest.raises(ValueError, match="page_table"):
        fq.fq_attn_cache(q, cu, ln, 2, 6, *cache, tab[:1], 0.1, y, ws)
    with pytest.raises(ValueError, match="workspace"):
        fq.fq_attn_cache(q, cu, ln, 2, 6, *cache, tab, 0.1, y, ws.cpu())
    with pytest.raises(fq.FqError, match="FQ_ERR_WORKSPACE"):
        fq.fq_attn_cache(q, cu, ln, 2, 100000, *cache, tab, 0.1, y, ws[:16])
    with pytest.raises(ValueError, match="go together"):
        fq.fq_kv_append(q, k, k, cu, ln, 2, *cache, tab, rope_cos=cos)
    with pytest.raises(ValueError, match="rope_sin"):
        fq.fq_kv_append(q, k, k, cu, ln, 2, *cache, tab, rope_cos=cos, rope_sin=cos[:5])
    with pytest.raises(ValueError, match="Q_out without Q"):
        fq.fq_kv_append(None, k, k, cu, ln, 2, *cache, tab, Q_out=y)
    with pytest.raises(ValueError, match="heads"):
        fq.fq_kv_append(None, q, q, cu, ln, 2, *cache, tab)
    with pytest.raises(ValueError, match="tokens"):
        fq.fq_kv_append(q[:3], k, k, cu, ln, 2, *cache, tab, Q_out=y[:3])
    with pytest.raises(fq.FqError, match="FQ_ERR_SHAPE"):
        fq.fq_kv_append(None, k, k, cu, ln, 2, *cache, tab, rope_cos=torch.zeros((9, 40), device=U.DEV), rope_sin=torch.zeros((9, 40), device=U.DEV))
