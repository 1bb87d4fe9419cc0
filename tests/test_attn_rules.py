"""What the attention kernels make of device-resident offsets, lengths and page tables (csrc/fq_attn_rules.h), compiled with the host
compiler and walked on the CPU: every address they form comes from these."""
import ctypes
import random
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2402_17985_amd", "csrc")
LO, HI = -(2**31), 2**31 - 1

DRIVER = """
#include "fq_attn_rules.h"
using namespace fq;
extern "C" void rows(int from, int to, int rows, int most, int* out)
{
    const Rows r = packed_rows(from, to, rows, most);
    out[0] = r.first; out[1] = r.count;
}
extern "C" void fill(int first, int count, int past, int j, int page, int capacity, int* out)
{
    const Fill f = page_fill(Rows{first, count}, past, j, page, capacity);
    out[0] = f.index; out[1] = f.slot0; out[2] = f.slot1; out[3] = f.row; out[4] = f.pos;
}
extern "C" long long touched(int tokens, int page) { return pages_touched(tokens, page); }
extern "C" int append(int max_new, int page, int dim)
{
    const AppendPlan p = append_plan(max_new, page, dim);
    return p.few ? p.threads : -p.threads;
}
extern "C" int keys(int len, int max_len, int capacity) { return cached_keys(len, max_len, capacity); }
extern "C" int visible(int keys, int n, int i) { return visible_keys(keys, n, i); }
extern "C" int share(int keys, int splits, int round) { return share_keys(keys, splits, round); }
extern "C" int used(int keys, int share) { return shares_used(keys, share); }
extern "C" void plan(int batch, int tokens, int max_q, int max_len, int heads_q, int heads_kv, long long* out)
{
    const CachePlan p = cache_plan(batch, tokens, max_q, max_len, heads_q, heads_kv);
    out[0] = p.tiles; out[1] = p.round; out[2] = p.splits; out[3] = cache_holds(p, heads_kv); out[4] = p.places;
}
extern "C" void unit(unsigned id, unsigned members, unsigned heads_kv, unsigned* out)
{
    const TileUnit u = tile_unit(id, members, heads_kv);
    out[0] = u.place; out[1] = u.head_kv; out[2] = u.member;
}
extern "C" void pages(int batch, int tokens, int max_new, int page, long long* out)
{
    const AppendPages p = append_pages(batch, tokens, max_new, page);
    out[0] = p.places; out[1] = p.each;
}
extern "C" int first_page(int row, int page, int b) { return first_page_place(row, page, b); }
extern "C" long long places(long long tokens, int batch, long long longest, int rows) { return tile_places(tokens, batch, longest, rows); }
extern "C" long long workgroups(long long places, int members, int heads_kv) { return tile_workgroups(places, members, heads_kv); }
extern "C" int first(long long row, int rows, int b) { return first_place(row, rows, b); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("attn_rules")
    src, so = str(d / "rules.cpp"), str(d / "rules.so")
    with open(src, "w") as f:
        f.write(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan",
                    "-shared", "-fPIC", "-I", CSRC, "-o", so, src], check=True)
    lib = ctypes.CDLL(so)
    lib.touched.restype = lib.places.restype = lib.workgroups.restype = ctypes.c_longlong
    lib.places.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int]
    lib.workgroups.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    lib.first.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return lib


@pytest.mark.parametrize("total", [0, 1, 100, HI])
def test_rows_stay_within_the_array(rules, total):
    out = (ctypes.c_int * 2)()
    for a in (LO, -1, 0, 1, 50, 100, 101, HI):
        for b in (LO, -1, 0, 1, 50, 100, 101, HI):
            for most in (1, 7, HI):
                rules.rows(a, b, total, most, out)
                first, count = out
                assert 0 <= first <= total and 0 <= count <= min(most, total - first)
                if 0 <= a <= b <= total and b - a <= most:
                    assert (first, count) == (a, b - a)


@pytest.mark.parametrize("page", [64, 128])
def test_page_fills_cover_the_new_tokens_once_and_stay_within_a_page(rules, page):
    out = (ctypes.c_int * 5)()
    for width in (1, 3, 9):
        for reach in (width * page, width * page - 37):
            for past in (0, 1, page - 1, page, 2 * page + 3, 5 * page - 1):
                for n in (0, 1, 2, page - 1, page, page + 1, 3 * page + 5):
                    seen = {}
                    for j in range(rules.touched(max(n, 1), page)):
                        rules.fill(1000, n, past, j, page, reach, out)
                        index, s0, s1, row, pos = out
                        if s1 <= s0:
                            continue
                        assert 0 <= index < width and 0 <= s0 < s1 <= page and pos == index * page + s0 and row == 1000 + pos - past
                        for s in range(s0, s1):
                            assert index * page + s not in seen
                            seen[index * page + s] = row + s - s0
                    assert seen == {p: 1000 + p - past for p in range(past, min(past + n, reach))}


@pytest.mark.parametrize("past", [LO, -1, 0, 2**30 - 1, 2**30, HI])
@pytest.mark.parametrize("capacity", [64, 2**30])
def test_page_fills_of_wild_lengths_stay_within_the_table(rules, past, capacity):
    out = (ctypes.c_int * 5)()
    for n in (0, 1, 200, HI):
        for j in (0, 1, 5, 2**25, HI // 64):
            rules.fill(0, n, past, j, 64, capacity, out)
            index, s0, s1, row, pos = out
            if s1 > s0:
                assert 0 <= index < capacity // 64 and 0 <= s0 < s1 <= 64 and 0 <= row and row + s1 - s0 <= n and pos + s1 - s0 <= capacity


@pytest.mark.parametrize("n,page,most", [(1, 64, 1), (2, 64, 2), (64, 64, 2), (65, 64, 2), (66, 64, 3), (HI, 64, 2**25 + 1)])
def test_pages_touched(rules, n, page, most):
    assert rules.touched(n, page) == most


def test_keys_and_visible_keys(rules):
    for length in (LO, -1, 0, 5, 1000, HI):
        for max_len in (1, 100, HI):
            for capacity in (64, 2**30):
                assert rules.keys(length, max_len, capacity) == max(0, min(length, max_len, capacity))
    for keys in (0, 1, 5, 2**30):
        for n in (1, 3, 7, 2**30):
            for i in {0, 1, n - 1}:
                assert rules.visible(keys, n, i) == max(0, keys - n + i + 1)


@pytest.mark.parametrize("waves", [1, 2, 4])
def test_shares_cover_all_keys_in_whole_steps(rules, waves):
    for splits in (1, 2, 3, 7, 64, 256):
        for keys in (0, 1, 255, 256, 257, 1000, 4096, 131072, 2**30 - 1, 2**30):
            share = rules.share(keys, splits, waves)
            assert share >= 64 * waves and share % (64 * waves) == 0 and share * splits >= keys
            used = rules.used(keys, share)
            assert used <= splits and (used - 1) * share < keys <= used * share or (keys == 0 and used == 0)


def test_plans_are_bounded_and_do_not_split_where_there_is_work_enough(rules):
    out = (ctypes.c_longlong * 5)()
    for batch in (1, 4, 64, 65535):
        for max_q in (1, 5, 512, 65472):
            for max_len in (1, 256, 257, 8192, 2**30):
                for hq, hkv in ((1, 1), (64, 8), (64, 64), (16384, 1)):
                    if max_q * hq >= 2**30:
                        continue
                    tokens = min(batch * max_q, HI)
                    rules.plan(batch, tokens, max_q, max_len, hq, hkv, out)
                    tiles, rnd, splits, holds, places = out
                    columns = max_q * (hq // hkv)
                    by32 = -(-columns // 32)
                    many = columns > 32 and (batch * hkv * by32 > 768 or (columns > 64 and columns * batch * hkv > 2**25 // max_len))
                    assert tiles == (1 if columns <= 16 else 8 if many else 2)
                    assert places == (rules.places(tokens * (hq // hkv), batch, columns, 128) if many else by32) > 0
                    wgs = hkv * places * (1 if many else batch)
                    assert rnd == (1 if tiles == 8 else 2 if tiles == 1 and wgs <= 256 and max_len // (256 // wgs) >= 2048 else 4)
                    assert 1 <= splits <= 256 and (splits - 1) * 64 * rnd < max_len
                    assert splits == 1 or wgs * splits <= (512 if tiles == 8 else 256)
                    along_x = -(-wgs // 8) * 8 * splits if tiles == 8 else splits
                    assert holds == (along_x * 512 < 2**32)
                    assert splits == 1 or min(max_q, tokens) <= 65535      # the join has the query tokens along y


@pytest.mark.parametrize("rows", [16, 128])
@pytest.mark.parametrize("batch", [1, 2, 7, 64, 65, 300, 5000])
def test_every_tile_of_every_sequence_has_a_place(rules, batch, rows):
    r = random.Random(1000 * batch + rows)
    for longest in (1, rows - 1, rows, rows + 1, 10 * rows + 3):
        for lens in ([longest] * batch, [r.randrange(longest + 1) for _ in range(batch)], [longest] + [0] * (batch - 1), [0] * (batch - 1) + [longest]):
            tiles, tokens = [-(-n // rows) for n in lens], sum(lens)
            places = rules.places(tokens, batch, longest, rows)
            assert sum(tiles) <= places <= tokens // rows + batch
            if batch <= 64:
                assert places <= batch * -(-longest // rows)
                continue
            row = 0
            for b, n in enumerate(lens):      # a sequence's tiles end before the next one's first place
                behind = rules.first(row + n, rows, b + 1)
                assert rules.first(row, rows, b) + tiles[b] <= behind <= places
                row += n


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("batch", [1, 2, 30, 64, 65, 3000])
def test_every_page_of_every_append_has_a_place(rules, batch, page):
    r, out, forms = random.Random(batch + page), (ctypes.c_longlong * 2)(), set()
    for longest in (1, 2, page, page + 1, page + 2, 20 * page + 5):
        for new in ([longest] * batch, [r.randrange(longest + 1) for _ in range(batch)], [longest] + [1] * (batch - 1), [1] * (batch - 1) + [longest]):
            rules.pages(batch, sum(new), max(new + [1]), page, out)
            places, each = out
            forms.add(each > 0)
            if each:
                assert places == batch * each and each == rules.touched(max(new + [1]), page)
                continue
            row = 0
            for b, n in enumerate(new):
                touched = rules.touched(n, page) if n else 0
                assert rules.first_page(row, page, b) + touched <= rules.first_page(row + n, page, b + 1) <= places
                row += n
    assert forms == ({True} if batch <= 2 else {True, False})


@pytest.mark.parametrize("places,members,heads_kv", [(1, 1, 1), (1, 7, 1), (3, 8, 5), (5, 9, 8), (16, 2, 12), (2, 64, 40), (7, 1, 3), (64, 8, 8)])
def test_units_are_each_taken_once_and_a_heads_members_stay_on_an_xcd(rules, places, members, heads_kv):
    out, seen, xcds, taken = (ctypes.c_uint * 3)(), set(), {}, [0] * 8
    for i in range(rules.workgroups(places, members, heads_kv)):
        rules.unit(i, members, heads_kv, out)
        place, head, member = out
        assert head < heads_kv and member < members
        if place < places:
            seen.add((place, head, member))
            xcds.setdefault((place, head), set()).add(i % 8)
            xcds.setdefault(head, set()).add(i % 8)
            taken[i % 8] += 1
    assert len(seen) == places * members * heads_kv == sum(taken)
    assert all(len(x) == 1 for k, x in xcds.items() if isinstance(k, tuple) or heads_kv % 8 == 0)
    assert max(taken) - min(taken) <= members


def test_units_of_a_launch_of_2_to_the_31_workgroups(rules):
    out = (ctypes.c_uint * 3)()
    for places, members, heads_kv in ((2**15, 65535, 1), (2**31 - 8, 1, 1), (1, 1, 2**31 - 8), (2**24, 127, 1), (2**10, 2**8, 2**12)):
        n = rules.workgroups(places, members, heads_kv)
        assert places * members * heads_kv <= n < 2**31 + 2**20
        for i in (0, 7, n // 2, n - 1):
            rules.unit(i, members, heads_kv, out)
            assert out[1] < heads_kv and out[2] < members and out[0] * heads_kv + out[1] <= -(-places * heads_kv // 8) * 8


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
def test_append_threads_hold_what_a_call_adds_to_a_page(rules, page, dim):
    for new in (1, 2, 4, 5, 16, 17, 32, 33, 63, 64, 65, 1000, HI):
        threads, pieces = rules.append(new, page, dim), min(new, page) * dim // 8
        few = threads > 0
        threads = abs(threads)
        assert threads % 64 == 0 and 64 <= threads <= 512 and pieces <= threads * (1 if few else -(-dim // 8 // 4))
        assert few == (pieces <= 512)
