// What the attention kernels take from device-resident lengths and page tables, and their launch rules: plain arithmetic on
// sizes without HIP types, so that a test can compile it with the host compiler and walk it.  Lengths, offsets and page numbers
// live on the device and cannot be checked when a call is made; every one that a kernel uses for an address passes through here.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

#ifdef __HIPCC__
#define FQ_BOTH __attribute__((host, device)) inline
#else
#define FQ_BOTH inline
#endif

namespace fq {

constexpr int CACHE_STEP = 64;        // keys that a wave of the cache's attention takes at a time; pages are a multiple of it
constexpr int MAX_PAGE = 128;
constexpr int ATTN_DIMS[] = {64, 80, 96, 128};

// Rows [first, first + count) of a packed array of `rows` rows, from two neighbouring offsets; at most `most` of them.
struct Rows {
    int first, count;
};
FQ_BOTH Rows packed_rows(int from, int to, int rows, int most)
{
    const int a = from < 0 ? 0 : from > rows ? rows : from;
    const int b = to < a ? a : to > rows ? rows : to;
    return Rows{a, b - a < most ? b - a : most};
}

// The j-th page that a sequence's new tokens touch: slots [slot0, slot1) of the sequence's page `index` take the rows from
// `row` on, the first of them at position `pos`.  Tokens at `capacity` or beyond have no place.
struct Fill {
    int index, slot0, slot1, row, pos;
};
FQ_BOTH Fill page_fill(Rows r, int past, int j, int page, int capacity)
{
    const int begin = past < 0 ? 0 : past;
    const long long end = begin + (long long)r.count < capacity ? begin + (long long)r.count : capacity;
    const long long index = (long long)(begin / page) + j, base = index * page;
    const long long lo = base < begin ? begin : base, hi = base + page < end ? base + page : end;
    if (lo >= hi) return Fill{0, 0, 0, 0, 0};
    return Fill{(int)index, (int)(lo - base), (int)(hi - base), (int)(r.first + (lo - begin)), (int)lo};
}
// Pages that `tokens` tokens can touch, wherever the first one lies in its page.
inline long long pages_touched(int tokens, int page) { return ((long long)tokens + page - 2) / page + 1; }

// The pages that an append's workgroups look at.  As many for each sequence as max_new tokens can touch; or, where that is twice what all tokens' rows
// can need, place by place: sequence b's pages begin at place cu_new[b] / page + 2 b (n tokens touch n / page + 2 pages at most, rounded down).
// us, so many for each / place by place: 64 sequences, one with 4096 new tokens and 63 with one, 40 heads, 411 / 84; one with 512, 64 heads over 8, 21 / 18;
// 30 of 10 to 1000 tokens (1.7 times what they need), 32 heads over 8, 114 / 118.
struct AppendPages {
    long long places;
    int each;      // of a sequence, or 0: place by place
};
inline AppendPages append_pages(int batch, int tokens, int max_new, int page)
{
    const long long each = pages_touched(max_new, page), by_rows = tokens / page + 2LL * batch;
    return 2 * by_rows < batch * each ? AppendPages{by_rows, 0} : AppendPages{batch * each, (int)each};
}
FQ_BOTH int first_page_place(int row, int page, int b) { return row / page + 2 * b; }

// An append's workgroup takes what one call adds to a page of one head: 8 elements a thread where 512 threads are enough for the most new
// tokens (64 sequences, one token each, 64 heads over 8: 5.2 us with 64 threads, 7.2 with 256), else up to 32 and four threads a token of the page.
struct AppendPlan {
    bool few;
    int threads;
};
inline AppendPlan append_plan(int max_new, int page, int head_dim)
{
    const long long pieces = std::min(max_new, page) * (long long)(head_dim / 8);
    if (pieces <= 512) return AppendPlan{true, (int)(pieces + 63) / 64 * 64};
    return AppendPlan{false, 4 * page};
}
// Inside a page tokens are addressed with 32-bit byte offsets.
constexpr long long MAX_TOKEN_STRIDE = 1 << 22;

// Keys of a sequence that the cache holds and its page table reaches.
FQ_BOTH int cached_keys(int len, int max_len, int capacity)
{
    const int most = max_len < capacity ? max_len : capacity;
    return len < 0 ? 0 : len > most ? most : len;
}

// Keys that query i of n sees when the last one sees all `keys` (causal; none: 0).
FQ_BOTH int visible_keys(int keys, int n, int i)
{
    const int v = keys - n + i + 1;
    return v < 0 ? 0 : v;
}

// Places for the tiles of `rows` rows each that packed sequences of `tokens` rows in all have, at least as many as there can be.  Their number, not
// the longest sequence times the sequences, sets a launch: most of that would be workgroups without work where lengths differ.  Of up to 64 sequences,
// which the kernels order by their lengths, the tiles follow one another without gaps; of more, sequence b's begin at place (its first row) / rows + b,
// which leaves room for its last, partly filled one and is found without adding up the others.
constexpr int SORTED_SEQUENCES = 64;
inline long long tile_places(long long tokens, int batch, long long longest, int rows)
{
    const long long by_rows = tokens / rows + batch, by_length = batch * ((longest + rows - 1) / rows);
    return batch <= SORTED_SEQUENCES ? std::min(by_rows, by_length) : by_rows;
}
FQ_BOTH int first_place(long long row, int rows, int b) { return (int)(row / rows) + b; }

// Workgroup -> place, key head and one of its `members` (heads of the group).  Workgroups are dealt round-robin to the 8 XCDs.
// The (place, key head)s go round them as well, with their members together: with a multiple of 8 key heads each head's keys and values are in one
// XCD's L2, and with any number all XCDs have tiles of the longest sequence.
struct TileUnit {
    unsigned place, head_kv, member;
};
FQ_BOTH TileUnit tile_unit(unsigned id, unsigned members, unsigned heads_kv)
{
    const unsigned at = id / 8, unit = at / members * 8 + id % 8, place = unit / heads_kv;
    return TileUnit{place, unit - place * heads_kv, at - at / members * members};
}
inline long long tile_workgroups(long long places, int members, int heads_kv) { return (places * heads_kv + 7) / 8 * 8 * members; }

// How fq_attn_cache deals out its work.  A workgroup takes a tile of columns (query token, head of the group; 16 * tiles of them) of one
// sequence and key head, and of its keys all or one of `splits` shares, `round` steps at a time: its waves take the steps of a round in turn, or (128
// columns, the kernel for many) each step together.
constexpr int MAX_SPLITS = 256, CACHE_CUS = 256, WIDE_COLUMNS = 128;
enum CacheOrder { CACHE_AS_GIVEN, CACHE_LONGEST_FIRST, CACHE_FOLDED };
struct CachePlan {
    int tiles, round, splits, order;      // order of the sequences
    long long places;                     // tiles of columns: of all sequences with many columns, else of one
};
inline CachePlan cache_plan(int batch, int tokens, int max_q, int max_len, int heads_q, int heads_kv)
{
    // Many columns go by tiles of 128 where there is much to compute, else by as many of 32 as they need, which are spread over more of the device.
    // us, tiles of 128 / of 32, 64 heads over 8: 32 columns, 64 sequences of 4096 121 / 105; 64 columns, one of 1000 14.5 / 12.1, 32 of 2048 46.4 / 35.9, three of
    // 40000 72 / 60, but 64 of 1024 41 / 44; 128 columns, one of 8192 27.5 / 19.1, 8 of 8192 58 / 55, three of 40000 91 / 123, 64 of 500 32 / 52; 320 columns, 100 of
    // 128 63 / 123; 1024 columns, one of 4096 39 / 31.
    const long long pairs = (long long)batch * heads_kv, columns = (long long)max_q * (heads_q / heads_kv), by32 = (columns + 31) / 32;
    const bool wide = columns > 32 && (pairs * by32 > 3 * CACHE_CUS || (columns > 64 && columns * pairs > (1LL << 25) / max_len));
    const int tiles = columns <= 16 ? 1 : wide ? WIDE_COLUMNS / 16 : 2;
    const long long places = wide ? tile_places((long long)tokens * (heads_q / heads_kv), batch, columns, WIDE_COLUMNS) : by32;
    const long long wgs = std::max(wide ? places * heads_kv : pairs * places, 1LL);
    // Four waves; two where a CU has one workgroup, of one tile of columns, and the longest share is long: fewer streams a CU then
    // read the cache faster.  us, two / four, 64 heads over 8: two sequences of 131072 tokens 97.5 / 99.8, 8 of 16384 44.5 / 48.0, 32 of 4096 41.5 / 44.1; but one of
    // 16384 (shares of 512) 13.4 / 12.7, 20 of up to 1200 13.8 / 11.1, two column tiles of 8 x 32768 106 / 102.  (Eight: 1001 tokens 11.7 / 8.7, 8192 13.2 / 10.1.)
    const bool few = wgs <= CACHE_CUS;
    const int round = wide ? 1 : tiles == 1 && few && max_len / (CACHE_CUS / wgs) >= 2048 ? 2 : 4;
    const long long rounds = ((long long)max_len + CACHE_STEP * round - 1) / (CACHE_STEP * round);
    const long long splits = std::min({wide ? rounds / 4 : rounds, (wide ? 2 * CACHE_CUS : CACHE_CUS) / wgs, (long long)MAX_SPLITS});
    // One workgroup a CU where the keys are split (two: 8 x 2000 tokens 14.2 us, one 11.6; 24 x 1500 21.1, 16.1), two of many columns (512 behind 7680: one
    // 225 us, two 158, four 186), and no split into two rounds or fewer, whose join costs more (300 tokens 8.4 us, 6.9; 500 8.6, 7.2).
    // Ordering the sequences costs each workgroup about 0.3 us, too much for short ones.
    const int order = wide || batch == 1 || batch > 64 || few || max_len < 1024 ? CACHE_AS_GIVEN : wgs <= 2 * CACHE_CUS ? CACHE_FOLDED : CACHE_LONGEST_FIRST;
    return CachePlan{tiles, round, rounds > 2 && splits > 1 ? (int)splits : 1, order, places};
}

// Whether the launches hold it.  (The kernel for many columns has all its workgroups along x.  The join has a sequence's query tokens along y: no more
// than there are tokens, 32768 at most where there are shares to join.)
inline bool cache_holds(const CachePlan& p, int heads_kv)
{
    const long long along_x = p.tiles > 2 ? tile_workgroups(p.places, p.splits, heads_kv) : p.splits;
    return along_x * 512 < (1LL << 32);
}

// Keys of one share when `keys` are dealt over `splits` workgroups: whole rounds, so that the last shares may be empty.
FQ_BOTH int share_keys(int keys, int splits, int round)
{
    const unsigned step = CACHE_STEP * round, rounds = ((unsigned)keys + step * splits - 1) / (step * splits);
    return (int)(rounds < 1 ? step : rounds * step);
}
FQ_BOTH int shares_used(int keys, int share) { return (int)(((unsigned)keys + share - 1) / share); }

// Queries of one head that a workgroup of the prompt's attention takes, 32 a wave.
constexpr int PROMPT_WAVES = 4, PROMPT_ROWS = 32 * PROMPT_WAVES, PROMPT_THREADS = 64 * PROMPT_WAVES;
inline long long prompt_workgroups(int tokens, int batch, int max_q, int heads_q, int heads_kv)
{
    return tile_workgroups(tile_places(tokens, batch, max_q, PROMPT_ROWS), heads_q / heads_kv, heads_kv);
}

}  // namespace fq
