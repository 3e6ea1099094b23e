// Host test of the arithmetic that the paged cache's kernels place their work by (test infrastructure): the functions are
// the ones the kernels call, compiled for the host, with every access checked against its array.  Built and run by
// tests/test_paged_host.py.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "paged_internal.h"

using namespace buzz;

#define CHECK(x) do { if (!(x)) { fprintf(stderr, "paged_schedule: line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

// Every key that the new token sees lies in exactly one tile, no tile is empty of such keys, tiles are inside the sequence.
static void check_tiles(int length, int sink, int window, int tile, int64_t most)
{
    const Visible v = visible(length, sink, window, most);
    if (length < 0 || length > most) { CHECK(v.length < 0); CHECK(tiles_of(v, tile).count == 0); return; }
    const Tiles t = tiles_of(v, tile);
    std::set<int> seen;
    for (int i = 0; i < t.count; ++i) {
        const int at = t.at(i) * tile;
        CHECK(at >= 0 && at < length && seen.insert(at).second);
        bool any = false;
        for (int j = at; j < at + tile; ++j) any |= v.sees(j);
        CHECK(any);
    }
    for (int j = 0; j < length + tile; ++j) {
        const bool want = j < length && (window == 0 || j >= length - window || j < sink);
        CHECK(v.sees(j) == want);
        for (int n : {4, 8, 16}) CHECK(((v.bits(j / n * n, n) >> (j % n)) & 1) == (uint32_t)want);
        if (want) CHECK(seen.count(j / tile * tile));
    }
    if (length == 0) CHECK(t.count == 0);
}

// The walk of the decode kernel's blocks over all units: each unit once, each pair's partial results in slots of their own
// within the workspace, as many arrivals as the merging block waits for.
static void check_share(const std::vector<int>& n, int heads, unsigned blocks)
{
    uint64_t total = 0;
    for (int x : n) total += (uint64_t)(x > 0 ? x : 1) * heads;
    const uint64_t share = units_per_block((uint32_t)total, blocks);
    std::vector<std::map<int64_t, int>> slots(n.size() * heads);     // pair -> slot -> units
    std::vector<int> done(n.size() * heads, 0), alone(n.size() * heads, 0);
    std::set<int64_t> used;
    CHECK(share * blocks >= total);
    for (unsigned block = 0; block < blocks; ++block) {
        uint64_t cur = share * block;
        if (cur >= total) continue;
        const uint64_t end = cur + share < total ? cur + share : total;
        uint64_t off = cur;
        size_t b = 0;
        auto in_sequence = [&](size_t i) { return (uint64_t)(n[i] > 0 ? n[i] : 1) * heads; };
        for (; off >= in_sequence(b); ++b) off -= in_sequence(b);
        while (cur < end) {
            const uint64_t m = n[b] > 0 ? n[b] : 1;
            const size_t pair = b * heads + off / m;
            const uint64_t first = off % m, here = m - first < end - cur ? m - first : end - cur;
            done[pair] += (int)here;
            if (first == 0 && here == m) {
                alone[pair] = 1;
            } else {
                const int64_t slot = 2 * (int64_t)block + (first == 0 ? 1 : 0);
                CHECK(slot < 2 * kPagedMaxBlocks && used.insert(slot).second);
                slots[pair][slot] = (int)here;
                const Parts p = parts_of((uint32_t)(cur - first), (uint32_t)m, (uint32_t)share);
                bool mine = false;
                for (int i = 0; i < p.parts; ++i) mine |= p.slot(i) == slot;
                CHECK(mine);
                // the merging block's list is the list of all slots that get written for the pair
                for (int i = 0; i < p.parts; ++i) slots[pair].insert({p.slot(i), 0});
                CHECK((int)slots[pair].size() == p.parts);
            }
            cur += here;
            off += here;
            if (off == m * heads) { off = 0; ++b; }
        }
    }
    // groups of partial results: every part in one, whose slot is one of the pair's own
    uint64_t begin = 0;
    for (size_t pair = 0; pair < done.size(); ++pair) {
        const uint64_t m = n[pair / heads] > 0 ? n[pair / heads] : 1;
        const Parts all = parts_of((uint32_t)begin, (uint32_t)m, (uint32_t)share);
        begin += m;
        if (slots[pair].empty()) continue;
        const int group = group_of(all.parts), groups = (all.parts + group - 1) / group;
        CHECK(group <= 32 && groups <= 16 && (groups - 1) * group < all.parts && (group > 1 || groups == all.parts));
        for (int i = 0; i < all.parts; ++i) {
            CHECK(i / group < groups && slots[pair].count(all.slot(i / group * group)));
            CHECK(all.slot(i) >= 0 && all.slot(i) < 2 * kPagedMaxBlocks);
        }
    }
    for (size_t pair = 0; pair < done.size(); ++pair) {
        CHECK(done[pair] == (n[pair / heads] > 0 ? n[pair / heads] : 1));
        CHECK(alone[pair] == (slots[pair].empty() ? 1 : 0));
        for (auto& s : slots[pair]) CHECK(s.second > 0);
    }
}

int main()
{
    std::mt19937 rng(7);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
    for (int tile : {16, 32, 64})
        for (int i = 0; i < 3000; ++i)
            check_tiles(upto(700) - 2, i % 3 ? upto(90) : 0, i % 2 ? upto(300) : 0, tile, 690);
    check_tiles(0, 4, 8, 32, 64);
    check_tiles(1, 0, 1, 32, 64);
    check_tiles(64, 64, 1, 32, 64);
    check_tiles(65, 0, 0, 32, 64);
    for (int i = 0; i < 400; ++i) {
        std::vector<int> n(1 + upto(i % 10 == 0 ? 300 : 12));
        for (int& x : n) x = upto(4) == 0 ? 0 : upto(i % 7 == 0 ? 4000 : 60);
        check_share(n, 1 + upto(9), 1 + upto(i % 2 ? 40 : kPagedMaxBlocks));
    }
    check_share({0}, 1, 1);
    check_share({1 << 22}, 1, kPagedMaxBlocks);
    check_share(std::vector<int>(511, 1 << 22), 1, kPagedMaxBlocks);         // 2^31 - 2^22 units
    CHECK(units_of(0, 4) == 1 && units_of(1, 4) == 1 && units_of(4, 4) == 1 && units_of(5, 4) == 2 && units_of(1 << 24, 1) == 1 << 24);
    CHECK(units_countable(511, 1, 1 << 20, 256) && !units_countable(512, 1, 1 << 20, 256) && !units_countable(65535, 65535, 1, 16));

    // rows of a call: spans, and the tiles of 16 positions that cover them
    for (int i = 0; i < 3000; ++i) {
        const int64_t n_rows = upto(200);
        const int32_t start = upto(300) - 20, count = upto(260) - 30;
        const Span s = row_span(i % 5 ? &start : nullptr, i % 3 ? &count : nullptr, 0, n_rows);
        const int64_t at = i % 5 ? start : 0;
        int64_t want = i % 3 ? count : n_rows;
        want = want < 0 ? 0 : want > n_rows ? n_rows : want;
        if (at < 0) { CHECK(s.lo >= s.hi); continue; }
        CHECK(s.start == at && s.lo == at && s.hi == at + want);
        std::set<int64_t> rows;
        for (int64_t x = 0; x < tiles_of_rows(n_rows); ++x) {
            const int64_t p0 = (s.start / kPagedTileTokens + x) * kPagedTileTokens;
            const int64_t lo = s.lo > p0 ? s.lo : p0, hi = s.hi < p0 + kPagedTileTokens ? s.hi : p0 + kPagedTileTokens;
            for (int64_t p = lo; p < hi; ++p) CHECK(p - s.start >= 0 && p - s.start < n_rows && rows.insert(p).second);
        }
        CHECK((int64_t)rows.size() == want);
    }
    {
        const int32_t start = INT32_MAX, count = 40;               // positions beyond 2^31 stay what they are
        const Span s = row_span(&start, &count, 0, 40);
        CHECK(s.lo == INT32_MAX && s.hi == (int64_t)INT32_MAX + 40);
    }
    CHECK(tiles_of_rows(0) == 0 && tiles_of_rows(1) == 1 && tiles_of_rows(2) == 2 && tiles_of_rows(17) == 2 && tiles_of_rows(18) == 3);

    // pages: numbers that are none of the pool's come back as -1, whatever they are
    const std::vector<int32_t> table = {3, 0, -1, 7, INT32_MAX, INT32_MIN, 6, 8};
    const std::vector<int32_t> want = {3, 0, -1, -1, -1, -1, 6, -1};
    for (size_t c = 0; c < table.size(); ++c)
        for (int row = 0; row < 32; ++row) CHECK(page_of(table.data(), (int64_t)c * 32 + row, 5, 7) == want[c]);
    printf("paged_schedule ok\n");
    return 0;
}
