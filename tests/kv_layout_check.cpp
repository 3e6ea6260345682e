// Replays csrc/mx_kv_layout.h on the host: every byte of a cache array has one owner, requests stay inside their tensors whatever
// the index arrays hold, rows see the keys of the definition, and the pieces of a batch cover every tile of keys once and fit the grid.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "mx_kv_layout.h"

using namespace mx;

static int failures = 0;
#define CHECK(cond, ...) do { if (!(cond)) { if (++failures < 20) { printf("FAIL %s: ", #cond); printf(__VA_ARGS__); printf("\n"); } } } while (0)

static void layout(int shift, int heads, int D, int pages) {
    const KvLayout at = {shift, heads, D};
    const int64_t places = (int64_t)pages << shift, words = (D + 127) / 128;
    std::vector<int> k(places * heads * D / 2), v(k.size()), s(places * heads * D / 32), w(places * heads * words);
    auto hit = [](std::vector<int>& a, int64_t at, int n) {
        for (int i = 0; i < n; ++i) {
            CHECK(at + i >= 0 && at + i < (int64_t)a.size(), "byte %lld of %zu", (long long)(at + i), a.size());
            if (at + i >= 0 && at + i < (int64_t)a.size()) ++a[at + i];
        }
    };
    for (int page = 0; page < pages; ++page)
        for (int head = 0; head < heads; ++head)
            for (int place = 0; place < 1 << shift; ++place) {
                for (int b = 0; b < D / 32; ++b) {
                    hit(k, at.k_block(page, head, b, place), 16);
                    hit(s, at.scale(page, head, b, place), 1);
                    CHECK(at.k_block(page, head, b, place) % 16 == 0, "block");
                }
                for (int u = 0; u < D / 8; ++u) hit(v, at.v_unit(page, head, u, place), 4);
                for (int x = 0; x < words; ++x) hit(w, at.word(page, head, x, place), 1);
                // neighbours that one load takes: 4 tokens of a unit and of a block's scales
                if (place % 4 == 0) {
                    CHECK(at.v_unit(page, head, 0, place) % 16 == 0 && at.v_unit(page, head, 1, place) == at.v_unit(page, head, 0, place) + 16, "unit");
                    CHECK(at.scale(page, head, 0, place) % 4 == 0, "scales");
                }
            }
    for (const auto* a : {&k, &v, &s, &w})
        for (int n : *a) CHECK(n == 1, "a byte has %d owners (page %d heads %d D %d)", n, 1 << shift, heads, D);
}

static void request(int64_t begin, int64_t end, int64_t len, int32_t T, int32_t room, int32_t window, int causal, bool sane) {
    const KvRequest r = KvRequest::make(begin, end, len, T, room);
    CHECK(r.first >= 0 && r.rows >= 0 && (int64_t)r.first + r.rows <= T, "rows %d + %d of %d", r.first, r.rows, T);
    CHECK(r.keys >= 0 && r.keys <= room, "keys");
    const int32_t some[] = {0, 1, r.rows / 2, r.rows - 1};
    for (int32_t i : some) {
        if (i < 0 || i >= r.rows) continue;
        const int32_t lo = r.lo(i, window), hi = r.hi(i, causal);
        CHECK(lo >= 0 && hi >= 0 && hi <= r.keys, "lo %d hi %d keys %d", lo, hi, r.keys);
        if (i) CHECK(r.lo(i - 1, window) <= lo && r.hi(i - 1, causal) <= hi, "limits grow with the row");
        if (sane) {
            const int64_t p = len - (end - begin) + (r.first + i - begin);
            for (int64_t j = 0; j < room + 3; ++j) {
                bool sees = j < len && j < room;
                if (causal) sees = sees && j <= p && (!window || j > p - window);
                CHECK(sees == (j >= lo && j < hi), "row %d key %lld: begin %lld end %lld len %lld T %d room %d window %d", i, (long long)j, (long long)begin,
                      (long long)end, (long long)len, T, room, window);
            }
        }
        if (lo < hi) {
            CHECK(r.first_tile(window) <= lo / kKvTile, "first tile");
            CHECK(r.first_tile(window) + r.tiles(window, causal) >= (hi + kKvTile - 1) / kKvTile, "tiles");
        }
    }
}

static void batch(std::mt19937& rng) {
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    const int S = pick(1, 40), group = pick(1, 9), heads = pick(1, 8), height = 16 * pick(1, 8), window = pick(0, 1) * pick(1, 3000), least = pick(1, 8);
    const int log2 = pick(0, 11), workers = 1 << log2;
    const int64_t far = log2 < 6 || pick(0, 3) ? 0 : (int64_t)pick(1, 9) << 31;  // (positions beyond 32 bits are reached with one long request in front)
    int64_t begin = 0, total = far;
    struct Item { int64_t at; int32_t tiles; };
    std::vector<Item> items;
    for (int s = 0; s < S; ++s) {
        const int n = pick(0, pick(0, 1) ? 1 : 200), len = pick(0, pick(0, 1) ? 20 : 40000);
        const KvRequest r = KvRequest::make(begin, begin + n, len, 1 << 20, 1 << 20);
        begin += n;
        const int32_t tiles = r.tiles(window, 1), row_tiles = r.row_tiles(group, height);
        CHECK((int64_t)row_tiles * height >= (int64_t)r.rows * group && (int64_t)(row_tiles - 1) * height < (int64_t)r.rows * group, "row tiles");
        for (int i = 0; i < row_tiles * heads; ++i) items.push_back({total + (int64_t)i * KvLine::item(tiles), KvLine::item(tiles)});
        total += KvLine::request(tiles, row_tiles, heads);
    }
    const int32_t share = KvLine::share(total, log2, least);
    CHECK((int64_t)share * workers >= total && share >= least, "the groups take all");
    std::vector<int> used(2 * workers), taken(items.size());
    size_t item = 0;
    for (int w = 0; w < workers; ++w) {  // as the workers go along the line
        const int64_t first = (int64_t)share * w, end = std::min(total, first + share);
        for (int64_t at = std::max(far, std::min(total, first)); at < end;) {
            while (item < items.size() && items[item].at + items[item].tiles <= at) ++item;
            const Item& x = items[item];
            const int64_t stop = std::min(end, x.at + x.tiles);
            const KvLine::Parts parts = KvLine::parts(x.at, x.tiles, share);
            CHECK(at == std::max(x.at, first) && w >= parts.first && w < parts.first + parts.count, "worker %d of %d + %d", w, parts.first, parts.count);
            const bool whole = KvLine::whole(x.at, x.tiles, first, first + share);
            CHECK(whole == (parts.count == 1) && whole == (at == x.at && stop == x.at + x.tiles), "whole or not");
            if (!whole) {
                const int32_t place = KvLine::place(x.at, first, w);
                CHECK(place == 2 * w + (w == parts.first ? parts.late : 0), "place %d", place);
                CHECK(place >= 0 && place < 2 * workers, "place %d", place);
                if (place >= 0 && place < 2 * workers) CHECK(++used[place] == 1, "place %d used twice", place);
            }
            // the tiles of an item go to its workers in order, none twice
            CHECK(KvLine::tiles_before((int32_t)(at - x.at)) == taken[item], "tiles");
            taken[item] = KvLine::tiles_before((int32_t)(stop - x.at));
            at = stop;
        }
    }
    for (size_t i = 0; i < items.size(); ++i) CHECK(taken[i] == items[i].tiles - KvLine::kItemCost, "all tiles of item %zu", i);
}

int main() {
    for (int D : {64, 96, 128, 192, 256})
        for (int shift : {4, 5, 7}) layout(shift, 3, D, 2);
    std::mt19937 rng(1);
    auto near = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    for (int i = 0; i < 20000; ++i) {
        const int32_t T = (int32_t)near(1, 40), room = (int32_t)near(0, 12) * 16;
        const int64_t begin = near(0, T), end = near(begin, T + 3), len = near(0, room + 20);
        const int causal = near(0, 3) != 0;
        request(begin, end, len, T, room, causal ? (int32_t)(near(0, 1) * near(1, 50)) : 0, causal, true);
    }
    const int64_t wild[] = {INT64_MIN, INT64_MIN + 1, -(1ll << 40), INT32_MIN, -5, -1, 0, 1, 7, 1000, 1 << 30, INT32_MAX, 1ll << 40, INT64_MAX - 1, INT64_MAX};
    for (int64_t begin : wild)
        for (int64_t end : wild)
            for (int64_t len : wild)
                for (int32_t T : {1, 1000, 1 << 30})
                    for (int32_t room : {0, 16, 1 << 30})
                        for (int32_t window : {0, 1, 100, 1 << 30}) request(begin, end, len < INT32_MIN || len > INT32_MAX ? 5 : len, T, room, window, window || (begin & 1), false);
    for (int i = 0; i < 2000; ++i) batch(rng);
    for (int tiles = 0; tiles < 300; ++tiles)
        for (int most = 1; most <= 64; ++most) {
            const int pieces = kv_pieces(tiles, most);
            CHECK(pieces >= 1 && pieces <= most && kv_piece_begin(tiles, pieces, 0) == 0 && kv_piece_begin(tiles, pieces, pieces) == tiles, "pieces");
            for (int i = 0; i < pieces && pieces > 1; ++i) CHECK(kv_piece_begin(tiles, pieces, i + 1) - kv_piece_begin(tiles, pieces, i) >= 4, "a short piece");
        }
    printf(failures ? "%d failures\n" : "layout, requests and pieces hold\n", failures);
    return failures != 0;
}
