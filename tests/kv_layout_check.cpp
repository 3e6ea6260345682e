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
    const int target = pick(1, 1) * 1024;
    std::vector<int64_t> offsets = {0};
    std::vector<int> lens;
    for (int s = 0; s < S; ++s) {
        offsets.push_back(offsets.back() + pick(0, pick(0, 1) ? 1 : 200));
        lens.push_back(pick(0, pick(0, 1) ? 20 : 40000));
    }
    const int32_t T = (int32_t)offsets.back();
    int64_t total = 0, row_tiles = 0;
    std::vector<KvRequest> r;
    for (int s = 0; s < S; ++s) {
        r.push_back(KvRequest::make(offsets[s], offsets[s + 1], lens[s], T, 1 << 20));
        total += (int64_t)r[s].row_tiles(group, height) * r[s].tiles(window, 1);
        row_tiles += r[s].row_tiles(group, height);
    }
    CHECK(row_tiles <= S + ((int64_t)T * group + height - 1) / height, "row tiles");
    const int32_t share = kv_share(total * heads, target, least);
    int64_t units = 0;
    for (int s = 0; s < S; ++s) {
        const int32_t tiles = r[s].tiles(window, 1), pieces = kv_pieces(tiles, share);
        CHECK(pieces >= 1 && (int64_t)pieces * share >= tiles && (int64_t)(pieces - 1) * share < (tiles ? tiles : 1), "pieces");
        units += (int64_t)r[s].row_tiles(group, height) * pieces;
    }
    CHECK(units * heads <= target + (S + ((int64_t)T * group + height - 1) / height) * heads, "the grid holds %lld units", (long long)units);
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
    printf(failures ? "%d failures\n" : "layout, requests and pieces hold\n", failures);
    return failures != 0;
}
