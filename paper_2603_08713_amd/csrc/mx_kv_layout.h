// Where a row of the paged MXFP4 cache lies, and which pieces of work a batch of requests is cut into (plain C++ on integers: the
// kernels use it, and a host test replays it).
//
// A page holds page_size tokens (a power of two from 16) of every head.  Everything is block-major, so that the 16 tokens that
// one matrix instruction takes lie next to each other:
//   K codes  [page][head][D/32][place][16]         a lane of the product Q K^T wants 32 codes of one token: 16 bytes
//   V codes  [page][head][place/4][D/8][4][4]      a lane of the product P V wants 8 codes of each of 4 neighbouring tokens: 16 bytes
//   scales   [page][head][D/32][place], MBS words [page][head][ceil(D/128)][place]
// A wavefront's load of 16 tokens then covers whole 256-byte pieces (K) or one 1 KiB piece (V) for heads of 128.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define MX_HD __host__ __device__ __forceinline__
#else
#define MX_HD inline
#endif

namespace mx {

struct KvLayout {
    int32_t page_shift;  // page_size = 1 << page_shift
    int32_t heads;       // of keys and values
    int32_t D;
    MX_HD int32_t page_size() const { return 1 << page_shift; }
    MX_HD int32_t blocks() const { return D >> 5; }
    MX_HD int32_t words() const { return (D + 127) >> 7; }
    // bytes from the start of the array; block, unit (8 codes), word: which of the row's
    MX_HD int64_t k_block(int64_t page, int32_t head, int32_t block, int32_t place) const {
        return ((((page * heads + head) * blocks() + block) << page_shift) + place) * 16;
    }
    MX_HD int64_t v_unit(int64_t page, int32_t head, int32_t unit, int32_t place) const {
        return (((page * heads + head) << (page_shift - 2)) + (place >> 2)) * (2 * (int64_t)D) + unit * 16 + (place & 3) * 4;
    }
    MX_HD int64_t scale(int64_t page, int32_t head, int32_t block, int32_t place) const {
        return (((page * heads + head) * blocks() + block) << page_shift) + place;
    }
    MX_HD int64_t word(int64_t page, int32_t head, int32_t word, int32_t place) const {
        return (((page * heads + head) * words() + word) << page_shift) + place;
    }
};

MX_HD int32_t kv_min(int32_t a, int32_t b) { return a < b ? a : b; }
MX_HD int32_t kv_max(int32_t a, int32_t b) { return a > b ? a : b; }
MX_HD int32_t kv_clamp(int64_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : (int32_t)x; }

constexpr int32_t kKvTile = 64;                 // keys that a wavefront takes at a time
constexpr int32_t kKvMostKeys = (int32_t)1 << 30;  // of a request; positions are clamped to +- this

// One request of a batch, with whatever the arrays say made safe: rows outside [0, T) and keys beyond the table do not exist.
struct KvRequest {
    int32_t first;  // its first query row that exists
    int32_t rows;   // how many of them (query tokens)
    int32_t pos0;   // position of the first one among the keys (negative: it sees none under the causal rule)
    int32_t keys;   // keys that exist

    // begin, end: row_offsets[s], row_offsets[s+1]; len: kv_lens[s]; T: rows of the query tensor; room: keys that the table has room for
    MX_HD static KvRequest make(int64_t begin, int64_t end, int64_t len, int32_t T, int32_t room) {
        constexpr int64_t kFar = (int64_t)1 << 40;  // beyond any tensor: sums of what is below cannot overflow
        begin = begin < 0 ? 0 : begin > kFar ? kFar : begin;
        end = end < begin ? begin : end > kFar ? kFar : end;
        KvRequest r;
        r.first = kv_clamp(begin, 0, T);
        r.rows = kv_clamp(end, r.first, T) - r.first;
        // (the last row stands on the last key, also where rows are cut off)
        r.pos0 = kv_clamp(len - (end - begin), -kKvMostKeys, kKvMostKeys);
        r.keys = kv_clamp(len, 0, room);
        return r;
    }
    // keys [lo, hi) that query row i sees
    MX_HD int32_t hi(int32_t i, int causal) const { return causal ? kv_max(0, kv_min(keys, kv_min(pos0 + i, kKvMostKeys) + 1)) : keys; }
    MX_HD int32_t lo(int32_t i, int32_t window) const { return window ? kv_max(0, kv_min(pos0 + i, kKvMostKeys) - (window - 1)) : 0; }
    // first tile and number of tiles that any of its rows sees
    MX_HD int32_t first_tile(int32_t window) const { return lo(0, window) / kKvTile; }
    MX_HD int32_t tiles(int32_t window, int causal) const {
        const int32_t end = (hi(rows - 1, causal) + kKvTile - 1) / kKvTile;
        return rows > 0 ? kv_max(0, end - first_tile(window)) : 0;
    }
    // tiles of `height` rows that its rows times the query heads of one key head make
    MX_HD int32_t row_tiles(int32_t group, int32_t height) const { return (int32_t)(((int64_t)rows * group + height - 1) / height); }
};

// The work of a batch in one line: request after request, of each its items (key heads x row tiles), of each a fixed length that stands for
// what an item costs besides (and lets rows without keys be written too) and then its tiles of keys.  A worker takes `share` of that
// line, from share * its number on; an item that it does not take whole leaves a partial result, of which a worker has two places:
// one for the item that it begins with, one for an item that it only begins.
struct KvLine {
    static constexpr int32_t kItemCost = 2;  // in tiles
    // length of an item, and how many of its tiles lie before a place in it
    MX_HD static int32_t item(int32_t tiles) { return tiles + kItemCost; }
    MX_HD static int32_t tiles_before(int32_t place) { return kv_max(place - kItemCost, 0); }
    // length of a request
    MX_HD static int64_t request(int32_t tiles, int32_t row_tiles, int32_t heads) { return (int64_t)item(tiles) * row_tiles * heads; }
    MX_HD static int32_t share(int64_t total, int32_t workers_log2, int32_t least) {
        return kv_clamp((total + ((int64_t)1 << workers_log2) - 1) >> workers_log2, least, INT32_MAX);
    }
    // for the worker whose share is [begin, end): whether it takes all of the item at [at, at + item), and where its part of it goes if not
    MX_HD static bool whole(int64_t at, int32_t item, int64_t begin, int64_t end) { return at >= begin && at + item <= end; }
    MX_HD static int32_t place(int64_t at, int64_t begin, int32_t worker) { return 2 * worker + (at > begin); }
    // the same from the item's side: its parts are those of the workers first, first + 1, .. (count of them; 1: it is whole), the part of
    // the first in place 2 first + late, of another w in place 2 w
    struct Parts {
        int32_t first, count, late;
    };
    MX_HD static Parts parts(int64_t at, int32_t item, int32_t share) {
        Parts p;
        if ((at + item) >> 32) {  // (a division of 64 bits is some hundred instructions)
            p.first = (int32_t)(at / share);
            p.count = (int32_t)((at + item - 1) / share) - p.first + 1;
        } else {
            p.first = (int32_t)((uint32_t)at / (uint32_t)share);
            p.count = (int32_t)((uint32_t)(at + item - 1) / (uint32_t)share) - p.first + 1;
        }
        p.late = at > (int64_t)p.first * share;
        return p;
    }
};

// Pieces that the keys of a row tile (of many rows) are cut into, `tiles` of them: at most `most`, of four tiles at least; and where piece i
// begins.
MX_HD int32_t kv_pieces(int32_t tiles, int32_t most) { return kv_max(1, kv_min(most, tiles / 4)); }
MX_HD int32_t kv_piece_begin(int32_t tiles, int32_t pieces, int32_t i) { return (int32_t)((int64_t)tiles * i / pieces); }

}  // namespace mx
