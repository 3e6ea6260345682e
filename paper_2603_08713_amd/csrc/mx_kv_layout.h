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

// Pieces of a request along its keys, `share` tiles each; one at least, so that rows without keys are written too.
MX_HD int32_t kv_pieces(int32_t tiles, int32_t share) { return tiles <= share ? 1 : (tiles + share - 1) / share; }
// The share that cuts `total` tiles (of all requests, heads and row tiles) into about `target` pieces.
MX_HD int32_t kv_share(int64_t total, int32_t target, int32_t least) {
    const int64_t s = (total + target - 1) / target;
    return s < least ? least : kv_clamp(s, 1, kKvMostKeys / kKvTile);
}

}  // namespace mx
