// Sizes, pieces and workspaces of the calls from tokens to loss: plain host logic, apart from the launches so that a host program
// can check it (tests/token_plan_check.cpp).
#pragma once
#include <stddef.h>
#include <stdint.h>

#if defined(__HIPCC__)
#define ONECOMP_TOKEN_FN __host__ __device__ inline
#else
#define ONECOMP_TOKEN_FN inline
#endif

namespace onecomp {
namespace product {

// Workgroup -> tile.  Workgroup b runs on XCD b % 8; an XCD takes a run of ranks, which go through bands of BAND tiles of m
// column by column of n, so that the tiles at work at a time share operands in its L2.
constexpr int BAND = 8;
ONECOMP_TOKEN_FN bool tile_of(unsigned block, int m_tiles, int n_tiles, int& tm, int& tn) {
    const unsigned all = unsigned(m_tiles) * unsigned(n_tiles), run = (all + 7) / 8, rank = (block & 7) * run + (block >> 3);
    if ((block >> 3) >= run || rank >= all) return false;
    const unsigned band = rank / (BAND * unsigned(n_tiles)), rest = rank - band * BAND * unsigned(n_tiles);
    const unsigned left = unsigned(m_tiles) - band * BAND, high = left < BAND ? left : unsigned(BAND);
    tn = int(rest / high);
    tm = int(band * BAND + rest % high);
    return true;
}
// workgroups that reach every tile
inline int64_t tile_blocks(int64_t m_tiles, int64_t n_tiles) { return (m_tiles * n_tiles + 7) / 8 * 8; }

}  // namespace product
namespace token {

inline int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round_256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---- embedding gradient ----
// Vocabulary rows of a sorting workgroup: about one workgroup per compute unit, sixteen counters a row in LDS.
constexpr int SORT_WAVES = 16, SORT_MOST = 1024;
inline int sort_rows(int64_t vocab) {
    const int64_t r = ceil_of(ceil_of(vocab, 256), 64) * 64;
    return int(r > SORT_MOST ? SORT_MOST : r);
}
// Sorted tokens that a wave adds up.
inline int segment_of(int64_t tokens) { return tokens < 16384 ? 16 : 64; }

struct EmbeddingSpace {
    size_t order, starts, parts, all;   // offsets, and the whole size
    int64_t segments;
};
inline EmbeddingSpace embedding_space(int64_t tokens, int64_t vocab, int64_t width) {
    EmbeddingSpace s;
    s.segments = ceil_of(tokens, segment_of(tokens));
    s.order = 0;
    s.starts = s.order + round_256(size_t(tokens) * 4);
    s.parts = s.starts + round_256((size_t(vocab) + 1) * 4);
    s.all = s.parts + round_256(size_t(s.segments) * 2 * size_t(width) * 4);
    return s;
}

// ---- tiles of products ----
// Up to FEW rows of m are multiplied without tiles.
constexpr int64_t FEW = 64;
enum Tiles { BIG, MID, MID_SPLIT, HALF, HALF_SPLIT, SMALL, SMALL_SPLIT };
struct TileShape {
    int n, m, per_cu;
};
inline TileShape shape_of(Tiles t) {
    switch (t) {
        case BIG: return {256, 256, 1};
        case MID: return {128, 128, 2};
        case MID_SPLIT: return {128, 128, 1};
        case HALF: return {128, 64, 3};
        case HALF_SPLIT: return {128, 64, 1};
        case SMALL: return {64, 64, 4};
        default: return {64, 64, 1};
    }
}
inline int64_t tiles_of(Tiles t, int64_t m, int64_t n) { return ceil_of(m, shape_of(t).m) * ceil_of(n, shape_of(t).n); }
// The largest tiles that are many enough for the chip.
inline Tiles choose_tiles(int64_t m, int64_t n) {
    if (tiles_of(BIG, m, n) >= 192) return BIG;
    if (tiles_of(MID, m, n) > 256) return MID;
    if (tiles_of(MID, m, n) > 192) return MID_SPLIT;
    if (tiles_of(HALF, m, n) > 256) return HALF;
    if (tiles_of(HALF, m, n) > 192) return HALF_SPLIT;
    return tiles_of(SMALL, m, n) > 256 ? SMALL : SMALL_SPLIT;
}

// ---- loss ----
// Columns of the vocabulary that leave one maximum and sum per token.
inline int64_t part_columns(int64_t tokens, int64_t vocab) { return tokens <= FEW ? 32 : shape_of(choose_tiles(tokens, vocab)).n; }
// Gradients of logits are formed for a piece of the vocabulary at a time, a multiple of 256 columns: 1 GB of them.
constexpr int64_t PIECE_BYTES = int64_t(1) << 30;
inline int64_t piece_columns(int64_t tokens, int64_t vocab, int esz) {
    const int64_t rows = ceil_of(tokens < 1 ? 1 : tokens, 256) * 256, all = ceil_of(vocab, 256) * 256;
    int64_t c = PIECE_BYTES / (rows * esz) / 256 * 256;
    if (c < 2048) c = 2048;
    if (c >= all) return all;
    return ceil_of(ceil_of(all, ceil_of(all, c)), 256) * 256;   // pieces of about one size
}
// Shares of the inner sum of dh (over a piece's columns): room for up to 16 of them, in 1 GB.
inline int64_t most_shares(int64_t tokens, int64_t width) {
    const int64_t s = (int64_t(1) << 30) / ((tokens < 1 ? 1 : tokens) * width * 4);
    return s < 1 ? 1 : s > 16 ? 16 : s;
}
// How many are taken, from the number of kept tokens: the fewest rounds of the chip's `slots` tiles, by the columns that a
// workgroup goes through one after the other and 256 for the beginning and end of each tile.
ONECOMP_TOKEN_FN int shares_of(int tiles, int columns, int slots, int most) {
    int best = 1;
    uint64_t least = 0;
    for (int s = 1; s <= most; ++s) {
        const unsigned rounds = (unsigned(tiles) * unsigned(s) + unsigned(slots) - 1) / unsigned(slots);
        const uint64_t cost = uint64_t(rounds) * ((unsigned(columns) + unsigned(s) - 1) / unsigned(s) + 256u);
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

inline int64_t round_up(int64_t x, int64_t to) { return ceil_of(x, to) * to; }

struct LossSpace {
    size_t index, place, count, coef, rows, parts, hit, piece, dh, all;
    int64_t columns, shares;
};
// Rows in panels.
inline size_t panel_bytes(int64_t rows, int64_t width, int esz) { return size_t(rows) * size_t(round_up(width * esz, 64)); }
// n_parts: tiles of the vocabulary that leave a maximum and a sum per token
inline LossSpace loss_space(int64_t tokens, int64_t width, int64_t vocab, int esz, int64_t n_parts, bool gradient) {
    LossSpace s{};
    const size_t t = size_t(tokens);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_256(bytes);
        return here;
    };
    s.count = take(4);
    s.index = take(t * 4);
    s.place = take(gradient ? t * 4 : 0);
    s.coef = take(t * (gradient ? 16 : 4));
    s.rows = take(panel_bytes(tokens, width, esz));
    s.parts = take(gradient ? 0 : t * size_t(n_parts) * 8);
    s.hit = take(gradient ? 0 : t * 4);
    if (gradient) {
        s.columns = piece_columns(tokens, vocab, esz);
        s.shares = most_shares(tokens, width);
        s.piece = take(panel_bytes(tokens, s.columns, esz));
        s.dh = take(t * size_t(width) * 4 * size_t(s.shares));
    }
    s.all = at;
    return s;
}

}  // namespace token
}  // namespace onecomp
