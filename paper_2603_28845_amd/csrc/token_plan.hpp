// Sizes, pieces and workspaces of the calls from tokens to loss: plain host logic, apart from the launches so that a host program
// can check it (tests/token_plan_check.cpp).
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <initializer_list>

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
// A launch has less than 2^32 threads along x: tiles of 64 x 64 with 256 threads, the smallest, have room for m x n results.
inline bool product_fits(int64_t m, int64_t n) { return (m + 63) / 64 * ((n + 63) / 64) < int64_t(1) << 24; }
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
// A token's row among the `rows` from lo on, or -1, for tokens of any 32 bits.
ONECOMP_TOKEN_FN int row_of(int32_t token, int lo, int rows) { return token >= lo && token - lo < rows ? token - lo : -1; }
// Sorted tokens that a wave adds up: more where there is enough to read that fewer waves still fill the chip, since each segment
// may leave two partial sums to be joined.  us in segments of 16 : 32 : 64, tokens x width: 1392 x 80 17.9 : 23.2 : 34.6;
// 8000 x 2048 38.7 : 36.1 : 43.9; 25915 x 144 32.3 : 34.6 : 44.2; 23215 x 891 fp32 53.5 : 50.6 : 52.0; 65536 x 512 88.9 : 76.7 : 74.5;
// 16384 x 4096 254 : 247 : 242; 45583 x 6336 131 : 118 : 113.
inline int segment_of(int64_t tokens, int64_t width) {
    if (tokens < 16384) return 16;
    return tokens * width < int64_t(1) << 25 ? 32 : 64;
}

struct EmbeddingSpace {
    size_t order, starts, parts, all;   // offsets, and the whole size
    int64_t segments;
};
inline EmbeddingSpace embedding_space(int64_t tokens, int64_t vocab, int64_t width) {
    EmbeddingSpace s;
    s.segments = ceil_of(tokens, segment_of(tokens, width));
    s.order = 0;
    s.starts = s.order + round_256(size_t(tokens) * 4);
    s.parts = s.starts + round_256((size_t(vocab) + 1) * 4);
    s.all = s.parts + round_256(size_t(s.segments) * 2 * size_t(width) * 4);
    return s;
}

// ---- tiles of products ----
// Whether m rows are multiplied without tiles, straight from memory: up to 64, the fewer the more n there are, since tiles of enough n
// fill the chip and read the rows once for 64 to 256 of n instead of 16 or 32.  esz: bytes of an element; 1: the 8-bit layers.
// us without tiles : with them.  bf16, k 4096: 16 x 4000 19 : 27, 32 x 8000 28 : 33, 48 x 4000 30 : 30, 64 x 1000 30 : 24, 16 x 32000 64 : 71, 24 x 12000
// 43 : 34, 16 x 64000 114 : 114, 16 x 128000 215 : 186, 1 x 128000 193 : 201; k 512: 48 x 4000 11 : 12, 16 x 64000 28 : 25, 1 x 200000 60 : 48.  fp32,
// k 4096: 64 x 8000 65 : 79, 48 x 12000 108 : 82, 32 x 12000 81 : 82, 32 x 32000 172 : 152, 16 x 128000 435 : 567; k 512: 32 x 16000 19 : 21, 24 x 64000
// 59 : 48.  8 bits: 64 x 4096, k 14336 40 : 46, k 4096 12.6 : 12.2; k 4096, 32 x 8192 15.0 : 15.1, 48 x 8192 21 : 16, 16 x 14336 17.2 : 19.4.  The bounds
// lie where both are about equal; close to them either is faster by up to a tenth, after k.
inline bool few_rows(int64_t m, int64_t n, int esz) {
    if (esz == 1) return m <= (n <= 4096 ? 64 : n <= 8192 ? 32 : 16);
    if (esz == 2) return m <= (n <= 8192 ? 32 : n <= 65536 ? 16 : 0);
    return m <= (n <= 8192 ? 64 : n <= 16384 ? 32 : 16);
}
enum Tiles { BIG, MID, HALF, SMALL, SMALL_SPLIT };
// fixed, step: ns that a compute unit takes for a tile's beginning and end and for 64 bytes of k, all units at work (several small
// tiles overlap, so that they cost less than one alone): logits of 8192 tokens over 32000 entries, widths 64 to 4096, bf16 and
// fp32.  8-bit layers go by bf16, which puts the shapes in about the right order but is no time of theirs: 1999 x 777, k 2000 would
// take 6.7 us and takes 16.
struct TileShape {
    int n, m, fixed, step;
};
inline TileShape shape_of(Tiles t, bool f32) {
    switch (t) {
        case BIG: return {256, 256, 7100, f32 ? 3740 : 770};
        case MID: return {128, 128, 1600, f32 ? 933 : 255};
        case HALF: return {128, 64, 800, f32 ? 473 : 185};
        default: return {64, 64, 500, f32 ? 244 : 125};
    }
}
// what the fullest compute unit takes for `tiles` of a shape
ONECOMP_TOKEN_FN uint64_t tile_cost(unsigned tiles, unsigned steps, unsigned fixed, unsigned step) {
    return uint64_t((tiles + 255u) / 256u) * (fixed + uint64_t(steps) * step);
}
inline unsigned tiles_of(const TileShape& t, int64_t m, int64_t n) { return unsigned(ceil_of(m, t.m) * ceil_of(n, t.n)); }
// Tiles for m x n results of `steps` times 64 bytes of k: from the largest on, the next smaller shape as long as its cost is at most a
// twentieth above that of the last one taken.  us, chosen : largest tiles : smallest: 512 x 8000, k 4096 bf16 46 : 87 : 74; 2048 x 8000 122 : 122 : 244;
// 128 x 32000, k 1024 fp32 83 : 256 : 83; 512 x 32000, k 64 bf16 18 : 20 : 22.  Chosen : the least cost: logits (within a twentieth of it) 884 x 149623,
// k 544 fp32 1135 : 1092, 1745 x 8049, k 112 bf16 21.0 : 20.2; the weight's gradient 18946 x 3360 over 5351 bf16 1297 : 1283, 46547 x 5976 over 253 529 : 584;
// 8-bit layers, whose steps are others than the table's, 8965 x 12250, k 448 124 : 147, 8447 x 955, k 352 15.6 : 18.2, but 542 x 8373, k 2576 34.8 : 28.3.
// In fp32 128 x 64 is never dearer than the two larger shapes by a twentieth: four tiles of 128 x 128 cost less than one of 256 x 256,
// two of 128 x 64 less than 1.02 of 128 x 128, for any number of steps.  Where a unit has one small tile of many steps, four groups of
// waves share these out (512 x 1000, k 4096: 31.6 -> 29.1 bf16, 94 -> 84 fp32).
inline Tiles choose_tiles(int64_t m, int64_t n, int64_t steps, bool f32) {
    Tiles best = BIG;
    uint64_t least = uint64_t(1) << 62;
    for (Tiles t : {BIG, MID, HALF, SMALL}) {
        if (f32 && (t == BIG || t == MID)) continue;
        const TileShape s = shape_of(t, f32);
        const uint64_t cost = tile_cost(tiles_of(s, m, n), unsigned(steps), unsigned(s.fixed), unsigned(s.step));
        if (cost < least + least / 20) {
            best = t;
            least = cost;
        }
    }
    return best == SMALL && steps >= 64 && tiles_of(shape_of(SMALL, f32), m, n) <= 256 ? SMALL_SPLIT : best;
}
inline int64_t steps_of(int64_t inner, int esz) { return ceil_of(inner * esz, 64); }

// ---- loss ----
// Columns of the vocabulary that leave one maximum and sum per token.
inline int64_t part_columns(int64_t tokens, int64_t width, int64_t vocab, int esz) {
    return few_rows(tokens, vocab, esz) ? 32 : shape_of(choose_tiles(tokens, vocab, steps_of(width, esz), esz == 4), esz == 4).n;
}
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
// How many are taken, from the number of kept tokens (of whose tiles there are `tiles`): more only where they save a twelfth, since
// a second small tile for every compute unit is not dealt out evenly (231 x 832 over 76393 fp32: 297 us in 8 shares of
// 28 tiles, 484 in 16).
ONECOMP_TOKEN_FN int shares_of(unsigned tiles, unsigned steps, unsigned fixed, unsigned step, int most) {
    int best = 1;
    uint64_t least = ~uint64_t(0);
    for (int s = 1; s <= most; ++s) {
        const uint64_t cost = tile_cost(tiles * unsigned(s), (steps + unsigned(s) - 1) / unsigned(s), fixed, step);
        if (s == 1 || cost < least - least / 12) {
            best = s;
            least = cost;
        }
    }
    return best;
}
// The shape of dh's tiles, if all tokens are kept: with the shares that it would take.  Each share's sums go to memory in 32 bits
// and are read again (by the next piece of the vocabulary, by the kernel that adds the shares up): 13 us for a quarter MB of every
// compute unit at 5 TB/s, three times.
inline TileShape rows_shape(Tiles t, bool f32) {
    TileShape s = shape_of(t, f32);
    s.fixed += int(int64_t(39000) * s.n * s.m / 65536);
    return s;
}
inline Tiles choose_rows(int64_t tokens, int64_t width, int64_t columns, int esz) {
    Tiles best = BIG;
    uint64_t least = ~uint64_t(0);
    const unsigned steps = unsigned(steps_of(columns, esz));
    for (Tiles t : {BIG, MID, HALF, SMALL}) {
        const TileShape s = rows_shape(t, esz == 4);
        const unsigned tiles = tiles_of(s, tokens, width);
        const unsigned shares = unsigned(shares_of(tiles, steps, unsigned(s.fixed), unsigned(s.step), int(most_shares(tokens, width))));
        const uint64_t cost = tile_cost(tiles * shares, (steps + shares - 1) / shares, unsigned(s.fixed), unsigned(s.step));
        if (cost < least) {
            best = t;
            least = cost;
        }
    }
    return best;
}

inline int64_t round_up(int64_t x, int64_t to) { return ceil_of(x, to) * to; }

struct LossSpace {
    size_t index, place, count, unit, coef, rows, parts, hit, piece, dh, all;
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
    s.unit = take(gradient ? 4 : 0);
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
