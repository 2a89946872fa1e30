// Host check of csrc/token_plan.hpp.  Prints "ok <number of checks>" on success, the first failure otherwise.
#include "../paper_2603_28845_amd/csrc/token_plan.hpp"

#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>

using namespace onecomp;
using namespace onecomp::token;

static long checked = 0;
#define REQUIRE(c, ...)                                                                                          \
    do {                                                                                                         \
        ++checked;                                                                                               \
        if (!(c)) { std::printf("FAILED %s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } \
    } while (0)

// Every tile has one workgroup, whatever part of the tiles that the launch was made for is there.
static void check_tiles() {
    for (int64_t m : {0, 1, 2, 7, 8, 9, 16, 31, 64})
        for (int64_t n : {1, 2, 3, 8, 33, 500})
            for (int64_t launched : {m, m + 1, 2 * m + 5}) {
                std::vector<int> seen(size_t(m * n), 0);
                const int64_t blocks = product::tile_blocks(launched, n);
                for (int64_t b = 0; b < blocks; ++b) {
                    int tm, tn;
                    if (!product::tile_of(unsigned(b), int(m), int(n), tm, tn)) continue;
                    REQUIRE(tm >= 0 && tm < m && tn >= 0 && tn < n, "%ld of %ld x %ld", long(b), long(m), long(n));
                    ++seen[size_t(tm * n + tn)];
                }
                for (int s : seen) REQUIRE(s == 1, "%ld x %ld, %ld launched", long(m), long(n), long(launched));
            }
}

static void check_embedding() {
    for (int64_t vocab = 1; vocab <= (int64_t(1) << 24); vocab = vocab * 3 + 1) {
        const int r = sort_rows(vocab);
        REQUIRE(r >= 64 && r <= SORT_MOST && r % 64 == 0, "%ld", long(vocab));
        for (int64_t n : {0, 1, 15, 16, 17, 16383, 16384, 100000, 1 << 30})
            for (int64_t width : {1, 64, 4097}) {
                const EmbeddingSpace s = embedding_space(n, vocab, width);
                REQUIRE(s.segments * segment_of(n, width) >= n && (s.segments - 1) * segment_of(n, width) < n, "%ld", long(n));
                REQUIRE(s.starts >= s.order + size_t(n) * 4 && s.parts >= s.starts + (size_t(vocab) + 1) * 4 && s.all >= s.parts + size_t(s.segments) * 2 * size_t(width) * 4,
                        "%ld %ld %ld", long(n), long(vocab), long(width));
                REQUIRE(s.order % 256 == 0 && s.starts % 256 == 0 && s.parts % 256 == 0, "%ld", long(n));
            }
    }
}

static void check_loss() {
    for (int esz : {2, 4})
        for (int64_t tokens : {0, 1, 64, 65, 100, 1535, 1536, 4096, 16384, 100000, 1 << 20})
            for (int64_t vocab : {1, 255, 256, 257, 5000, 128000, 1 << 20, 1 << 24})
                for (int64_t width : {8, 64, 1000, 4096, 8192}) {
                    const size_t t = size_t(tokens), row = size_t(ceil_of(width * esz, 64) * 64);
                    const int64_t parts = ceil_of(vocab, part_columns(tokens, width, vocab, esz));
                    for (bool gradient : {false, true}) {
                        const LossSpace s = loss_space(tokens, width, vocab, esz, parts, gradient);
                        const int64_t c = s.columns, shares = s.shares;
                        REQUIRE(s.index >= s.count + 4 && s.coef >= s.index + 4 * t && s.rows >= s.coef + (gradient ? 16 : 4) * t, "%ld", long(tokens));
                        if (gradient) {
                            REQUIRE(c > 0 && c % 256 == 0 && c < vocab + 256 + 2048, "%ld %ld", long(tokens), long(vocab));
                            REQUIRE(c <= 2048 || tokens * c * esz <= PIECE_BYTES, "%ld %ld", long(tokens), long(vocab));
                            REQUIRE(s.place >= s.index + 4 * t && s.coef >= s.place + 4 * t, "%ld", long(tokens));
                            REQUIRE(s.piece >= s.rows + t * row && s.dh >= s.piece + t * size_t(c) * esz, "%ld", long(tokens));
                            REQUIRE(s.all >= s.dh + t * size_t(width) * 4 * size_t(shares), "%ld", long(tokens));
                            REQUIRE(shares >= 1 && shares <= 16, "%ld", long(shares));
                            const TileShape tile = rows_shape(choose_rows(tokens, width, c, esz), esz == 4);
                            for (unsigned tiles : {0u, 1u, 20u, 255u, 256u, 257u, 320u, 5000u}) {
                                const int taken = shares_of(tiles, unsigned(steps_of(c, esz)), unsigned(tile.fixed), unsigned(tile.step), int(shares));
                                REQUIRE(taken >= 1 && taken <= shares, "%d of %ld", taken, long(shares));
                            }
                        } else {
                            REQUIRE(s.parts >= s.rows + t * row && s.hit >= s.parts + t * size_t(parts) * 8 && s.all >= s.hit + 4 * t, "%ld", long(tokens));
                        }
                        // offsets of the loads of a tile stay below 2^31: up to sixteen panels
                        REQUIRE(tokens * 64 * 16 < (int64_t(1) << 31), "%ld", long(tokens));
                        for (size_t at : {s.count, s.index, s.place, s.coef, s.rows, s.parts, s.hit, s.piece, s.dh}) REQUIRE(at % 256 == 0, "%ld", long(tokens));
                    }
                }
}

int main() {
    check_tiles();
    check_embedding();
    check_loss();
    std::printf("ok %ld\n", checked);
    return 0;
}
