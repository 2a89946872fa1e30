// Host check of csrc/attention_plan.hpp: runs and shares tile the keys at any length.  Prints "ok <number of checks>" on success, the
// first failure otherwise.
#include "../paper_2603_28845_amd/csrc/attention_plan.hpp"

#include <cstdio>
#include <cstdlib>
#include <vector>

using namespace onecomp::attn;

static long checked = 0;
#define REQUIRE(c, ...)                                                                                          \
    do {                                                                                                         \
        ++checked;                                                                                               \
        if (!(c)) { std::printf("FAILED %s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } \
    } while (0)

static const int LONGEST = 2147483647 - 4095;     // the longest sequence that the entry points take

static std::vector<int> lengths() {
    std::vector<int> all;
    for (int n = 0; n < 1200; ++n) all.push_back(n);
    for (long n = 1200; n < LONGEST; n = n * 17 / 16 + 1) all.push_back(int(n));
    for (int back = 0; back < 70000; back += 61) all.push_back(LONGEST - back);
    return all;
}

// every key lies in one run, and no more than `splits` runs are needed
static void check_runs(int nk) {
    for (int run : {128, 256, 1536, 1 << 20, 1 << 30})
        for (int splits : {1, 2, 7, 64, 256}) {
            const int each = run_of(run, splits, nk), runs = runs_of(run, splits, nk);
            REQUIRE(each >= run && runs >= 1 && runs <= splits, "%d keys, run %d, splits %d: %d runs of %d", nk, run, splits, runs, each);
            int upto = 0;
            for (int r = 0; r < runs; ++r) {
                const Range x = run_range(each, r, nk);
                REQUIRE(x.begin == upto || nk == 0, "%d keys, run %d, splits %d: run %d begins at %d", nk, run, splits, r, x.begin);
                REQUIRE(x.end >= x.begin, "%d keys, run %d, splits %d: run %d ends at %d", nk, run, splits, r, x.end);
                upto = x.end;
            }
            REQUIRE(upto == nk, "%d keys, run %d, splits %d: %d covered", nk, run, splits, upto);
        }
}

static void check_shares(int nk) {
    for (int keys : {32, 64})
        for (int shares : {1, 2, 5, 64, 512}) {
            int upto = 0;
            for (int s = 0; s < shares; ++s) {
                const Range x = share_of(nk, keys, shares, s);
                if (x.begin >= x.end) continue;
                REQUIRE(x.begin == upto && x.begin % keys == 0 && x.end <= nk, "%d keys, share %d of %d: %d to %d", nk, s, shares, x.begin, x.end);
                upto = x.end;
            }
            REQUIRE(upto == nk, "%d keys in %d shares: %d covered", nk, shares, upto);
        }
}

// the last sequence whose slots begin at `slot` or before; as the kernels search for it, 64 places at a time
static int search(const std::vector<int>& starts, int group, int unit, int64_t slot) {
    int lo = 0, hi = int(starts.size());
    do {
        const int step = (hi - lo + 63) / 64;
        int who = -1;
        for (int lane = 0; lane < 64; ++lane) {
            const int at = lo + lane * step;
            if (at < hi && first_slot(int64_t(starts[at]) * group, unit, at) <= slot) who = lane;
        }
        if (who < 0) return -1;
        lo += who * step;
        hi = hi < lo + step ? hi : lo + step;
    } while (hi - lo > 1);
    return lo;
}

// every tile of every sequence, and of the padding behind them, has one slot, and no slot is another sequence's
static void check_slots(int n, int longest, int padding, int group, int unit, unsigned seed) {
    std::vector<int> starts{0};
    unsigned x = seed * 2654435761u + 1;
    for (int i = 0; i < n; ++i) {
        x = x * 1664525u + 1013904223u;
        starts.push_back(starts.back() + int((x >> 8) % unsigned(longest + 1)));
    }
    const int total = starts.back() + padding;
    const int64_t slots = all_slots(int64_t(total) * group, unit, n);
    int64_t slot = 0;
    for (int i = 0; i <= n; ++i) {
        const int64_t rows = (int64_t(i < n ? starts[i + 1] : total) - starts[i]) * group, tiles = (rows + unit - 1) / unit;
        const int64_t first = first_slot(int64_t(starts[i]) * group, unit, i);
        REQUIRE(first >= slot && first + tiles <= slots, "%d sequences to %d, group %d, unit %d: sequence %d at %ld", n, longest, group, unit, i, long(first));
        for (int64_t t = 0; t < tiles; ++t)
            REQUIRE(search(starts, group, unit, first + t) == i, "%d sequences to %d, group %d, unit %d: tile %ld of %d", n, longest, group, unit, long(t), i);
        slot = first + tiles;
    }
}

int main() {
    for (int n : {64, 65, 127, 128, 1000, 4097})
        for (int longest : {0, 1, 31, 129, 700})
            for (int padding : {0, 1, 300})
                for (int unit : {32, 128}) check_slots(n, longest, padding, unit == 32 ? 1 + n % 8 : 1, unit, unsigned(n + longest));
    for (int n = 0; n < (1 << 24); n += 1 + n / 64)
        REQUIRE(most_splits(n) >= 1 && most_splits(n) <= 256 && (n < MANY_TOKENS || int64_t(most_splits(n)) * n <= 65536 + n), "%d sequences", n);
    for (int nk : lengths()) {
        check_runs(nk);
        check_shares(nk);
    }
    std::printf("ok %ld\n", checked);
    return 0;
}
