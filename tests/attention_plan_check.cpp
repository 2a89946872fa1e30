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

int main() {
    for (int nk : lengths()) {
        check_runs(nk);
        check_shares(nk);
    }
    std::printf("ok %ld\n", checked);
    return 0;
}
