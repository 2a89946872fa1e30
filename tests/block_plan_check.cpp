// Host check of csrc/block_plan.hpp.  Prints "ok <number of checks>" on success, the first failure otherwise.
#include "../paper_2603_28845_amd/csrc/block_plan.hpp"

#include <cstdio>
#include <cstdlib>
#include <initializer_list>

using namespace onecomp::block;

static long checked = 0;
#define REQUIRE(c, ...)                                                                                          \
    do {                                                                                                         \
        ++checked;                                                                                               \
        if (!(c)) { std::printf("FAILED %s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } \
    } while (0)

// Nothing of the workspace is used where no parameter's gradient is wanted; else its parts lie one behind the other.
static void check_scratch() {
    char base[1];
    for (int64_t width = 1; width <= 32768; width += 13)
        for (int64_t rows : {0, 1, 3, 37, 4096, 65536}) {
            for (void* ws : {static_cast<void*>(nullptr), static_cast<void*>(base)}) {
                const Scratch none = scratch_of(ws, rows, width, 0);
                REQUIRE(!none.numbers && !none.sums, "rows %ld width %ld: scratch without a parameter's gradient", long(rows), long(width));
            }
            for (int wanted = 1; wanted < 32; ++wanted) {
                const Scratch s = scratch_of(base, rows, width, wanted);
                const size_t numbers = numbers_bytes(rows, width);
                REQUIRE(s.numbers == base && s.sums == base + numbers && numbers % 256 == 0, "rows %ld width %ld", long(rows), long(width));
                REQUIRE(width <= 4096 || numbers >= size_t(rows) * sizeof(RowNumbers), "rows %ld width %ld", long(rows), long(width));
            }
        }
    for (int capacity : {512, 2048, 4096}) REQUIRE(own_sums(capacity, true) && own_sums(capacity, false), "%d", capacity);
}

int main() {
    check_scratch();
    std::printf("ok %ld\n", checked);
    return 0;
}
