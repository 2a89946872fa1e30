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

// The strips read every input anew: a result over any of them has to wait, one that is not wanted over an input that is not
// there does not.
static void check_over() {
    char b[8];
    const char* in[5] = {b, b + 1, b + 2, b + 3, b + 4};         // h, y, dn, dh_out, gate
    for (int missing = 0; missing < 32; ++missing) {
        const void* inputs[5];
        for (int i = 0; i < 5; ++i) inputs[i] = missing >> i & 1 ? nullptr : in[i];
        for (int which = 0; which < 27; ++which) {                // each output not wanted, apart, or over the chosen input
            for (int input = 0; input < 5; ++input) {
                const void* outputs[3];
                bool any = false;
                for (int o = 0, w = which; o < 3; ++o, w /= 3) {
                    outputs[o] = w % 3 == 0 ? nullptr : w % 3 == 1 ? b + 5 + o : static_cast<const void*>(in[input]);
                    any = any || (w % 3 == 2 && inputs[input]);
                }
                REQUIRE(over_inputs(outputs, inputs) == any, "outputs %d, input %d, missing %d", which, input, missing);
            }
        }
    }
}

int main() {
    check_scratch();
    check_over();
    std::printf("ok %ld\n", checked);
    return 0;
}
