// Host check, built with the sanitizer of undefined behaviour: which row of a sorting workgroup a token of any 32 bits belongs to.
// Prints "ok <number of checks>" on success, the first failure otherwise.
#include "../paper_2603_28845_amd/csrc/token_plan.hpp"

#include <cstdio>

int main() {
    using namespace onecomp::token;
    long checked = 0;
    for (int64_t vocab : {1, 63, 64, 65, 777, 70000, 128000, 1 << 24}) {
        const int each = sort_rows(vocab);
        for (int32_t token : {INT32_MIN, INT32_MIN + 1, -100, -1, 0, 1, 63, 64, 500, int(vocab) - 1, int(vocab), int(vocab) + 63, INT32_MAX - 1, INT32_MAX}) {
            int owners = 0;
            for (int64_t lo = 0; lo < vocab; lo += each) {
                const int rows = int(vocab - lo < each ? vocab - lo : each), row = row_of(token, int(lo), rows);
                ++checked;
                if (row >= rows || (row >= 0 && lo + row != token)) {
                    std::printf("FAILED %d of %ld: row %d of %ld\n", token, long(vocab), row, long(lo));
                    return 1;
                }
                owners += row >= 0;
            }
            if (owners != (token >= 0 && token < vocab)) {
                std::printf("FAILED %d of %ld: %d owners\n", token, long(vocab), owners);
                return 1;
            }
        }
    }
    std::printf("ok %ld\n", checked);
    return 0;
}
