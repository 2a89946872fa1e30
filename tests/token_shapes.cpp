// Which forms csrc/token_plan.hpp chooses: a question a line, answered by a number a line.
#include "../paper_2603_28845_amd/csrc/token_plan.hpp"

#include <iostream>
#include <string>

int main() {
    using namespace onecomp::token;
    std::string what;
    while (std::cin >> what) {
        long a, b, c, d;
        if (what == "few" && std::cin >> a >> b >> c) std::cout << few_rows(a, b, int(c));                                         // m n esz
        else if (what == "tiles" && std::cin >> a >> b >> c >> d) std::cout << choose_tiles(a, b, steps_of(c, int(d)), d == 4);    // m n k esz
        else if (what == "rows" && std::cin >> a >> b >> c >> d) std::cout << choose_rows(a, b, c, int(d));                        // tokens width columns esz
        else if (what == "columns" && std::cin >> a >> b >> c) std::cout << piece_columns(a, b, int(c));                           // tokens vocab esz
        else if (what == "segment" && std::cin >> a >> b) std::cout << segment_of(a, b);                                           // tokens width
        else return 1;
        std::cout << "\n";
    }
    return 0;
}
