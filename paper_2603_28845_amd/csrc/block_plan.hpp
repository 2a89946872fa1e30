// What a call for the gradients of a block's norms does with the caller's memory: plain host logic, apart from the launches so
// that a host program can check it (tests/block_plan_check.cpp).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace onecomp {
namespace block {

// 32 bytes per row: what the strips of wide rows' parameter gradients take from the rows' sums
struct RowNumbers {
    float mean_h, inv_h, mean_d, along, mean_y, inv_y, unused[2];
};

// Registers for the parameters' sums: rows of this capacity (entries that a workgroup holds) keep them in the kernel that reads
// the rows, wider ones leave them to the strips.
constexpr bool own_sums(int capacity, bool layer) { return capacity <= (layer ? 4096 : 8192); }

inline size_t round_up_256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Workspace: the rows' numbers, where the width can need them, then the parameters' sums.
inline size_t numbers_bytes(int64_t rows, int64_t width) { return width > 4096 ? round_up_256(size_t(rows < 1 ? 1 : rows) * sizeof(RowNumbers)) : 0; }

struct Scratch {
    char *numbers, *sums;
};
// Calls that want no parameter's gradient (wanted == 0) write nothing to the workspace, which may then be missing or of any size.
inline Scratch scratch_of(void* workspace, int64_t rows, int64_t width, int wanted) {
    if (!wanted || !workspace) return Scratch{nullptr, nullptr};
    char* at = static_cast<char*>(workspace);
    return Scratch{at, at + numbers_bytes(rows, width)};
}

// Whether any of the outputs lies over one of the inputs; NULL: not there.
template <int N, int M>
inline bool over_inputs(const void* const (&outputs)[N], const void* const (&inputs)[M]) {
    for (const void* o : outputs)
        for (const void* i : inputs)
            if (o && o == i) return true;
    return false;
}

}  // namespace block
}  // namespace onecomp
