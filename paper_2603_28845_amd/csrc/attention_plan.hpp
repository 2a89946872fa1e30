// How attention's keys are shared out: plain integer logic of kernels and launchers that compiles as ordinary C++ too, so that a
// host program can check it at any length (tests/attention_plan_check.cpp).
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define ONECOMP_HD __host__ __device__ inline
#else
#define ONECOMP_HD inline
#endif

namespace onecomp {
namespace attn {

// Few rows: keys of one piece of work.  Runs of `run` or, where the host knew of fewer keys than there are, as many as it takes for
// `splits` runs to cover them all.  Lengths reach 2^31 - 4096, runs 2^30 and the keys of all shares in a tile's steps 2^15: sums
// of two of these take 32 bits without a sign.  (In 64 bits the divisions cost a call of single tokens 2 us of 100.)
ONECOMP_HD int run_of(int run, int splits, int nk) {
    const uint32_t unit = uint32_t(splits) * 128u, least = (uint32_t(nk) + unit - 1u) / unit * 128u;
    return least > uint32_t(run) ? int(least) : run;
}
ONECOMP_HD int runs_of(int run, int splits, int nk) {
    const uint32_t each = uint32_t(run_of(run, splits, nk)), runs = (uint32_t(nk) + each - 1u) / each;
    return runs > 1u ? int(runs) : 1;
}

// Many sequences: each has its slots, as many units of `unit` rows (tiles of tokens from MANY sequences on, blocks of a few rows from
// MANY_TOKENS on) as its place can need and one more at most, so that a slot's sequence is found by search and not by counting
// all before it: ceil((b - a) / unit) <= floor(b / unit) - floor(a / unit) + 1 for a sequence of rows a .. b - 1.
constexpr int MANY = 256, MANY_TOKENS = 1024;
ONECOMP_HD int64_t first_slot(int64_t rows_before, int unit, int sequence) { return rows_before / unit + sequence; }
// slots of all sequences and of the padding behind them
ONECOMP_HD int64_t all_slots(int64_t rows, int unit, int sequences) { return rows / unit + sequences + 1; }
// Runs of keys for each slot of a few rows: a slot that has fewer is looked at for nothing, so that many sequences get few.
ONECOMP_HD int most_splits(int sequences) {
    const int n = sequences < MANY_TOKENS ? 256 : 65536 / sequences;
    return n < 1 ? 1 : n > 256 ? 256 : n;
}

struct Range {
    int begin, end;
};
// Run `split` of the keys 0 .. seen - 1.
ONECOMP_HD Range run_range(int run, int split, int seen) {
    const uint32_t begin = uint32_t(run) * uint32_t(split), end = begin + uint32_t(run);
    return Range{int(begin), int(end < uint32_t(seen) ? end : uint32_t(seen))};
}
// Share `which` of `shares` of the keys 0 .. end - 1, in tiles of `keys`; empty where begin >= end.
ONECOMP_HD Range share_of(int end, int keys, int shares, int which) {
    const uint32_t unit = uint32_t(keys) * uint32_t(shares), share = (uint32_t(end) + unit - 1u) / unit * uint32_t(keys), begin = share * uint32_t(which), to = begin + share;
    if (begin >= uint32_t(end)) return Range{0, 0};
    return Range{int(begin), int(to < uint32_t(end) ? to : uint32_t(end))};
}

}  // namespace attn
}  // namespace onecomp
