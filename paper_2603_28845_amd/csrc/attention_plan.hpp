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
// `splits` runs to cover them all.  Lengths reach 2^31 - 4096: sums of theirs take 64 bits.
ONECOMP_HD int run_of(int run, int splits, int nk) {
    const int64_t least = (int64_t(nk) + int64_t(splits) * 128 - 1) / (int64_t(splits) * 128) * 128;
    return least > run ? int(least) : run;
}
ONECOMP_HD int runs_of(int run, int splits, int nk) {
    const int64_t each = run_of(run, splits, nk), runs = (nk + each - 1) / each;
    return runs > 1 ? int(runs) : 1;
}

struct Range {
    int begin, end;
};
// Run `split` of the keys 0 .. seen - 1.
ONECOMP_HD Range run_range(int run, int split, int seen) {
    const int64_t begin = int64_t(run) * split, end = begin + run;
    return Range{int(begin), int(end < seen ? end : seen)};
}
// Share `which` of `shares` of the keys 0 .. end - 1, in tiles of `keys`; empty where begin >= end.
ONECOMP_HD Range share_of(int end, int keys, int shares, int which) {
    const int64_t unit = int64_t(keys) * shares, share = (end + unit - 1) / unit * keys, begin = share * which, to = begin + share;
    if (begin >= end) return Range{0, 0};
    return Range{int(begin), int(to < end ? to : end)};
}

}  // namespace attn
}  // namespace onecomp
