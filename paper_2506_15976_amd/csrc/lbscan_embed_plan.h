// How the embedding's gradient divides its tokens, in plain C++ so that it can be checked over ranges of sizes on the CPU.
#pragma once

namespace lbscan {

// A wave of the sort notes which of its groups of 64 ids have some of its block's rows, in a mask of 64 bits: a bit stands
// for 2^span_log2 groups, so that the last group has one of them.
constexpr int sort_span_log2(long groups)
{
    int span_log2 = 0;
    while ((groups - 1) >> span_log2 > 63) ++span_log2;
    return span_log2;
}

}  // namespace lbscan
