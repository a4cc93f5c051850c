// Memory spans of a call's arguments: entry points whose workgroups read
// their inputs at any time refuse outputs that lie on an input or on another
// output.  Not part of the public interface.
#pragma once

#include <cstdint>

namespace triattn {

struct Span {
    const void *at;
    int64_t bytes;
};

// Whether one of the first `outputs` of n spans shares memory with another.
inline bool spans_overlap(const Span *spans, int outputs, int n)
{
    for (int i = 0; i < outputs; ++i)
        for (int j = i + 1; j < n; ++j) {
            const uintptr_t a = (uintptr_t)spans[i].at, b = (uintptr_t)spans[j].at;
            if (spans[i].at && spans[j].at && spans[i].bytes > 0 && spans[j].bytes > 0 &&
                a < b + (uintptr_t)spans[j].bytes && b < a + (uintptr_t)spans[i].bytes)
                return true;
        }
    return false;
}

}  // namespace triattn
