// Arithmetic of the batch operators that decides which memory a launch touches: plain C++, so that it is checked
// on the CPU.
#pragma once

namespace dllm {

// Rows [begin, end) of a call of T rows.
struct RowRange {
    int begin, end;
};
// Rows [first, behind) cut to [0, T) and to at most `most` of them.  first and behind come from device memory and may be
// anything: the result lies in [0, T], begin <= end, and no sum leaves 32 bits (most is cut before it is added).
constexpr RowRange row_range(int first, int behind, int most, int T) {
    const int begin = first < 0 ? 0 : (first > T ? T : first);
    const int room = T - begin, n = most < 0 ? 0 : (most < room ? most : room), top = begin + n;
    return RowRange{begin, behind < begin ? begin : (behind < top ? behind : top)};
}

}  // namespace dllm
