// Small arithmetic of the host code.
#pragma once

namespace dllm {

inline int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }
inline long round_up(long a, long b) { return (a + b - 1) / b * b; }

}  // namespace dllm
