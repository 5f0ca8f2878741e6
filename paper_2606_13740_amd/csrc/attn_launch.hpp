// Launches of the paged attention: which of its tiles a call gets.
#pragma once

#include "attn_paged.hpp"

namespace dllm {

template <typename T, int DH, bool TREE>
void launch_attn_dh(const PagedArgs& a, const AttnPlan& p, hipStream_t s) {
    constexpr int SUB = sizeof(T) == 4 ? 1 : 2;
    const dim3 grid((unsigned)(p.wgs_s + p.wgs_o));
#define ATTN(QG_, RT_, KG_) \
    hipLaunchKernelGGL((attn_paged_kernel<T, DH, QG_, RT_, KG_, SUB, TREE>), grid, dim3(QG_ * KG_ * 64), 0, s, a)
    if constexpr (sizeof(T) == 2) {
        if (p.qt == 2) ATTN(4, 32, 1);
        else if (p.qg == 4) ATTN(4, 16, 1);
        else if (p.qg == 2) ATTN(2, 16, 2);
        else ATTN(1, 16, 2);
    } else {
        if (p.qg == 4) ATTN(4, 16, 1);
        else if (p.qg == 2) ATTN(2, 16, 1);
        else ATTN(1, 16, 1);
    }
#undef ATTN
}

template <typename T, bool TREE>
void launch_attn_t(const PagedArgs& a, const AttnPlan& p, int Dh, hipStream_t s) {
    if (Dh == 128) launch_attn_dh<T, 128, TREE>(a, p, s);
    else if (Dh == 64) launch_attn_dh<T, 64, TREE>(a, p, s);
    else if constexpr (sizeof(T) == 4) launch_attn_dh<T, 32, TREE>(a, p, s);
}

// All parts of an attention call of type `dtype`; what is left is their merge.
template <bool TREE>
void launch_attn(int dtype, const PagedArgs& a, const AttnPlan& p, int Dh, hipStream_t s) {
    if (dtype == DLLM_F32) launch_attn_t<float, TREE>(a, p, Dh, s);
    else if (dtype == DLLM_F16) launch_attn_t<_Float16, TREE>(a, p, Dh, s);
    else launch_attn_t<__bf16, TREE>(a, p, Dh, s);
}

// The same with masks (attn_tree.hip, a translation unit of its own: these are many kernels).
void launch_attn_tree(int dtype, const PagedArgs& a, const AttnPlan& p, int Dh, hipStream_t s);

}  // namespace dllm
