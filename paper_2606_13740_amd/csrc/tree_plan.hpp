// Positions and masks of the rows of drafted trees, from their parents.
#pragma once

#include "batch_rules.hpp"
#include "common.hpp"

namespace dllm {

struct TreeArgs {
    const int *parent, *row0, *len;
    int T, B;
    int* pos;
    uint32_t* mask;
    int ld;
};

// mask_i = {i} and mask_{parent_i}: row i sees itself and its ancestors, and its depth is their number.
//
// A workgroup takes a sequence.  Inside blocks of 32 rows the ancestors are found by doubling (after step s a row knows
// its next 2^s nodes and the one behind them: five steps), for all blocks at once.  What lies before a row's block is
// the mask of the first ancestor outside of it, complete when the blocks are taken in order: one step a block, whatever
// the trees' depth (walking up would take a dependent LDS read a node: a chain of 1024 rows 1024 of them).
constexpr int TREE_NT = 256;
__global__ void __launch_bounds__(TREE_NT) tree_plan_kernel(TreeArgs a) {
    extern __shared__ uint32_t tree_lds[];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int first = a.row0[b], len = a.len[b];
    const RowRange rows = row_range(first, a.row0[b + 1], a.T, a.T);
    const int R0 = rows.begin, n_rows = rows.end - rows.begin, n = min(n_rows, 32 * a.ld);
    const int base = max(len, 0) - n_rows;
    uint32_t* M = tree_lds;                              // [32 ld][ld] masks
    uint32_t* own_s = M + 32 * a.ld * a.ld;              // [32 ld] a row's bits in its own block
    int* exit_s = (int*)(own_s + 32 * a.ld);             // [32 ld] its first ancestor outside of the block, or -1
    int* depth_s = exit_s + 32 * a.ld;                   // [32 ld] nodes of its path

    for (int i0 = tid & ~63; i0 < n; i0 += TREE_NT) {    // (whole waves: two blocks each)
        const int i = i0 + lane, blk = i & ~31;
        const int p0 = i < n ? a.parent[R0 + i] : -1, p = p0 >= 0 && p0 < i ? p0 : -1;
        uint32_t word = 1u << (i & 31);
        int anc = p >= blk ? p : -1, out = anc >= 0 ? -1 : p;
#pragma unroll
        for (int s = 0; s < 5; ++s) {
            const int from = anc >= 0 ? anc - i0 : lane;
            const uint32_t w = __shfl(word, from);
            const int o = __shfl(out, from), up = __shfl(anc, from);
            if (anc >= 0) {
                word |= w;
                out = o;
                anc = up;
            }
        }
        if (i < n) {
            own_s[i] = word;
            exit_s[i] = out;
        }
    }
    __syncthreads();
    int lw = 0;                                          // log2 of the lanes of a row
    while ((1 << lw) < a.ld) ++lw;
    const int w = tid & ((1 << lw) - 1), step = TREE_NT >> lw;
    for (int k = 0; 32 * k < n; ++k) {
        const int end = min(n, 32 * k + 32);
        for (int i = 32 * k + (tid >> lw); i < end; i += step) {
            const int e = exit_s[i];
            const uint32_t own = own_s[i];
            if (w < a.ld) {
                const uint32_t v = w == k ? own : (w < k && e >= 0 ? M[e * a.ld + w] : 0u);
                M[i * a.ld + w] = v;
                a.mask[(size_t)(R0 + i) * a.ld + w] = v;
            }
            if (w == 0) {
                const int d = __popc(own) + (e >= 0 ? depth_s[e] : 0);
                depth_s[i] = d;
                a.pos[R0 + i] = base + d - 1;
            }
        }
        __syncthreads();
    }
}

}  // namespace dllm
