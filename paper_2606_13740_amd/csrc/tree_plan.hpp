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
// its next 2^s nodes and the one behind them: five steps), for all blocks at once.  What lies before a row's block are the
// bits that its first ancestor outside of it has in its own block, and so on: a thread takes a row and one LDS read a
// block, whatever the trees' depth.  What bounds it is launch and latency: 1.9 us a call in a row of them for 8 trees of 16 rows,
// 2.9 for 64 of up to 256 (block after block in order, with the rows' masks in LDS and a barrier each, 2.1 and 4.7); alone 3.4 and 4.7.
constexpr int TREE_NT = 256;
__global__ void __launch_bounds__(TREE_NT) tree_plan_kernel(TreeArgs a) {
    __shared__ uint2 node_s[32 * TREE_MAX_LD];           // a row's bits in its block, and its first ancestor outside, or -1
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int first = a.row0[b], len = a.len[b];
    const RowRange rows = row_range(first, a.row0[b + 1], a.T, a.T);
    const int R0 = rows.begin, n_rows = rows.end - rows.begin, n = min(n_rows, 32 * a.ld);
    const int base = max(len, 0) - n_rows;

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
        if (i < n) node_s[i] = make_uint2(word, (uint32_t)out);
    }
    __syncthreads();
    for (int i = tid; i < n; i += TREE_NT) {
        uint2 at = node_s[i];
        uint32_t* mask = a.mask + (size_t)(R0 + i) * a.ld;
        for (int w = a.ld - 1; w > i >> 5; --w) mask[w] = 0;
        mask[i >> 5] = at.x;
        int depth = __popc(at.x);
        for (int w = (i >> 5) - 1; w >= 0; --w) {
            const int up = (int)at.y;                    // (an earlier block's row, or none)
            uint32_t word = 0;
            if (up >= 0 && up >> 5 == w) {
                at = node_s[up];
                word = at.x;
                depth += __popc(word);
            }
            mask[w] = word;
        }
        a.pos[R0 + i] = base + depth - 1;
    }
}

}  // namespace dllm
