// Plan of a batched step: block tables, row positions and cache slots from request lengths.
#pragma once

#include "common.hpp"

namespace dllm {

struct PlanArgs {
    const int* len;
    const int* nw;
    const int* owned;
    int* owned_out;
    int B;
    int* table;
    int ld;
    int* free_;
    const int* n_free;
    int* n_free_out;
    int n_pages, page_shift, shared, max_rows;
    int *row0, *pos, *slot, *seq, *lim, *status;
};

// Exclusive scan of three 64-bit counts over a workgroup of NT threads; `total` gets the sums.
struct PlanSum {
    long long rows, take, give;
};
__device__ __forceinline__ PlanSum operator+(const PlanSum& a, const PlanSum& b) {
    return PlanSum{a.rows + b.rows, a.take + b.take, a.give + b.give};
}

// With need_b = ceil((len_b + new_b) / page), exclusive sums over the sequences
//   row0_b = sum new,  t0_b = sum max(0, need - owned),  g0_b = sum max(0, owned - need)
// place everything: given back page i lies at stack index n_free + i, missing page k comes
// from stack index n_free + g - 1 - k (g = all given back), row r belongs to the last b with
// row0_b <= r.  A stack index past n_free is a given back page, which is read where it still
// stands, in its table: takers write their tables only at [owned, need), givers' entries
// [need, owned) and stack entries below n_free are never written, so no workgroup reads
// what another writes, every workgroup repeats the scan (three loads a sequence, L2) and one launch
// does all.
//
// What bounds it: launch and the chain of dependent loads (lengths, scan, table or stack
// entry, slot).
constexpr int PLAN_NT = 512;
constexpr int PLAN_MAXB = 4096;
__global__ void __launch_bounds__(PLAN_NT) batch_plan_kernel(PlanArgs a) {
    constexpr int NW = PLAN_NT / 64;
    __shared__ int row0[PLAN_MAXB + 1], t0[PLAN_MAXB + 1], g0[PLAN_MAXB + 1];
    __shared__ PlanSum wsum[NW];
    __shared__ int bad_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long page = 1ll << a.page_shift;
    const int n_free = *a.n_free;
    const int per = (a.B + PLAN_NT - 1) / PLAN_NT;          // consecutive sequences per thread
    if (tid == 0) bad_s = 0;
    __syncthreads();

    auto counts = [&](int b, bool& bad) {
        const int len = a.len[b], nw = a.nw[b], own = a.owned[b];
        const long long need = ((long long)len + nw + page - 1) >> a.page_shift;
        bad = len < 0 || nw < 0 || own < 0 || own > a.ld || need > a.ld;
        PlanSum s{0, 0, 0};
        if (len >= 0 && nw >= 0 && own >= 0 && own <= a.ld) {
            s.rows = nw;
            s.take = need > own ? need - own : 0;
            const long long keep = max(need, (long long)min(a.shared, own));
            s.give = own > keep ? own - keep : 0;
        }
        return s;
    };

    PlanSum mine{0, 0, 0};
    bool any_bad = n_free < 0 || n_free > a.n_pages;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= a.B) break;
        bool bad;
        mine = mine + counts(b, bad);
        any_bad |= bad;
    }
    if (any_bad) bad_s = 1;
    PlanSum inc = mine;                                      // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        PlanSum up{__shfl_up(inc.rows, o), __shfl_up(inc.take, o), __shfl_up(inc.give, o)};
        if (lane >= o) inc = inc + up;
    }
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    PlanSum at{inc.rows - mine.rows, inc.take - mine.take, inc.give - mine.give}, total{0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) at = at + wsum[w];
        total = total + wsum[w];
    }
    const long long stack = (long long)n_free + total.give;  // entries after the pushes
    const long long shortage = total.take > stack ? total.take - stack : 0;
    const bool ok = !bad_s && shortage == 0 && total.rows <= a.max_rows && stack <= a.n_pages;
    for (int i = 0; i < per; ++i) {                          // where every count fits (ok): exact in 32 bits
        const int b = tid * per + i;
        if (b >= a.B) break;
        bool bad;
        const PlanSum s = counts(b, bad);
        row0[b] = ok ? (int)at.rows : 0;
        t0[b] = (int)at.take;
        g0[b] = (int)at.give;
        at = at + s;
    }
    if (tid == 0) {
        row0[a.B] = ok ? (int)total.rows : 0;
        t0[a.B] = (int)total.take;
        g0[a.B] = (int)total.give;
    }
    __syncthreads();

    // largest b with first[b] <= x (first is ascending, first[0] <= x < first[B])
    auto find = [&](const int* first, int x) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= x) lo = mid;
            else hi = mid;
        }
        return lo;
    };
    // the page at index i of the stack after the pushes
    auto stack_at = [&](int i) {
        if (i < n_free) return a.free_[i];
        const int k = i - n_free, b = find(g0, k);
        const int own = a.owned[b];
        return a.table[(size_t)b * a.ld + own - (g0[b + 1] - g0[b]) + (k - g0[b])];
    };
    const int n_stack = (int)stack;
    const int gtid = blockIdx.x * PLAN_NT + tid, gn = gridDim.x * PLAN_NT;

    for (int r = gtid; r < a.max_rows; r += gn) {
        int pos = 0, slot = -1, seq = -1, lim = 0;
        if (r < row0[a.B]) {
            seq = find(row0, r);
            const int len = a.len[seq], own = a.owned[seq];
            pos = len + r - row0[seq];
            lim = len + a.nw[seq];
            const int p = pos >> a.page_shift;
            const int pg = p < own ? a.table[(size_t)seq * a.ld + p] : stack_at(n_stack - 1 - t0[seq] - (p - own));
            if (pg >= 0 && pg < a.n_pages) slot = (pg << a.page_shift) + (pos & ((int)page - 1));
        }
        a.pos[r] = pos;
        a.slot[r] = slot;
        a.seq[r] = seq;
        a.lim[r] = lim;
    }
    for (int b = gtid; b <= a.B; b += gn) a.row0[b] = row0[b];
    for (int b = gtid; b < a.B; b += gn)
        a.owned_out[b] = a.owned[b] + (ok ? (t0[b + 1] - t0[b]) - (g0[b + 1] - g0[b]) : 0);
    if (ok) {
        const int n_take = t0[a.B], left = n_stack - n_take;
        for (int k = gtid; k < n_take; k += gn) {            // missing page k
            const int b = find(t0, k);
            a.table[(size_t)b * a.ld + a.owned[b] + (k - t0[b])] = stack_at(n_stack - 1 - k);
        }
        for (int i = n_free + gtid; i < left; i += gn) a.free_[i] = stack_at(i);
    }
    if (gtid == 0) {
        *a.n_free_out = ok ? n_stack - t0[a.B] : n_free;
        a.status[0] = (int)min(total.rows, 0x7FFFFFFFll);
        a.status[1] = (int)min(shortage, 0x7FFFFFFFll);
        a.status[2] = ok ? 0 : 1;
    }
}

}  // namespace dllm
