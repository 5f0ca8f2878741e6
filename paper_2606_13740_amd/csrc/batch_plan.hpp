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

// Sums over sequences: rows (64 bits: a refused plan may ask for anything), pages taken and given back.
struct PlanSum {
    long long rows;
    int take, give;
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
// does all: the first row_wgs workgroups the rows, the others the sequences, tables and stack.
//
// What bounds it: launch and the chain of dependent loads (lengths, scan, table or stack
// entry, slot): 4.7 us for 4 sequences of one row, 8.1 for 2048 of 32 (9.4 where each workgroup did
// its share of both kinds, one after the other).
constexpr int PLAN_NT = 512;
constexpr int PLAN_MAXB = 4096;
__global__ void __launch_bounds__(PLAN_NT) batch_plan_kernel(PlanArgs a, int row_wgs) {
    constexpr int NW = PLAN_NT / 64, PER = PLAN_MAXB / PLAN_NT;
    __shared__ int row0[PLAN_MAXB + 1], t0[PLAN_MAXB + 1], g0[PLAN_MAXB + 1], len_s[PLAN_MAXB], own_s[PLAN_MAXB];
    __shared__ PlanSum wsum[NW];
    __shared__ int wbad[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long page = 1ll << a.page_shift;
    const int n_free = *a.n_free;
    const int per = (a.B + PLAN_NT - 1) / PLAN_NT;          // consecutive sequences per thread

    int len[PER], nw[PER], own[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * per + i;
        len[i] = nw[i] = own[i] = 0;
        if (i < per && b < a.B) {
            len[i] = a.len[b];
            nw[i] = a.nw[b];
            own[i] = a.owned[b];
        }
    }
    PlanSum part[PER], mine{0, 0, 0};
    bool bad = n_free < 0 || n_free > a.n_pages;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        // pages past the table count as one too many, so that the sums stay in range
        const long long need = min(((long long)len[i] + nw[i] + page - 1) >> a.page_shift, (long long)a.ld + 1);
        const bool in = len[i] >= 0 && nw[i] >= 0 && own[i] >= 0 && own[i] <= a.ld;
        bad |= !in || need > a.ld;
        const int keep = max((int)need, min(a.shared, own[i]));
        part[i] = in ? PlanSum{nw[i], max((int)need - own[i], 0), max(own[i] - keep, 0)} : PlanSum{0, 0, 0};
        mine = mine + part[i];
    }
    PlanSum inc = mine;                                      // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        PlanSum up{__shfl_up(inc.rows, o), __shfl_up(inc.take, o), __shfl_up(inc.give, o)};
        if (lane >= o) inc = inc + up;
    }
    if (lane == 63) wsum[wave] = inc;
    const bool wave_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) wbad[wave] = wave_bad;
    __syncthreads();
    PlanSum at{inc.rows - mine.rows, inc.take - mine.take, inc.give - mine.give}, total{0, 0, 0};
    bad = false;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) at = at + wsum[w];
        total = total + wsum[w];
        bad |= wbad[w] != 0;
    }
    const int stack = n_free + total.give;                   // entries after the pushes
    const int shortage = max(total.take - stack, 0);
    const bool ok = !bad && shortage == 0 && total.rows <= a.max_rows && stack <= a.n_pages;
#pragma unroll
    for (int i = 0; i < PER; ++i) {                          // (rows fit 32 bits where they are used, in a granted plan)
        const int b = tid * per + i;
        if (i >= per || b >= a.B) break;
        row0[b] = ok ? (int)at.rows : 0;
        t0[b] = at.take;
        g0[b] = at.give;
        len_s[b] = len[i];
        own_s[b] = own[i];
        at = at + part[i];
    }
    if (tid == 0) {
        row0[a.B] = ok ? (int)total.rows : 0;
        t0[a.B] = total.take;
        g0[a.B] = total.give;
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
        return a.table[(size_t)b * a.ld + own_s[b] - (g0[b + 1] - g0[b]) + (k - g0[b])];
    };
    const int n_stack = stack;
    const bool rows = (int)blockIdx.x < row_wgs;
    const int gtid = (rows ? blockIdx.x : blockIdx.x - row_wgs) * PLAN_NT + tid;
    const int gn = (rows ? row_wgs : gridDim.x - row_wgs) * PLAN_NT;

    for (int r = rows ? gtid : a.max_rows; r < a.max_rows; r += gn) {
        int pos = 0, slot = -1, seq = -1, lim = 0;
        if (r < row0[a.B]) {
            seq = find(row0, r);
            const int own = own_s[seq];
            pos = len_s[seq] + r - row0[seq];
            lim = len_s[seq] + row0[seq + 1] - row0[seq];
            const int p = pos >> a.page_shift;
            const int pg = p < own ? a.table[(size_t)seq * a.ld + p] : stack_at(n_stack - 1 - t0[seq] - (p - own));
            if (pg >= 0 && pg < a.n_pages) slot = (pg << a.page_shift) + (pos & ((int)page - 1));
        }
        a.pos[r] = pos;
        a.slot[r] = slot;
        a.seq[r] = seq;
        a.lim[r] = lim;
    }
    if (rows) return;
    for (int b = gtid; b <= a.B; b += gn) a.row0[b] = row0[b];
    for (int b = gtid; b < a.B; b += gn)
        a.owned_out[b] = own_s[b] + (ok ? (t0[b + 1] - t0[b]) - (g0[b + 1] - g0[b]) : 0);
    if (ok) {
        const int n_take = t0[a.B], left = n_stack - n_take;
        for (int k = gtid; k < n_take; k += gn) {            // missing page k
            const int b = find(t0, k);
            a.table[(size_t)b * a.ld + own_s[b] + (k - t0[b])] = stack_at(n_stack - 1 - k);
        }
        for (int i = n_free + gtid; i < left; i += gn) a.free_[i] = stack_at(i);
    }
    if (gtid == 0) {
        *a.n_free_out = ok ? n_stack - t0[a.B] : n_free;
        a.status[0] = (int)min(total.rows, 0x7FFFFFFFll);
        a.status[1] = shortage;
        a.status[2] = ok ? 0 : 1;
    }
}

}  // namespace dllm
