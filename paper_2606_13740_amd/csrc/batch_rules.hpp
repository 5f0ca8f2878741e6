// Which launch a batch call gets, and the arithmetic that decides which memory it touches: plain C++, so that both are
// checked on the CPU.
#pragma once

#include <algorithm>

#include "../../include/dllm.h"
#include "arith.hpp"

namespace dllm {

constexpr int N_CU = 256;
inline int esize(int dtype) { return dtype == DLLM_F32 ? 4 : 2; }

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

constexpr int QK_VROWS = 64;                  // rows of a V workgroup

// Heads a lane group takes one after another: as many as leave 16384 groups (eight waves for every CU's
// worth of 8-lane groups), at most eight.
inline int qk_heads_per(long T, int H, int Hk) { return (int)std::min<long>(8, std::max<long>(1, T * (H + Hk) / 16384)); }
// Workgroups for Q and K, and with those for V.
inline long qk_wgs(long T, int H, int Hk, int Dh) {
    const int hp = qk_heads_per(T, H, Hk), per_wg = 256 / (Dh / 16);
    return (T * (ceil_div(H, hp) + ceil_div(Hk, hp)) + per_wg - 1) / per_wg;
}
inline long qk_grid(long T, int H, int Hk, int Dh) { return qk_wgs(T, H, Hk, Dh) + (long)ceil_div(T, QK_VROWS) * Hk; }

constexpr int MAX_ATTN_SPLITS = 64;           // key splits of a part

// Launch of an attention call.  Both parts (the shared prefix for all rows, and the sequences' own
// keys) run in one launch of one tile shape: QG row tiles of 16 QT rows (qt 2: one 32 x 32 tile a wave),
// a wave or, with up to two 16-row tiles of a 16-bit type, two waves each, which take a step's
// two blocks; waves without rows only help staging.
struct AttnPlan {
    int qg, qt;
    int shared;           // positions taken as the shared part
    int nt_s, ns_s;       // its row tiles and key splits per K/V head (0: no such part)
    int nt_o, ns_o;       // and of a sequence's own keys
    long wgs_s, wgs_o;
    bool direct() const { return ns_s == 0 && ns_o == 1; }
};

// Workgroups resident at once: two for every CU (their LDS, at head_dim 128).
constexpr int ATTN_SLOTS = 512;

// us with its merge, measured (bf16 / fp16, 28 heads over 4 or 32 over 32, head_dim 128, but where said):
//  - shared part or not: 16 x 1 rows behind 8192 keys 49 and 255; 16 x 3 behind 9984 26 and 38; 4 x 8 behind 2048
//    (13 MB that the sequences would read again) 16.7 and 17.8; 16 x 48 rows, 4 heads of 64, behind 512 (8 MB) equal;
//    8 x 1 behind 64 15.0 and 14.8.  With one sequence it is that sequence's own.
//  - tile: 64 rows against 128 (32 x 32 tiles): 12 x 40 rows of 32 heads behind 1024 37 and 40, 16 x 3 behind 9984 25.6
//    and 27.2, 6 x 20 rows of 16 heads of 64 behind 2976 13.6 and 14.8; from 12 steps of 128 rows a slot on
//    128 rows, which halve the LDS reads per product: 16 x 64 behind 16384 (56 steps) 186 and 145.  The border
//    lies lower for some calls: 8 x 32 of 32 heads behind 4096 (8 steps) 51.5 and 49.2, where the rule keeps 64 rows.  fp32 is bound by its products, where idle waves cost: by the rows of one sequence
//    (6 x 24 rows of 32 heads behind 1024: 32 rows 62, 64 rows 66).
//  - waves of a row tile, for tiles of 32 rows and fewer: two against one 46.5 and 48.7 (16 x 1 rows of 32 heads behind
//    8192), 20.9 and 22.8 (1 x 32 of 32 heads behind 4096), 5.6 and 6.2 (3 x 1 of 4 heads of 64 behind 80), 14.9 and 14.7
//    (8 x 1 behind 1564); 64 rows as two 32 x 32 tiles of two waves each against four of 16 rows: 50 and 51, 36.1
//    and 36.6, 25.7 and 25.6, 14.0 and 13.6 in the calls above: not taken.
//  - steps of a workgroup: all the call's steps (and two for each workgroup's start) over the slots, so that one
//    round takes them, rounded towards fewer workgroups: 16 x 64 behind 16384 in 4 splits (448 workgroups) 150, 3 174,
//    5 190; 8 x 32 of 32 heads behind 4096 in 3 splits 50, 2 62, 4 54; and at least four (two for tiles of 16 rows
//    and in fp32), since a split is written and merged: 4 x 8 behind 2048 in 8 splits of 4 steps 16.2, in 16 of 2 19.0.
//
// With masks (tree) the rows of a sequence are drafts, of which some sequences have many and some few or none: max_rows
// makes nt_o tiles for each, n_rows says how many of them can have rows.
inline AttnPlan attn_plan(const dllm_attn_args* g, bool tree = false) {
    const int G = g->n_heads / g->n_kv_heads, es = esize(g->dtype), step = es == 4 ? 32 : 64;
    AttnPlan p{};
    p.shared = std::min(g->shared_len, g->max_len);
    const long rows_o = (long)std::min(g->max_rows, g->n_rows) * G, rows_s = (long)g->n_rows * G;
    if ((long)(g->n_seqs - 1) * p.shared * g->n_kv_heads * g->head_dim * 2 * es < (8l << 20)) p.shared = 0;
    const int steps_s = ceil_div(p.shared, step), steps_o = std::max(1, ceil_div(g->max_len - p.shared, step));
    const long units_o = (long)g->n_seqs * g->n_kv_heads;
    const long rows = es == 4 || p.shared == 0 ? rows_o : std::max(rows_s, rows_o);
    p.qg = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    p.qt = 1;
    if (es == 2 && rows > 64 &&
        g->n_kv_heads * (rows_s / 128) * steps_s + units_o * (rows_o / 128) * steps_o >= 12 * ATTN_SLOTS)
        p.qt = 2;
    const int tm = 16 * p.qg * p.qt;
    p.nt_s = ceil_div(rows_s, tm);
    p.nt_o = std::max(1, ceil_div(rows_o, tm));
    // (rows behind the last sequence make no work: rows_s / tm, not rounded up)
    const double wgs_s = p.shared > 0 ? g->n_kv_heads * std::max(1.0, (double)rows_s / tm) : 0, wgs_o = tree ? g->n_kv_heads * std::min((double)g->n_seqs * p.nt_o, (double)rows_s / tm + 0.5 * g->n_seqs) : (double)units_o * p.nt_o;
    const double per = std::max((wgs_s * (steps_s + 2) + wgs_o * (steps_o + 2)) / ATTN_SLOTS, tm <= 16 || es == 4 ? 2.0 : 4.0);
    auto splits = [&](int steps) {
        const int ns = std::min(MAX_ATTN_SPLITS, std::max(1, (int)(steps / per + 0.25)));
        return ceil_div(steps, ceil_div(steps, ns));           // none empty
    };
    if (p.shared > 0) p.ns_s = splits(steps_s);
    p.ns_o = splits(steps_o);
    p.wgs_s = p.shared > 0 ? (long)g->n_kv_heads * p.nt_s * p.ns_s : 0;
    p.wgs_o = units_o * p.ns_o;
    if (tree) p.wgs_o = (p.wgs_o + 7) / 8 * 8;                 // (dealt to the XCDs one by one)
    p.wgs_o *= p.nt_o;
    return p;
}

inline size_t attn_ws_bytes(const dllm_attn_args* g, const AttnPlan& p) {
    if (p.direct()) return 0;
    return (size_t)(p.ns_s + p.ns_o) * g->n_rows * g->n_heads * (g->head_dim + 2) * 4;
}

// Threads and ids of a selection's workgroup, ids of a thread, rows loaded at once and at most.
constexpr int SEL_NT = 256, SEL_PT = 8, SEL_IDS = SEL_NT * SEL_PT, SEL_RB = 4, SEL_MAX_ROWS = 16;

// Ranges of SEL_IDS ids, and rows of a workgroup: as many as keep a sequence's tables and still leave
// 1024 workgroups, from four (the rows loaded at once) or, where that is less than one for every CU, two.
inline int select_ranges(int vocab) { return ceil_div(vocab, SEL_IDS); }
inline int select_rows_per(int T, int n_ranges) {
    const long per = (long)T * n_ranges / 1024;
    if ((long)T * n_ranges < 4 * N_CU) return 2;
    return (int)std::min<long>(SEL_MAX_ROWS, std::max<long>(SEL_RB, per / SEL_RB * SEL_RB));
}
inline long select_wgs(int T, int n_ranges) { return (long)n_ranges * ceil_div(T, select_rows_per(T, n_ranges)); }
inline bool select_four_waves(long wgs) { return wgs <= 4 * N_CU; }

// Words of a mask row in the plan of trees, whose LDS holds 32 rows a word.
constexpr int TREE_MAX_LD = DLLM_MAX_TREE / 32;

// Threads of a log probability workgroup, logits of a lane, ids of a wave's block.
constexpr int LP_NT = 256, LP_PT = 32, LP_BLOCK = 64 * LP_PT;
static_assert(DLLM_MAX_TOP <= 64, "a row's best ids are a lane's each");

// Blocks of a part of a row: whole rounds of the four waves, as many as leave 1024 workgroups (four for every CU).  A call in
// us with parts for 256, 512, 768, 1024 and 2048 workgroups: 256 rows of 152064 bf16 logits 39.6, 30.1, 28.0, 28.3, 31.3, 300 rows 42.2,
// 42.7, 34.3, 32.2, 32.3, 128 rows 26.7, 22.1, 21.6, 22.0, 24.4; 256 of 126464 fp32 36.1, 30.4, 33.0, 32.6, 33.4, 64 rows 16.7, 15.6,
// 15.5, 16.2, 16.1; 1000 of 50000 bf16 30 with one part each, 37.4 with two; 32 of 126464, 8 and 64 of 32000 and 600 of
// 152064 within 3%.
inline int lp_per(int T, int vocab) {
    const int blocks = ceil_div(vocab, LP_BLOCK), waves = LP_NT / 64;
    const long parts = std::max<long>(1, 4 * N_CU / std::max(T, 1));
    return waves * ceil_div(ceil_div(blocks, parts), waves);
}
inline int lp_parts(int T, int vocab) { return ceil_div(ceil_div(vocab, LP_BLOCK), lp_per(T, vocab)); }
inline size_t lp_ws_bytes(int T, int vocab, int top) {
    const int parts = lp_parts(T, vocab);
    return parts == 1 ? 0 : (size_t)T * parts * (LP_NT / 64) * (16 + 8 * (size_t)top);
}
// Given tokens whose rows are named: every row's workgroup looks through a short list, and a long one gets a launch of its
// own once the rows' sums are in the workspace (8 bytes a row).  That launch takes 1.2 us; a list costs a row 0.4 us for each
// 256 tokens and the chip 1 us for each 2^20 (row, token): 32 rows of 126464 and 1024 tokens 13.5 us searched, 13.8 apart, 2048 tokens
// 15.2 and 13.7; 2048 rows of 1024 and 512 tokens 15.7 and 16.2, 1024 tokens 16.9 and 16.2; 16384 rows of 1024 and 64 tokens 92.4
// and 91.3, 16384 tokens 339 and 93.
constexpr int LP_SEARCHED = 1024;
constexpr long LP_SEARCHED_ALL = 1l << 20;
inline bool lp_tokens_apart(int T, int n_tok, bool named) {
    return named && (n_tok > LP_SEARCHED || (long)T * n_tok > LP_SEARCHED_ALL);
}

// Heads (of all layers) of a compaction's workgroup for V^T: as many as leave 1536 workgroups (six for every CU, which its
// registers hold), at most eight; and workgroups, with K's of COMPACT_NT lanes of 16 bytes.  With 1, 2, 3, 4, 6 and 8 heads, fp16:
// 32 trees of 64 rows, 28 layers of 4 heads 34.6, 32.6, 33.2, 33.1, 33.9, 33.9 us (the rule's 2), 16 trees 18.0, 17.3, 16.4, 17.3, 17.1, 16.7
// (1), 64 trees 81.5, 81.7, 84.6, 84.5, 84.0, 86.3 (4); 32 trees, 24 layers of 8 heads of 64 23.1, 21.7, 22.8, 21.9, 23.4, 23.1 (4); 32
// layers of 32 heads 354 with one, 361 to 365 with more (8).
constexpr int COMPACT_NT = 256;
inline int compact_heads_per(long B, int L, int Hk) { return (int)std::min<long>(8, std::max<long>(1, B * L * Hk / (6 * N_CU))); }
inline long compact_wgs(long B, int L, int Hk, int Dh, int es) {
    return B * (ceil_div((long)L * Hk * (Dh * es / 16), COMPACT_NT) + ceil_div((long)L * Hk, compact_heads_per(B, L, Hk)));
}

// Threads of a fork's workgroup, and pages whose marks its LDS holds (beside 48 KB of the sequences').
constexpr int FORK_NT = 1024, FORK_LDS_PAGES = 27 * 1024;
// The copies' count (16 bytes), their list, the new tables' sources, and the marks where they do not fit.
inline size_t fork_ws_bytes(int n_seqs, int n_pages) {
    return 16 + (size_t)n_seqs * 24 + (n_pages > FORK_LDS_PAGES ? (size_t)n_pages * 4 : 0);
}

}  // namespace dllm
