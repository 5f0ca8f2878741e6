// Moves inside a paged K/V cache: accepted rows behind their sequence's text, and sequences that go on as copies of
// others.
#pragma once

#include "batch_rules.hpp"
#include "common.hpp"

namespace dllm {

// A cache of all layers: [layers][K, V^T][n_pages][Hk][page * Dh].
struct CacheArgs {
    char* pages;
    int L, Hk, Dh, page_shift, n_pages;
};

// Base of head hk of page pg in a plane (0 K, 1 V^T) of layer l, in bytes.
template <int ES> __device__ __forceinline__ char* head_of(const CacheArgs& c, int l, int plane, int pg, int hk) {
    return c.pages + (((((size_t)l * 2 + plane) * c.n_pages + pg) * c.Hk + hk) * ((size_t)c.Dh << c.page_shift)) * ES;
}

struct CompactArgs {
    CacheArgs c;
    const int* table;
    int ld;
    const int* base;
    const int* path;
    int path_ld;
    const int* n;
    int B;
};

// Position base + path[i] to base + i, for i < n: path ascends, so path[i] >= i and a chunk's destinations lie before the
// sources of the chunks behind it: load a chunk, wait, store it, in place.
//
// A workgroup takes one sequence's K of as many heads (of all layers) as have 16 bytes for each of its lanes, or its V^T of hp
// heads.  K: a position is Dh consecutive elements of each head; a lane takes the positions in chunks of eight.  V^T: a position is a
// column; 16 lanes have 16 positions of a dim, which lie in one or two lines of its page, and are read and written
// together.  Either way a chunk's source and destinations are one wave's, which needs no barrier.
//
// What bounds it: V^T, of which a position is 2 or 4 bytes of a line for every dim.  32 trees of 64 rows, 28 layers of 4 heads,
// fp16, 7 MB moved: 36 us, of which K takes 5.  49 MB are fetched and 28 written, 16 us at a copy's rate; the rest is instructions, a
// load and a store for every element of V^T, many to a part of a line that others write too (the waves are ready and wait to
// issue for 63% of their cycles).  fp32: 62 us.  Small calls: four dependent loads (4.9 us).
constexpr int COMPACT_POS = 16, COMPACT_K = 8;
template <typename E, int DH>
__global__ void __launch_bounds__(COMPACT_NT) cache_compact_kernel(CompactArgs a, int hp) {
    constexpr int ES = sizeof(E);
    __shared__ int src_s[DLLM_MAX_TREE], dst_s[DLLM_MAX_TREE], end_s;       // slots (page id * page + offset), -1: not moved
    constexpr int LP = DH * ES / 16;                      // lanes of a head's position
    const int tid = threadIdx.x, heads = a.c.L * a.c.Hk;  // (head u is head u % Hk of layer u / Hk)
    // K's workgroups first: they are few and short, and next to V^T's those wait for less
    const int k_parts = (heads * LP + COMPACT_NT - 1) / COMPACT_NT, v_parts = (heads + hp - 1) / hp;
    const bool is_k = (int)blockIdx.x < k_parts * a.B;
    const int at0 = is_k ? blockIdx.x : blockIdx.x - k_parts * a.B, parts = is_k ? k_parts : v_parts;
    const int part = at0 % parts, b = at0 / parts;
    const int n = min(max(a.n[b], 0), a.path_ld), base = a.base[b];
    if (n == 0 || base < 0) return;
    if (tid == 0) end_s = n;
    __syncthreads();
    const int page = 1 << a.c.page_shift;
    const long top = (long)a.ld << a.c.page_shift;        // positions of a table
    auto slot_of = [&](int p) {
        const int pg = a.table[(size_t)b * a.ld + (p >> a.c.page_shift)];
        return pg >= 0 && pg < a.c.n_pages ? (pg << a.c.page_shift) + (p & (page - 1)) : -1;
    };
    bool moved = false;
    for (int i = tid; i < n; i += COMPACT_NT) {
        const int p = a.path[(size_t)b * a.path_ld + i], before = i > 0 ? a.path[(size_t)b * a.path_ld + i - 1] : -1;
        // (an ascending path that starts at 0 or later has path[i] >= i; what is behind an entry that breaks it is not read)
        if (p <= before || p < i || (long)base + p >= top) {
            atomicMin(&end_s, i);
            continue;
        }
        const int from = slot_of(base + p), to = slot_of(base + i);
        const bool go = from >= 0 && to >= 0 && from != to;
        src_s[i] = go ? from : -1;
        dst_s[i] = to;
        moved |= go;
    }
    if (!__syncthreads_or(moved)) return;
    const int m = end_s;
    if (is_k) {
        const int c = part * COMPACT_NT + tid, u = c / LP;
        if (u >= heads) return;
        auto at = [&](int s) {
            return (u32x4_t*)(head_of<ES>(a.c, u / a.c.Hk, 0, s >> a.c.page_shift, u % a.c.Hk) + (size_t)(s & (page - 1)) * (DH * ES)) + c % LP;
        };
        for (int i0 = 0; i0 < m; i0 += COMPACT_K) {
            u32x4_t v[COMPACT_K];
            int from[COMPACT_K];
#pragma unroll
            for (int k = 0; k < COMPACT_K; ++k) {
                from[k] = i0 + k < m ? src_s[i0 + k] : -1;
                if (from[k] >= 0) v[k] = *at(from[k]);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int k = 0; k < COMPACT_K; ++k)
                if (from[k] >= 0) *at(dst_s[i0 + k]) = v[k];
        }
        return;
    }
    constexpr int ND = COMPACT_NT / COMPACT_POS, PASS = DH / ND;
    const int u1 = min(heads, (part + 1) * hp), dim = tid / COMPACT_POS;
    for (int i0 = 0; i0 < m; i0 += COMPACT_POS) {
        const int i = i0 + tid % COMPACT_POS, from = i < m ? src_s[i] : -1;
        if (from < 0) continue;
        const int to = dst_s[i];
        auto at = [&](int s, int u) {
            return (E*)head_of<ES>(a.c, u / a.c.Hk, 1, s >> a.c.page_shift, u % a.c.Hk) + (s & (page - 1)) + ((size_t)dim << a.c.page_shift);
        };
        for (int u = part * hp; u < u1; u += 2) {
            const int other = min(u + 1, u1 - 1);         // (two heads' loads at once; the last one alone twice)
            const E *p0 = at(from, u), *p1 = at(from, other);
            E v[2][PASS];
#pragma unroll
            for (int k = 0; k < PASS; ++k) {
                v[0][k] = p0[(size_t)(k * ND) << a.c.page_shift];
                v[1][k] = p1[(size_t)(k * ND) << a.c.page_shift];
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            E *q0 = at(to, u), *q1 = at(to, other);
#pragma unroll
            for (int k = 0; k < PASS; ++k) {
                q0[(size_t)(k * ND) << a.c.page_shift] = v[0][k];
                q1[(size_t)(k * ND) << a.c.page_shift] = v[1][k];
            }
        }
    }
}

// Entries j .. j + 3 of a table's row (as far as they are below n; the others -1).
__device__ __forceinline__ int4 table4(const int* row, int j, int n, bool vec) {
    int4 v = make_int4(-1, -1, -1, -1);
    if (j >= n) return v;
    if (vec) {
        v = *(const int4*)(row + j);
    } else {
        v.x = row[j];
        if (j + 1 < n) v.y = row[j + 1];
        if (j + 2 < n) v.z = row[j + 2];
        if (j + 3 < n) v.w = row[j + 3];
    }
    return v;
}

struct ForkArgs {
    const int *src, *keep, *owned;
    int* owned_out;
    const int* table;
    int ld;
    bool vec;                     // rows of the table are whole 16-byte vectors
    int* free_;
    const int* n_free;
    int *n_free_out, *status;
    int B, n_pages, page_shift, shared;
    int* n_copies;                // workspace: how many,
    int4* copies;                 // (page from, page to, positions) of each,
    uint2* rows;                  // a new table's source | entries << 12, and the last entry's own page or -1,
    uint32_t* marks;              // [n_pages] where they do not fit the LDS
};

// Tables of sequences that go on as copies of others, and pages nobody has any more.
//
// With one mark a page everything is a minimum: 0 where some sequence goes on with the page whole, 1 + b where b is
// the first that goes on with a part of it, HELD where it only was in a table, FREE else.  A part is copied where the mark is
// less than the sequence's own 1 + b, a page is given back where it is HELD.  In order, pages given back are pushed onto the
// stack and copies' pages are popped off it.
//
// One workgroup does it, with the marks in LDS (or, for large pools, in the workspace): no launch waits for
// another's.  What bounds it: dependent loads.  A wave takes as many sequences at once as have room in its lanes, four
// entries a lane, four times over, so that one round trip brings up to 1024 entries (one sequence at a time: 512
// sequences of up to 47 pages 40 us, 14 so).  The new tables are written by the launch that copies the pages, on the whole chip.
constexpr uint32_t FORK_HELD = 0xFFFFFFFEu, FORK_FREE = 0xFFFFFFFFu;
template <bool LDS>
__global__ void __launch_bounds__(FORK_NT) batch_fork_kernel(ForkArgs a) {
    constexpr int NW = FORK_NT / 64, PER = DLLM_MAX_SEQS / FORK_NT, BATCH = 4;
    __shared__ int fresh_s[DLLM_MAX_SEQS];                // page of copy c
    __shared__ uint32_t to_s[DLLM_MAX_SEQS];              // source | pages needed << 12 | (whole pages only) << 31
    __shared__ int own_s[DLLM_MAX_SEQS];                  // pages owned; in a granted fork then copy of sequence b, or -1
    __shared__ int wsum[NW], gsum[NW], most_s[NW];
    extern __shared__ uint32_t marks_lds[];
    uint32_t* marks = LDS ? marks_lds : a.marks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_free = *a.n_free, in_page = (1 << a.page_shift) - 1;
    static_assert(DLLM_MAX_SEQS <= 1 << 12, "a source has 12 bits");

    // PER consecutive sequences a thread (as few as hold them all)
    const int per = (a.B + FORK_NT - 1) / FORK_NT;
    int src[PER], keep[PER], own[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = min(tid * per + k, a.B - 1);
        src[k] = a.src[b];
        keep[k] = a.keep[b];
        own[k] = a.owned[b];
    }
    for (int i = tid; i < a.n_pages; i += FORK_NT) {
        if (LDS) marks[i] = FORK_FREE;
        else __hip_atomic_store(&marks[i], FORK_FREE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // (what is out of range is cut here, so that the tables may be read before all sequences' checks are in)
    bool bad = n_free < 0 || n_free > a.n_pages;
    int longest = 0, part[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * per + k;
        part[k] = -1;
        if (k >= per || b >= a.B) continue;
        const long need = ((long)max(keep[k], 0) + in_page) >> a.page_shift;
        bad |= src[k] < 0 || src[k] >= a.B || keep[k] < 0 || own[k] < 0 || own[k] > a.ld || need > a.ld;
        const int s = min(max(src[k], 0), a.B - 1), n = (int)min(need, (long)a.ld), o = min(max(own[k], 0), a.ld);
        const bool whole = (keep[k] & in_page) == 0;
        to_s[b] = (uint32_t)s | (uint32_t)n << 12 | (whole ? 0x80000000u : 0u);
        own_s[b] = o;
        longest = max(longest, max(n, o));
        if (!whole && n > a.shared) part[k] = a.table[(size_t)s * a.ld + n - 1];        // the page kept in part
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o));
    if (lane == 0) most_s[wave] = longest;
    if (!LDS) __threadfence();                            // (a barrier alone does not wait for memory)
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) longest = max(longest, most_s[w]);
    // lanes of a sequence: a power of two, as many as the longest table has groups of four pages
    const int most = longest, quads = (most + 3) >> 2, lp = quads > 1 ? min(6, 32 - __builtin_clz(quads - 1)) : 0;
    const int per_wave = 64 >> lp, sub = lane >> lp, col = 4 * (lane & ((1 << lp) - 1));
    auto source = [&](uint32_t to) { return (int)(to & 0xFFF); };
    auto need_of = [&](uint32_t to) { return (int)(to >> 12 & 0x7FFFF); };
    auto mark = [&](int pg, uint32_t m) {
        if (pg < 0 || pg >= a.n_pages) return;
        if (LDS) atomicMin(&marks[pg], m);
        else __hip_atomic_fetch_min(&marks[pg], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    auto mark_at = [&](int pg) { return LDS ? marks[pg] : __hip_atomic_load(&marks[pg], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    for (int b0 = wave * per_wave * BATCH; b0 < a.B; b0 += NW * per_wave * BATCH) {
        for (int j0 = a.shared & ~3; j0 < most; j0 += 4 << lp) {
            const int j = j0 + col;
            int4 was[BATCH], now[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int b = min(b0 + k * per_wave + sub, a.B - 1);
                const uint32_t to = to_s[b];
                was[k] = table4(a.table + (size_t)b * a.ld, j, own_s[b], a.vec);
                now[k] = table4(a.table + (size_t)source(to) * a.ld, j, need_of(to), a.vec);
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int b = min(b0 + k * per_wave + sub, a.B - 1);           // (the last one again: the same marks)
                const uint32_t to = to_s[b];
                const int n_own = own_s[b], need = need_of(to);
                const int w[4] = {was[k].x, was[k].y, was[k].z, was[k].w}, n[4] = {now[k].x, now[k].y, now[k].z, now[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (j + e < a.shared) continue;
                    if (j + e < n_own) mark(w[e], FORK_HELD);
                    if (j + e < need) mark(n[e], j + e < need - 1 || to >> 31 ? 0u : 1u + b);
                }
            }
        }
    }
    // no sequence keeps more than its source has
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * per + k;
        if (k < per && b < a.B) bad |= need_of(to_s[b]) > own_s[source(to_s[b])];
    }
    if (!LDS) __threadfence();
    const bool any_bad = __syncthreads_or(bad);

    // copies, numbered by sequence
    int mine = 0;
    uint32_t is_copy = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (!any_bad && part[k] >= 0 && part[k] < a.n_pages && mark_at(part[k]) < 1u + tid * per + k) {
            is_copy |= 1u << k;
            ++mine;
        }
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(inc, o);
        if (lane >= o) inc += up;
    }
    // pages given back: a wave counts a run of pages
    const int run = (((a.n_pages + NW - 1) / NW) + 255) & ~255, p0 = wave * run, p1 = min(a.n_pages, p0 + run);
    int gone = 0;
    if (!any_bad) {
        for (int p = p0; p < p1; p += 256) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = p + 64 * k + lane;
                gone += __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < p1 && mark_at(min(at, a.n_pages - 1)) == FORK_HELD));
            }
        }
    }
    if (lane == 63) wsum[wave] = inc;
    if (lane == 0) gsum[wave] = gone;
    __syncthreads();
    int at = inc - mine, g0 = 0, n_copy = 0, n_gone = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) {
            at += wsum[w];
            g0 += gsum[w];
        }
        n_copy += wsum[w];
        n_gone += gsum[w];
    }
    const int stack = n_free + n_gone, shortage = max(n_copy - stack, 0);
    const bool ok = !any_bad && shortage == 0 && stack <= a.n_pages;
    const int left = stack - n_copy;
    if (ok) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int b = tid * per + k;
            if (k >= per || b >= a.B) break;
            const bool is = is_copy >> k & 1;
            own_s[b] = is ? at : -1;
            if (is) a.copies[at] = make_int4(part[k], -1, keep[k] & in_page, 0);       // (the page follows)
            at += is;
        }
        // page g of those given back is entry n_free + g of the stack, copy c's page its entry stack - 1 - c
        for (int p = p0; p < p1; p += 256) {
            bool is[4];
            uint64_t who[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int pg = p + 64 * k + lane;
                is[k] = pg < p1 && mark_at(min(pg, a.n_pages - 1)) == FORK_HELD;
                who[k] = __builtin_amdgcn_ballot_w64(is[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (is[k]) {
                    const int i = n_free + g0 + __builtin_amdgcn_mbcnt_hi((uint32_t)(who[k] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who[k], 0));
                    if (i < left) a.free_[i] = p + 64 * k + lane;
                    else fresh_s[stack - 1 - i] = p + 64 * k + lane;
                }
                g0 += __builtin_popcountll(who[k]);
            }
        }
        for (int c = tid; c < n_copy; c += FORK_NT)
            if (stack - 1 - c < n_free) fresh_s[c] = a.free_[stack - 1 - c];
    }
    __syncthreads();
    for (int c = tid; ok && c < n_copy; c += FORK_NT) a.copies[c].y = fresh_s[c];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * per + k;
        if (k >= per || b >= a.B) break;
        const uint32_t to = ok ? to_s[b] & 0x7FFFFFFFu : (uint32_t)b | (uint32_t)min(max(own[k], 0), a.ld) << 12;
        const int c = ok ? own_s[b] : -1;
        a.rows[b] = make_uint2(to, c >= 0 ? (uint32_t)fresh_s[c] : 0xFFFFFFFFu);
        a.owned_out[b] = ok ? need_of(to) : own[k];
    }
    if (tid == 0) {
        *a.n_copies = ok ? n_copy : 0;
        *a.n_free_out = ok ? left : n_free;
        a.status[0] = n_copy;
        a.status[1] = shortage;
        a.status[2] = ok ? 0 : 1;
    }
}

// A fork's new tables, a wave a sequence, and its copies: positions [0, n) of a page, of every layer, plane and head, a
// workgroup each; what lies past the positions stays.  8 sequences, 28 layers: 6 MB in 6.5 us, four dependent loads.
template <typename E, int DH>
__global__ void __launch_bounds__(256) fork_copy_kernel(CacheArgs c, const int* n_copies, const int4* copies, const uint2* rows, int B,
                                                        const int* table, int* table_out, int ld, bool vec) {
    constexpr int ES = sizeof(E), VE = 16 / ES;
    const int units = c.L * 2 * c.Hk, tid = threadIdx.x;
    // (the first job is asked for beside their number)
    int4 job = copies[min((int)(blockIdx.x / units), B - 1)];
    const long n = (long)min(*n_copies, B) * units;
    // (from the grid's end: a fork rarely copies for all sequences)
    for (int b = (gridDim.x - 1 - blockIdx.x) * 4 + (tid >> 6); b < B; b += gridDim.x * 4) {
        const uint2 to = rows[b];
        const int len = to.x >> 12 & 0x7FFFF;
        const int *src = table + (size_t)(to.x & 0xFFF) * ld;
        int* dst = table_out + (size_t)b * ld;
        for (int j = 4 * (tid & 63); j < len; j += 256) {
            int4 v = table4(src, j, len, vec);
            if ((int)to.y >= 0 && j + 4 >= len) {         // the last entry is a copy's
                const int e = len - 1 - j, own = (int)to.y;
                v = make_int4(e == 0 ? own : v.x, e == 1 ? own : v.y, e == 2 ? own : v.z, e == 3 ? own : v.w);
            }
            if (vec && j + 4 <= len) {
                *(int4*)(dst + j) = v;
            } else {
                dst[j] = v.x;
                if (j + 1 < len) dst[j + 1] = v.y;
                if (j + 2 < len) dst[j + 2] = v.z;
                if (j + 3 < len) dst[j + 3] = v.w;
            }
        }
    }
    for (long u = blockIdx.x; u < n; u += gridDim.x) {
        if (u >= gridDim.x) job = copies[u / units];
        if ((unsigned)job.x >= (unsigned)c.n_pages || (unsigned)job.y >= (unsigned)c.n_pages) continue;
        const int r = (int)(u % units), hk = r % c.Hk, plane = r / c.Hk & 1, l = r / c.Hk / 2, np = job.z;
        const char* from = head_of<ES>(c, l, plane, job.x, hk);
        char* to = head_of<ES>(c, l, plane, job.y, hk);
        if (plane == 0) {
            const int vecs = np * (DH * ES / 16);
            for (int i0 = tid; i0 < vecs; i0 += 4 * 256) {
                u32x4_t v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = ((const u32x4_t*)from)[min(i0 + 256 * k, vecs - 1)];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + 256 * k < vecs) ((u32x4_t*)to)[i0 + 256 * k] = v[k];
            }
        } else {
            const int rs = c.page_shift - (ES == 2 ? 3 : 2), vecs = DH << rs;      // (16-byte vectors of a dim: 2^rs)
            for (int i0 = tid; i0 < vecs; i0 += 4 * 256) {
                u32x4_t v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + 256 * k, p = (i & ((1 << rs) - 1)) * VE;
                    if (i < vecs && p < np) v[k] = ((const u32x4_t*)from)[i];
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + 256 * k, p = (i & ((1 << rs) - 1)) * VE;
                    if (i >= vecs || p >= np) continue;
                    if (p + VE <= np) {
                        ((u32x4_t*)to)[i] = v[k];
                    } else {
                        E e[VE];
                        __builtin_memcpy(e, &v[k], 16);
#pragma unroll
                        for (int j = 0; j < VE; ++j)
                            if (p + j < np) ((E*)to)[(size_t)i * VE + j] = e[j];
                    }
                }
            }
        }
    }
}

}  // namespace dllm
