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
// A workgroup takes one plane of one head of one layer of one sequence.  K: a position is Dh consecutive
// elements, 16 bytes a lane.  V^T: a position is a column: 16 positions by 16 dims at a time, so that a dim's positions,
// which lie in one or two lines of its page, are read and written together.
constexpr int COMPACT_NT = 256, COMPACT_POS = 16;
template <typename E, int DH>
__global__ void __launch_bounds__(COMPACT_NT) cache_compact_kernel(CompactArgs a) {
    constexpr int ES = sizeof(E);
    __shared__ int src_s[1024], dst_s[1024], end_s;       // slots (page id * page + offset), -1: no page
    const int tid = threadIdx.x;
    const int hk = blockIdx.x % a.c.Hk, i1 = blockIdx.x / a.c.Hk, plane = i1 & 1, i2 = i1 >> 1, l = i2 % a.c.L, b = i2 / a.c.L;
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
        src_s[i] = slot_of(base + p);
        dst_s[i] = slot_of(base + i);
        if (src_s[i] == dst_s[i]) src_s[i] = -1;
        moved |= src_s[i] >= 0;
    }
    const int some = __syncthreads_or(moved);
    const int m = end_s;
    if (!some) return;
    if (plane == 0) {
        constexpr int LP = DH * ES / 16, PER = COMPACT_NT / LP;      // lanes of a position, positions at a time
        for (int i0 = 0; i0 < m; i0 += PER) {
            const int i = i0 + tid / LP;
            const bool go = i < m && src_s[i] >= 0 && dst_s[i] >= 0;
            u32x4_t v{};
            auto at = [&](int s) {
                return (u32x4_t*)(head_of<ES>(a.c, l, 0, s >> a.c.page_shift, hk) + (size_t)(s & (page - 1)) * (DH * ES)) + tid % LP;
            };
            if (go) v = *at(src_s[i]);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(v) : : "memory");
            __syncthreads();
            if (go) *at(dst_s[i]) = v;
        }
    } else {
        constexpr int ND = COMPACT_NT / COMPACT_POS, PASS = DH / ND;
        for (int i0 = 0; i0 < m; i0 += COMPACT_POS) {
            const int i = i0 + tid % COMPACT_POS, dim = tid / COMPACT_POS;
            const bool go = i < m && src_s[i] >= 0 && dst_s[i] >= 0;
            E v[PASS];
            auto at = [&](int s) { return (E*)head_of<ES>(a.c, l, 1, s >> a.c.page_shift, hk) + (s & (page - 1)) + ((size_t)dim << a.c.page_shift); };
            if (go) {
                const E* from = at(src_s[i]);
#pragma unroll
                for (int k = 0; k < PASS; ++k) v[k] = from[(size_t)(k * ND) << a.c.page_shift];
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (go) {
                E* to = at(dst_s[i]);
#pragma unroll
                for (int k = 0; k < PASS; ++k) to[(size_t)(k * ND) << a.c.page_shift] = v[k];
            }
        }
    }
}

struct ForkArgs {
    const int *src, *keep, *owned;
    int* owned_out;
    const int* table;
    int* table_out;
    int ld;
    int* free_;
    const int* n_free;
    int *n_free_out, *status;
    int B, n_pages, page_shift, shared;
    int* n_copies;                // workspace: how many,
    int4* copies;                 // and (page from, page to, positions) of each
    uint32_t* marks;              // [n_pages] where they do not fit the LDS
};

// Tables of sequences that go on as copies of others, and pages nobody has any more.
//
// With one mark a page everything is a minimum: 0 where some sequence goes on with the page whole, 1 + b where b is
// the first that goes on with a part of it, HELD where it only was in a table, FREE else.  A part is copied where the mark is
// less than the sequence's own 1 + b, a page is given back where it is HELD.  In order, pages given back are pushed onto the
// stack and copies' pages are popped off it.  One workgroup does it: the tables are read twice and the marks once.
constexpr uint32_t FORK_HELD = 0xFFFFFFFEu, FORK_FREE = 0xFFFFFFFFu;
template <bool LDS>
__global__ void __launch_bounds__(FORK_NT) batch_fork_kernel(ForkArgs a) {
    constexpr int NW = FORK_NT / 64, PER = DLLM_MAX_SEQS / FORK_NT;
    __shared__ int fresh_s[DLLM_MAX_SEQS];               // page of copy c
    __shared__ int copy_s[DLLM_MAX_SEQS];                 // copy of sequence b, or -1
    __shared__ int wsum[NW], gsum[NW];
    extern __shared__ uint32_t marks_lds[];
    uint32_t* marks = LDS ? marks_lds : a.marks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_free = *a.n_free;

    for (int i = tid; i < a.n_pages; i += FORK_NT) {
        if (LDS) marks[i] = FORK_FREE;
        else __hip_atomic_store(&marks[i], FORK_FREE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // PER consecutive sequences a thread (as few as hold them all)
    const int per = (a.B + FORK_NT - 1) / FORK_NT;
    bool bad = n_free < 0 || n_free > a.n_pages;
    for (int k = 0; k < per; ++k) {
        const int b = tid * per + k;
        if (b >= a.B) break;
        const int s = a.src[b], kp = a.keep[b], own = a.owned[b];
        bad |= s < 0 || s >= a.B || kp < 0 || own < 0 || own > a.ld;
        if (s >= 0 && s < a.B && kp >= 0) {
            const long need = ((long)kp + (1l << a.page_shift) - 1) >> a.page_shift;
            bad |= need > a.owned[s];
        }
    }
    if (!LDS) __threadfence();                            // (a barrier alone does not wait for memory)
    const bool any_bad = __syncthreads_or(bad);
    auto need_of = [&](int keep) { return (int)(((long)keep + (1l << a.page_shift) - 1) >> a.page_shift); };
    auto mark = [&](int pg, uint32_t m) {
        if (pg < 0 || pg >= a.n_pages) return;
        if (LDS) atomicMin(&marks[pg], m);
        else __hip_atomic_fetch_min(&marks[pg], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    auto mark_at = [&](int pg) { return LDS ? marks[pg] : __hip_atomic_load(&marks[pg], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (!any_bad) {
        for (int b = wave; b < a.B; b += NW) {
            const int s = a.src[b], kp = a.keep[b], own = a.owned[b], need = need_of(kp);
            const bool whole = (kp & ((1 << a.page_shift) - 1)) == 0;
            for (int j = a.shared + lane; j < max(own, need); j += 64) {
                if (j < own) mark(a.table[(size_t)b * a.ld + j], FORK_HELD);
                if (j < need) mark(a.table[(size_t)s * a.ld + j], j < need - 1 || whole ? 0u : 1u + b);
            }
        }
    }
    if (!LDS) __threadfence();
    __syncthreads();

    // copies, numbered by sequence
    int mine = 0;
    uint32_t is_copy = 0;
    if (!any_bad) {
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= a.B) break;
            const int kp = a.keep[b], need = need_of(kp);
            if ((kp & ((1 << a.page_shift) - 1)) != 0 && need > a.shared) {
                const int pg = a.table[(size_t)a.src[b] * a.ld + need - 1];
                if (pg >= 0 && pg < a.n_pages && mark_at(pg) < 1u + b) {
                    is_copy |= 1u << k;
                    ++mine;
                }
            }
        }
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(inc, o);
        if (lane >= o) inc += up;
    }
    // pages given back: a wave counts a run of pages
    const int run = (((a.n_pages + NW - 1) / NW) + 63) & ~63, p0 = wave * run, p1 = min(a.n_pages, p0 + run);
    int gone = 0;
    if (!any_bad) {
        for (int p = p0; p < p1; p += 64) gone += __builtin_popcountll(__builtin_amdgcn_ballot_w64(p + lane < p1 && mark_at(p + lane) == FORK_HELD));
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
    for (int k = 0; k < per; ++k) {
        const int b = tid * per + k;
        if (b >= a.B) break;
        copy_s[b] = (is_copy >> k & 1) ? at++ : -1;
    }
    if (ok) {
        // page g of those given back is entry n_free + g of the stack, copy c's page its entry stack - 1 - c
        for (int p = p0; p < p1; p += 64) {
            const bool is = p + lane < p1 && mark_at(p + lane) == FORK_HELD;
            const uint64_t who = __builtin_amdgcn_ballot_w64(is);
            if (is) {
                const int i = n_free + g0 + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                if (i < left) a.free_[i] = p + lane;
                else fresh_s[stack - 1 - i] = p + lane;
            }
            g0 += __builtin_popcountll(who);
        }
        for (int c = tid; c < n_copy; c += FORK_NT)
            if (stack - 1 - c < n_free) fresh_s[c] = a.free_[stack - 1 - c];
    }
    __syncthreads();
    for (int b = wave; b < a.B; b += NW) {
        const int s = ok ? a.src[b] : b, own = any_bad ? min(max(a.owned[b], 0), a.ld) : a.owned[b], kp = a.keep[b];
        const int n = ok ? need_of(kp) : own, c = ok ? copy_s[b] : -1;
        const int fresh = c >= 0 ? fresh_s[c] : 0;
        for (int j = lane; j < n; j += 64) {
            const int pg = a.table[(size_t)s * a.ld + j];
            const bool copied = c >= 0 && j == n - 1;
            a.table_out[(size_t)b * a.ld + j] = copied ? fresh : pg;
            if (copied) a.copies[c] = make_int4(pg, fresh, kp & ((1 << a.page_shift) - 1), 0);
        }
        if (lane == 0) a.owned_out[b] = ok ? n : a.owned[b];
    }
    if (tid == 0) {
        *a.n_copies = ok ? n_copy : 0;
        *a.n_free_out = ok ? left : n_free;
        a.status[0] = n_copy;
        a.status[1] = shortage;
        a.status[2] = ok ? 0 : 1;
    }
}

// The copies of a fork: positions [0, n) of a page, of every layer, plane and head.  A wave takes 2 KB of K or
// of V^T's rows; what lies past the positions stays.
template <typename E, int DH>
__global__ void __launch_bounds__(256) cache_copy_kernel(CacheArgs c, const int* n_copies, const int4* copies, int B) {
    constexpr int ES = sizeof(E), VE = 16 / ES;
    const int n = min(*n_copies, B), units = c.L * 2 * c.Hk, tid = threadIdx.x;
    for (long u = blockIdx.x; u < (long)n * units; u += gridDim.x) {
        const int4 job = copies[u / units];
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
