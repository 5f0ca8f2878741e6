// Penalties, biases and masks on logits, then the id of the largest and its confidence.
#pragma once

#include <float.h>

#include <type_traits>

#include "attn_paged.hpp"
#include "batch_rules.hpp"
#include "common.hpp"
#include "qk_rope.hpp"

namespace dllm {

struct SelectArgs {
    const void* logits;
    long ld;
    int T, V, mask_id, B;
    const int *row0, *hist, *hist0, *n_prompt;
    const float *rep, *pres, *freq;
    const int* bias_id;
    const float* bias;
    const int* bias0;
    const uint32_t* allow;
    int n_allow, allow_ld;
    const int* allow_row;
    void* out;
    long ld_out;
    int* out_id;
    float* out_conf;
};

// Best id of a set of logits: (largest value, lowest id of it, sum of exp(l - largest)).
struct Best {
    float mx;
    int id;
    float s;
};
__device__ __forceinline__ Best best_merge(const Best& a, const Best& b) {
    if (b.id < 0) return a;
    if (a.id < 0) return b;
    const float mx = fmaxf(a.mx, b.mx);
    const int id = a.mx > b.mx ? a.id : (b.mx > a.mx ? b.id : min(a.id, b.id));
    return Best{mx, id, a.s * expf(a.mx - mx) + b.s * expf(b.mx - mx)};
}

// A logit after its sequence's penalties and bias (0: none); e: the id's table entry.  Separate
// roundings (no fused multiply-add), so that equal logits with equal adjustments stay equal.  l / rep by
// rcp = 1 / rep and one step of the remainder, which is the rounded quotient (but for the last bit of
// results near the underflow); div is rep there, but 0 for an infinite rep, whose rcp of 0 would make the step a NaN.
constexpr uint32_t SEL_SEEN = 0x80000000u, SEL_BIAS = 0x40000000u, SEL_COUNT = 0x3FFFFFFFu;
__device__ __forceinline__ float adjust_logit(float l, uint32_t e, float bias, float rep, float div, float rcp, float pres, float freq) {
#pragma clang fp contract(off)
    const float up = l * rep, q = l * rcp;
    const float d = fmaf(fmaf(-q, div, l), rcp, q);
    const float down = fabsf(q) < INFINITY ? d : q;
    l = (e & SEL_SEEN) ? (l > 0.f ? down : up) : l;
    const uint32_t made = e & SEL_COUNT;
    const float fm = freq * (float)made;
    l = l - fm;
    l = l - (made > 0 ? pres : 0.f);
    return l + bias;
}

// The six butterfly steps of a wave-wide reduction without LDS: lane permutes inside 16 lanes (a
// mirror stands for the exchange of groups whose lanes agree already), then the two swaps.
template <class F> __device__ __forceinline__ uint32_t wave_fold(uint32_t v, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));      // lane ^ 1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));      // lane ^ 2
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));     // mirror in 8
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));     // mirror in 16
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(b[0], b[1]);
}
__device__ __forceinline__ float wave_max_f(float v) {
    return __uint_as_float(wave_fold(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float wave_sum_f(float v) {
    return __uint_as_float(wave_fold(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t wave_min_u(uint32_t v) {
    return wave_fold(v, [](uint32_t a, uint32_t b) { return min(a, b); });
}
// Best of a wave's lanes, in every lane.
__device__ __forceinline__ Best wave_best(const Best& b) {
    const float mx = wave_max_f(b.id < 0 ? -INFINITY : b.mx);
    const uint32_t id = wave_min_u(b.id >= 0 && b.mx == mx ? (uint32_t)b.id : 0xFFFFFFFFu);
    const float s = wave_sum_f(b.id < 0 ? 0.f : b.s * __expf(b.mx - mx));
    return Best{mx, (int)id, s};
}

// Two rows' reductions over the wave at once: the swap leaves row 0's values in lanes 0-31 and row 1's in
// lanes 32-63, where the other steps run for both.
template <class F> __device__ __forceinline__ uint32_t wave_fold2(uint32_t v0, uint32_t v1, F f) {
    const auto a = __builtin_amdgcn_permlane32_swap(v0, v1, false, false);
    uint32_t v = f(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(b[0], b[1]);
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
    return f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
}

// A workgroup takes SEL_IDS consecutive ids of `rows_per` consecutive rows.  A thread holds eight ids
// for all of them, so a sequence's history and bias list are scanned once per workgroup, into
// LDS tables of its ids, and each thread keeps its eight entries in registers; an adjustment
// runs for the thread's j-th ids only where some lane of the wave has an entry there.  What may not be
// picked is a bit of a word (allow mask, vocabulary end, MASK id).  Per row and wave: the largest
// value, the lowest id of it from eight comparisons (lane masks, scalar), the sum of
// exp(l - largest); the waves and then the ranges are merged.  With one range (small
// vocabularies) the workgroup writes the result.
//
// What bounds it: reading the logits (16 bytes a lane, also from rows that start at odd
// elements: the hardware takes unaligned addresses) beside 31 VALU instructions an id (counted; 31 us of issue
// for 256 rows of 152064) and latency: five waves a SIMD (WPE 5: 96 VGPRs) hide more of it than four of 109 or six with spills
// (256 rows of 152064 bf16 logits, adjusted logits kept: 52 us, 59, and 3 us more than the latter; a torch
// copy of that size takes 45).  Where four a SIMD hold all workgroups, their registers save the spills (WPE 3, up to 123 VGPRs): 32 rows of
// 126464 fp32 logits 11.3 and 12.6 us, of 1024 7.8 and 8.2.  In fp32 five waves spill 26 registers (16-bit types 2 to 4): 256 rows
// of 126464, adjusted logits kept, 90 us a call where the bytes take 54, 128 rows not kept 37 and 14.
struct alignas(16) SelectPart {
    float mx;
    int id;
    float s;
    int pad;
};

template <typename T, int WPE>
__global__ void __launch_bounds__(SEL_NT) __attribute__((amdgpu_waves_per_eu(WPE))) select_kernel(SelectArgs a, SelectPart* part, int n_ranges, int rows_per) {
    constexpr int NL = 16 / (int)sizeof(T), U = SEL_PT / NL;   // ids per 16-byte load, loads per row
    constexpr int HB = 4;                                      // history entries a thread loads at once
    __shared__ uint32_t adj_s[SEL_IDS], last_s[SEL_IDS];
    __shared__ float bias_s[SEL_IDS];
    __shared__ Best red[SEL_MAX_ROWS][SEL_NT / 64];
    const int tid = threadIdx.x;
    const int range = (int)(blockIdx.x % n_ranges), group = (int)(blockIdx.x / n_ranges);
    const int v0 = range * SEL_IDS;
    const int first = a.row0 ? max(0, a.row0[0]) : 0, behind = a.row0 ? min(a.T, a.row0[a.B]) : a.T;
    const int r0 = max(first, group * rows_per), r1 = min(behind, (group + 1) * rows_per);
    if (r0 >= r1) return;
    // load u's first id of this thread
    auto id_of = [&](int u) { return v0 + u * SEL_NT * NL + tid * NL; };

    // bit j: of valid, this thread's j-th id may be picked; of jmask, some lane's j-th id has an adjustment
    uint32_t valid = 0, jmask = 0, adj[SEL_PT];
    float bias[SEL_PT], rep = 1.f, div = 1.f, rcp = 1.f, pres = 0.f, freq = 0.f;
#pragma unroll
    for (int j = 0; j < SEL_PT; ++j) {
        const int v = id_of(j / NL) + j % NL;
        adj[j] = 0;
        bias[j] = 0.f;
        valid |= (uint32_t)(v < a.V && v != a.mask_id) << j;
    }

    // the tables of sequence b's history and biases at this workgroup's ids
    auto enter = [&](int b) {
        // (unsigned: the threads' indexes go up to a step past the end, which may be 2^31 - 1)
        const uint32_t h0 = a.hist ? a.hist0[b] : 0, h1 = a.hist ? a.hist0[b + 1] : 0;
        const uint32_t i0 = a.bias ? a.bias0[b] : 0, i1 = a.bias ? a.bias0[b + 1] : 0;
        // (a prompt longer than the history, 2^31 - 1 as "all of it", is the history: no sum past 32 bits)
        const uint32_t hp = a.n_prompt ? h0 + min(max(a.n_prompt[b], 0), max((int)(h1 - h0), 0)) : h0;
        pres = a.pres ? a.pres[b] : 0.f;
        freq = a.freq ? a.freq[b] : 0.f;
        rep = a.rep ? a.rep[b] : 1.f;
        rep = fabsf(rep) < FLT_MIN ? copysignf(0.f, rep) : rep;      // (1 / a subnormal one overflows; a NaN stays)
        div = fabsf(rep) == INFINITY ? 0.f : rep;
        rcp = __fdiv_rn(1.f, rep);
        if (h0 >= h1 && i0 >= i1) {
            jmask = 0;
            return;
        }
        auto slot = [&](int v) { return (unsigned)(v - v0) < (unsigned)SEL_IDS && v < a.V ? v - v0 : -1; };
        // the first entries of both lists are asked for before the tables are cleared
        int hv[HB], bv = -1;
        float bw = 0.f;
        auto load_hist = [&](uint32_t at) {
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                const uint32_t i = at + k * SEL_NT;
                hv[k] = i < h1 ? slot(a.hist[i]) : -1;
            }
        };
        load_hist(h0 + tid);
        if (i0 + tid < i1) { bv = slot(a.bias_id[i0 + tid]); bw = a.bias[i0 + tid]; }
        __syncthreads();                                       // the tables of the sequence before are read
#pragma unroll
        for (int i = 0; i < SEL_IDS / SEL_NT; ++i) { adj_s[tid + i * SEL_NT] = 0; last_s[tid + i * SEL_NT] = 0; }
        __syncthreads();
        for (uint32_t at = h0 + tid; at < h1; at += HB * SEL_NT) {
            if (at != h0 + tid) load_hist(at);
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                if (hv[k] < 0) continue;
                // (whole numbers: any order gives the same sum)
                atomicOr(&adj_s[hv[k]], SEL_SEEN);
                if (at + k * SEL_NT >= hp) atomicAdd(&adj_s[hv[k]], 1u);
            }
        }
        if (i0 < i1) {
            if (bv >= 0) atomicMax(&last_s[bv], (uint32_t)tid + 1u);
            for (uint32_t i = i0 + tid + SEL_NT; i < i1; i += SEL_NT) {
                const int k = slot(a.bias_id[i]);
                if (k >= 0) atomicMax(&last_s[k], i - i0 + 1u);
            }
            __syncthreads();
            auto win = [&](int k, int i, float w) {            // the last entry of an id: one thread
                if (k < 0 || last_s[k] != (uint32_t)i + 1u) return;
                bias_s[k] = w;
                atomicOr(&adj_s[k], SEL_BIAS);
            };
            win(bv, tid, bw);
            for (uint32_t i = i0 + tid + SEL_NT; i < i1; i += SEL_NT) win(slot(a.bias_id[i]), i - i0, a.bias[i]);
        }
        __syncthreads();
        jmask = 0;
#pragma unroll
        for (int j = 0; j < SEL_PT; ++j) {
            const int k = id_of(j / NL) - v0 + j % NL;
            adj[j] = adj_s[k];
            bias[j] = (adj[j] & SEL_BIAS) ? bias_s[k] : 0.f;
            jmask |= (uint32_t)(__builtin_amdgcn_ballot_w64(adj[j] != 0) != 0) << j;
        }
    };

    // the rows' masks: lane i has row r0 + i's
    const int arow = a.allow == nullptr ? -1 : (a.allow_row ? a.allow_row[min(r0 + (tid & 63), r1 - 1)] : min(r0 + (tid & 63), r1 - 1));
    // FULL: no id of this range is past the vocabulary
    auto all_rows = [&](auto FULL) {
        constexpr bool full = decltype(FULL)::value;
        int b_end = r0, re;                                    // rows below b_end belong to the sequence entered
        for (int rb = r0; rb < r1; rb = re) {
            // every load of the rows goes out before any is used (the words are not taken apart here, and the
            // tables of a sequence that begins are made meanwhile); past the last row it is read again
            u32x4_t raw[SEL_RB][U];
            uint32_t w[SEL_RB][U];
#pragma unroll
            for (int i = 0; i < SEL_RB; ++i) {
                const T* src = (const T*)a.logits + (long)min(rb + i, r1 - 1) * a.ld;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if constexpr (full) {
                        __builtin_memcpy(&raw[i][u], src + id_of(u), 16);
                    } else {
                        T x[NL];
#pragma unroll
                        for (int j = 0; j < NL; ++j) x[j] = src[min(id_of(u) + j, a.V - 1)];
                        __builtin_memcpy(&raw[i][u], x, 16);
                    }
                }
            }
            if (a.allow != nullptr) {
#pragma unroll
                for (int i = 0; i < SEL_RB; ++i) {
                    const int ar = __builtin_amdgcn_readlane(arow, min(rb + i, r1 - 1) - r0);
                    const uint32_t* words = a.allow + (size_t)(ar >= 0 && ar < a.n_allow ? ar : 0) * a.allow_ld;
#pragma unroll
                    for (int u = 0; u < U; ++u) w[i][u] = words[min(id_of(u) >> 5, a.allow_ld - 1)];
                }
            }
            if (rb >= b_end) {
                int nb = 0;
                b_end = a.T;
                if (a.row0 != nullptr) {
                    nb = row_seq(a.row0, a.B, rb);
                    b_end = a.row0[nb + 1];
                }
                enter(nb);
            }
            re = min(min(r1, b_end), rb + SEL_RB);             // rows of one sequence
#pragma unroll
            for (int i0 = 0; i0 < SEL_RB; i0 += 2) {
                if (rb + i0 >= re) break;
                float l[2][SEL_PT];
                uint32_t top[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        T x[NL];
                        __builtin_memcpy(x, &raw[i0 + i][u], 16);
#pragma unroll
                        for (int j = 0; j < NL; ++j) l[i][u * NL + j] = elem_to_f32<T>(x[j]);
                    }
                    if (jmask != 0) {
#pragma unroll
                        for (int j = 0; j < SEL_PT; ++j)
                            if (jmask >> j & 1) l[i][j] = adjust_logit(l[i][j], adj[j], bias[j], rep, div, rcp, pres, freq);
                    }
                    // NaN counts as -inf: the median instruction returns the least of the others if one is a NaN
                    // (the bound is hidden from the compiler, which would drop it)
                    float least = -INFINITY;
                    asm("" : "+v"(least));
#pragma unroll
                    for (int j = 0; j < SEL_PT; ++j) l[i][j] = __builtin_amdgcn_fmed3f(l[i][j], least, FLT_MAX);
                    uint32_t bits = valid;
                    if (a.allow != nullptr) {
                        const int ar = __builtin_amdgcn_readlane(arow, min(rb + i0 + i, r1 - 1) - r0);
                        uint32_t ok = 0;
#pragma unroll
                        for (int u = 0; u < U; ++u) ok |= (w[i0 + i][u] >> (id_of(u) & 31) & ((1u << NL) - 1)) << (u * NL);
                        bits &= ar >= 0 && ar < a.n_allow ? ok : (ar == -1 ? 0xFFFFFFFFu : 0u);
                    }
                    if (__builtin_amdgcn_ballot_w64(bits != (1u << SEL_PT) - 1) != 0) {
#pragma unroll
                        for (int j = 0; j < SEL_PT; ++j) {
                            const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)bits, j, 1);
                            l[i][j] = __uint_as_float((__float_as_uint(l[i][j]) & m) | (0xFF800000u & ~m));
                        }
                    }
                    if (a.out != nullptr && rb + i0 + i < re) {
                        T* dst = (T*)a.out + (long)(rb + i0 + i) * a.ld_out;
                        if constexpr (full) {
                            T y[SEL_PT];
#pragma unroll
                            for (int j = 0; j < SEL_PT; ++j) y[j] = (T)l[i][j];
#pragma unroll
                            for (int u = 0; u < U; ++u) __builtin_memcpy(dst + id_of(u), &y[u * NL], 16);
                        } else {
#pragma unroll
                            for (int j = 0; j < SEL_PT; ++j) {
                                const int v = id_of(j / NL) + j % NL;
                                if (v < a.V) dst[v] = (T)l[i][j];
                            }
                        }
                    }
                    float mx = l[i][0];
#pragma unroll
                    for (int j = 1; j < SEL_PT; ++j) mx = fmaxf(mx, l[i][j]);
                    top[i] = __float_as_uint(mx);
                }
                const uint32_t tops = wave_fold2(top[0], top[1], [](uint32_t p, uint32_t q) {
                    return __float_as_uint(fmaxf(__uint_as_float(p), __uint_as_float(q))); });
                float sum[2];
                int id[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float mx = __uint_as_float(__builtin_amdgcn_readlane(tops, 32 * i));
                    id[i] = -1;
                    // (load by load) the first lane that has the largest value, and its first id
#pragma unroll
                    for (int u = U - 1; u >= 0; --u) {
                        float mu = l[i][u * NL];
#pragma unroll
                        for (int j = 1; j < NL; ++j) mu = fmaxf(mu, l[i][u * NL + j]);
                        const uint64_t any = __builtin_amdgcn_ballot_w64(mu == mx);
                        if (any == 0) continue;
                        const int ln = __builtin_ctzll(any);
                        int k = 0;
#pragma unroll
                        for (int j = NL - 1; j >= 0; --j)
                            if (__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l[i][u * NL + j]), ln)) == mx) k = j;
                        id[i] = v0 + u * SEL_NT * NL + ((tid & ~63) + ln) * NL + k;
                    }
                    const float ref = mx > -INFINITY ? mx : 0.f;
                    sum[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < SEL_PT; ++j) sum[i] += __builtin_amdgcn_exp2f((l[i][j] - ref) * 1.4426950408889634f);
                    if (!(mx > -INFINITY)) id[i] = -1;
                }
                const uint32_t sums = wave_fold2(__float_as_uint(sum[0]), __float_as_uint(sum[1]), [](uint32_t p, uint32_t q) {
                    return __float_as_uint(__uint_as_float(p) + __uint_as_float(q)); });
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if ((tid & 63) == 32 * i && rb + i0 + i < re)
                        red[rb + i0 + i - r0][tid >> 6] = Best{__uint_as_float(tops), id[i], __uint_as_float(sums)};
            }
        }
    };
    if (v0 + SEL_IDS <= a.V) all_rows(std::true_type{});
    else all_rows(std::false_type{});
    __syncthreads();
    if (tid < r1 - r0) {
        Best best = red[tid][0];
#pragma unroll
        for (int w = 1; w < SEL_NT / 64; ++w) best = best_merge(best, red[tid][w]);
        const int row = r0 + tid;
        if (n_ranges == 1) {
            a.out_id[row] = best.id;
            a.out_conf[row] = best.id >= 0 ? 1.f / best.s : 0.f;
        } else {
            part[(size_t)row * n_ranges + range] = SelectPart{best.mx, best.id, best.s, 0};
        }
    }
}

// Merge of the ranges: one wave per row.
__global__ void __launch_bounds__(256) select_merge_kernel(SelectArgs a, const SelectPart* part, int n_ranges) {
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= a.T || (a.row0 != nullptr && (row < a.row0[0] || row >= a.row0[a.B]))) return;
    Best best{-INFINITY, -1, 0.f};
    for (int i = lane; i < n_ranges; i += 64) {
        const SelectPart p = part[(size_t)row * n_ranges + i];
        best = best_merge(best, Best{p.mx, p.id, p.s});
    }
    best = wave_best(best);
    if (lane == 0) {
        a.out_id[row] = best.id;
        a.out_conf[row] = best.id >= 0 ? 1.f / best.s : 0.f;
    }
}

}  // namespace dllm
