// Penalties, biases and masks on logits, then the id of the largest and its confidence.
#pragma once

#include <float.h>

#include "attn_paged.hpp"
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

// l / rep, rounded once, where rcp is 1 / rep rounded once: one step of the remainder is exact for
// quotients away from the ends of the range, which take the division itself.
__device__ __forceinline__ float div_by(float l, float rep, float rcp) {
    const float q = l * rcp, d = fmaf(fmaf(-q, rep, l), rcp, q);
    const float m = fabsf(l), n = fabsf(rep);
    const bool plain = m > 0x1p-90f && m < 0x1p90f && n > 0x1p-30f && n < 0x1p30f;
    return plain ? d : __fdiv_rn(l, rep);
}

// A logit after its sequence's penalties and bias.  Separate roundings (no fused
// multiply-add), so that equal logits with equal adjustments stay equal.
__device__ __forceinline__ float adjust_logit(float l, bool seen, int made, float bias, bool has_bias, float rep,
                                              float rcp, float pres, float freq) {
#pragma clang fp contract(off)
    const float up = l * rep, down = div_by(l, rep, rcp);
    l = seen ? (l > 0.f ? down : up) : l;
    const float f = freq * (float)made;
    l = l - f;
    const float m = l - pres;
    l = made > 0 ? m : l;
    const float w = l + bias;
    return has_bias ? w : l;
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
// elements: the hardware takes unaligned addresses) and about 13 VALU instructions an id.
constexpr int SEL_NT = 256, SEL_PT = 8, SEL_IDS = SEL_NT * SEL_PT, SEL_RB = 4, SEL_MAX_ROWS = 16;
constexpr uint32_t SEL_SEEN = 0x80000000u, SEL_BIAS = 0x40000000u;

struct alignas(16) SelectPart {
    float mx;
    int id;
    float s;
    int pad;
};

template <typename T>
__global__ void __launch_bounds__(SEL_NT) select_kernel(SelectArgs a, SelectPart* part, int n_ranges, int rows_per) {
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

    uint32_t adj[SEL_PT], valid = 0, jmask = 0;                // jmask: the j whose adj is set in some lane
    float bias[SEL_PT], rep = 1.f, rcp = 1.f, pres = 0.f, freq = 0.f;
#pragma unroll
    for (int j = 0; j < SEL_PT; ++j) {
        const int v = id_of(j / NL) + j % NL;
        adj[j] = 0;
        bias[j] = 0.f;
        valid |= (uint32_t)(v < a.V && v != a.mask_id) << j;
    }

    // the tables of sequence b's history and biases at this workgroup's ids
    auto enter = [&](int b) {
        const int h0 = a.hist ? a.hist0[b] : 0, h1 = a.hist ? a.hist0[b + 1] : 0;
        const int i0 = a.bias ? a.bias0[b] : 0, i1 = a.bias ? a.bias0[b + 1] : 0;
        const int hp = a.n_prompt ? h0 + a.n_prompt[b] : h0;
        rep = a.rep ? a.rep[b] : 1.f;
        pres = a.pres ? a.pres[b] : 0.f;
        freq = a.freq ? a.freq[b] : 0.f;
        rcp = __fdiv_rn(1.f, rep);
        jmask = 0;
        if (h0 >= h1 && i0 >= i1) return;
        auto slot = [&](int v) { return (unsigned)(v - v0) < (unsigned)SEL_IDS && v < a.V ? v - v0 : -1; };
        // the first entries of both lists are asked for before the tables are cleared
        int hv[HB], bv = -1;
        float bw = 0.f;
        auto load_hist = [&](int at) {
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                const int i = at + k * SEL_NT;
                hv[k] = i < h1 ? slot(a.hist[i]) : -1;
            }
        };
        load_hist(h0 + tid);
        if (i0 + tid < i1) { bv = slot(a.bias_id[i0 + tid]); bw = a.bias[i0 + tid]; }
        __syncthreads();                                       // the tables of the sequence before are read
#pragma unroll
        for (int i = 0; i < SEL_IDS / SEL_NT; ++i) { adj_s[tid + i * SEL_NT] = 0; last_s[tid + i * SEL_NT] = 0; }
        __syncthreads();
        for (int at = h0 + tid; at < h1; at += HB * SEL_NT) {
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
            for (int i = i0 + tid + SEL_NT; i < i1; i += SEL_NT) {
                const int k = slot(a.bias_id[i]);
                if (k >= 0) atomicMax(&last_s[k], (uint32_t)(i - i0) + 1u);
            }
            __syncthreads();
            auto win = [&](int k, int i, float w) {            // the last entry of an id: one thread
                if (k < 0 || last_s[k] != (uint32_t)i + 1u) return;
                bias_s[k] = w;
                atomicOr(&adj_s[k], SEL_BIAS);
            };
            win(bv, tid, bw);
            for (int i = i0 + tid + SEL_NT; i < i1; i += SEL_NT) win(slot(a.bias_id[i]), i - i0, a.bias[i]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < SEL_PT; ++j) {
            const int k = id_of(j / NL) - v0 + j % NL;
            adj[j] = adj_s[k];
            bias[j] = (adj[j] & SEL_BIAS) ? bias_s[k] : 0.f;
            jmask |= (uint32_t)(__builtin_amdgcn_ballot_w64(adj[j] != 0) != 0) << j;
        }
    };

    int b = -1, b_end = r0;                                    // rows below b_end belong to b
    for (int rb = r0; rb < r1; rb += SEL_RB) {
        T x[SEL_RB][SEL_PT];
#pragma unroll
        for (int i = 0; i < SEL_RB; ++i) {
            const T* src = (const T*)a.logits + (long)min(rb + i, r1 - 1) * a.ld;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = id_of(u);
                if (v + NL <= a.V) {
                    __builtin_memcpy(&x[i][u * NL], src + v, 16);
                } else {
#pragma unroll
                    for (int j = 0; j < NL; ++j) x[i][u * NL + j] = v + j < a.V ? src[v + j] : (T)0.f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < SEL_RB; ++i) {
            const int row = rb + i;
            if (row >= r1) break;
            if (row >= b_end) {
                int nb = 0;
                b_end = a.T;
                if (a.row0 != nullptr) {
                    nb = row_seq(a.row0, a.B, row);
                    b_end = a.row0[nb + 1];
                }
                if (nb != b) enter(b = nb);
            }
            // bit j: this thread's j-th id may be picked
            uint32_t bits = valid;
            if (a.allow != nullptr) {
                const int ar = a.allow_row ? a.allow_row[row] : row;
                if (ar != -1) {
                    uint32_t ok = 0;
                    if (ar >= 0 && ar < a.n_allow) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int v = id_of(u);
                            const uint32_t w = v < a.V ? a.allow[(size_t)ar * a.allow_ld + (v >> 5)] >> (v & 31) : 0u;
                            ok |= (w & ((1u << NL) - 1)) << (u * NL);
                        }
                    }
                    bits &= ok;
                }
            }
            float l[SEL_PT];
#pragma unroll
            for (int j = 0; j < SEL_PT; ++j) l[j] = elem_to_f32<T>(x[i][j]);
            if (jmask != 0) {
#pragma unroll
                for (int j = 0; j < SEL_PT; ++j)
                    if (jmask >> j & 1) {
                        const float y = adjust_logit(l[j], (adj[j] & SEL_SEEN) != 0, (int)(adj[j] & 0x3FFFFFFFu), bias[j],
                                                     (adj[j] & SEL_BIAS) != 0, rep, rcp, pres, freq);
                        l[j] = adj[j] != 0 ? y : l[j];
                    }
            }
            // NaN counts as -inf: the median instruction returns the least of the others if one is a NaN (the
            // bound is hidden from the compiler, which would drop it)
            float least = -INFINITY;
            asm("" : "+v"(least));
#pragma unroll
            for (int j = 0; j < SEL_PT; ++j) l[j] = __builtin_amdgcn_fmed3f(l[j], least, FLT_MAX);
            if (__builtin_amdgcn_ballot_w64(bits != (1u << SEL_PT) - 1) != 0) {
#pragma unroll
                for (int j = 0; j < SEL_PT; ++j) {
                    const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)bits, j, 1);
                    l[j] = __uint_as_float((__float_as_uint(l[j]) & m) | (0xFF800000u & ~m));
                }
            }
            if (a.out != nullptr) {
                T* dst = (T*)a.out + (long)row * a.ld_out;
                T y[SEL_PT];
#pragma unroll
                for (int j = 0; j < SEL_PT; ++j) y[j] = (T)l[j];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int v = id_of(u);
                    if (v + NL <= a.V) {
                        __builtin_memcpy(dst + v, &y[u * NL], 16);
                    } else {
#pragma unroll
                        for (int j = 0; j < NL; ++j)
                            if (v + j < a.V) dst[v + j] = y[u * NL + j];
                    }
                }
            }
            float mx = l[0];
#pragma unroll
            for (int j = 1; j < SEL_PT; ++j) mx = fmaxf(mx, l[j]);
            mx = wave_max_f(mx);
            Best best{mx, -1, 0.f};
            if (mx > -INFINITY) {                              // the same in every lane
                // the first lane with the largest value and its first id, load by load
#pragma unroll
                for (int u = U - 1; u >= 0; --u) {
                    uint64_t eq[NL], any = 0;
#pragma unroll
                    for (int j = 0; j < NL; ++j) any |= eq[j] = __builtin_amdgcn_ballot_w64(l[u * NL + j] == mx);
                    if (any != 0) {
                        const int ln = __builtin_ctzll(any);
                        int j = NL - 1;
#pragma unroll
                        for (int k = NL - 2; k >= 0; --k)
                            if (eq[k] >> ln & 1) j = k;
                        best.id = v0 + u * SEL_NT * NL + ((tid & ~63) + ln) * NL + j;
                    }
                }
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < SEL_PT; ++j) s += __builtin_amdgcn_exp2f((l[j] - mx) * 1.4426950408889634f);
                best.s = wave_sum_f(s);
            }
            if ((tid & 63) == 0) red[row - r0][tid >> 6] = best;
        }
    }
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
