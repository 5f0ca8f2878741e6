// Log probabilities of given tokens, the rows' entropies and the most probable ids, in one pass over logits.
#pragma once

#include <float.h>

#include <type_traits>

#include "batch_rules.hpp"
#include "common.hpp"
#include "qk_rope.hpp"

namespace dllm {

typedef u32x4_t __attribute__((aligned(2))) any_u32x4;     // 16 bytes from any 16-bit element on

struct LogprobArgs {
    const void* logits;
    long ld;
    int T, V, mask_id;
    int n_tok;                    // given tokens that the rows' workgroups write (0: a launch of their own does)
    int top;
    const int *tok, *tok_row;
    float *logp, *entropy;
    int* top_id;
    float* top_logp;
    int parts, per;               // parts of a row, blocks of LP_BLOCK ids each
    struct LogStat* stat;         // [T][parts][waves]
    uint64_t* keys;               // [T][parts][waves][top]
    float2* row_stat;             // [T] largest logit and log of the sum, for the tokens' own launch, or NULL
};

// Sums over a set of logits: s = sum e^(x - m), t = sum (x - m) e^(x - m), m the largest.  Then the log of the
// sum is m + log s and the entropy log s - t / s.
struct LogStat {
    float m, s, t, pad;
};
// Exponents below this are as good as -inf (e^-256 = 0 in fp32), and finite: 0 times one is 0.
constexpr float LP_LEAST = -256.f;
__device__ __forceinline__ float lp_exp(float d) { return __builtin_amdgcn_exp2f(d * 1.4426950408889634f); }
__device__ __forceinline__ void stat_move(LogStat& a, float m) {           // (to a reference m >= a.m)
    const float d = __builtin_amdgcn_fmed3f(a.m - m, LP_LEAST, 0.f);       // (-inf - -inf, a NaN, gives the least)
    const float w = lp_exp(d);
    a.t = (a.t + a.s * d) * w;
    a.s *= w;
    a.m = m;
}
__device__ __forceinline__ LogStat stat_merge(LogStat a, LogStat b) {
    const float m = fmaxf(a.m, b.m);
    stat_move(a, m);
    stat_move(b, m);
    return LogStat{m, a.s + b.s, a.t + b.t, 0.f};
}

// The other lane of a butterfly step of distance M: lane permutes inside 16 lanes, swaps beyond.
template <int M> __device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    if constexpr (M == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);
    else if constexpr (M == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);
    else if constexpr (M == 4) {
        const int x = __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);       // lane ^ 7
        return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0x1B, 0xF, 0xF, true);          // lane ^ 3
    } else if constexpr (M == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true);   // rotate by 8 of 16
    else if constexpr (M == 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (threadIdx.x & 16) ? a[0] : a[1];
    } else {
        const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (threadIdx.x & 32) ? a[0] : a[1];
    }
}
template <int M> __device__ __forceinline__ LogStat stat_step(const LogStat& a) {
    return stat_merge(a, LogStat{__uint_as_float(lane_xor<M>(__float_as_uint(a.m))), __uint_as_float(lane_xor<M>(__float_as_uint(a.s))),
                                 __uint_as_float(lane_xor<M>(__float_as_uint(a.t))), 0.f});
}
__device__ __forceinline__ LogStat wave_stat(LogStat a) {
    return stat_step<32>(stat_step<16>(stat_step<8>(stat_step<4>(stat_step<2>(stat_step<1>(a))))));
}

// Key of an id: larger is more probable, equal logits by the lower id; 0 is no id.  Both zeros are one logit.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ uint64_t key_of_id(float x, int id) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - (uint32_t)id); }
__device__ __forceinline__ int id_of_key(uint64_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }
__device__ __forceinline__ float value_of_key(uint64_t k) { return of_order((uint32_t)(k >> 32)); }
// The float below x (-inf for -inf; of the zeros, which are one, the one below both): a strict bound that x itself passes.
__device__ __forceinline__ float below(float x) { return x > -INFINITY ? of_order(order_of(x) - (x == 0.f ? 2 : 1)) : x; }

// Compare and exchange with lane ^ M: lanes in `larger` keep the larger key.
template <int M> __device__ __forceinline__ uint64_t key_step(uint64_t v, bool larger) {
    const uint64_t o = (uint64_t)lane_xor<M>((uint32_t)(v >> 32)) << 32 | lane_xor<M>((uint32_t)v);
    return (v > o) == larger ? v : o;
}
// The last steps of a bitonic sort of 2 M keys, descending where `down`.
template <int M> __device__ __forceinline__ uint64_t key_clean(uint64_t v, int lane, bool down) {
    v = key_step<M>(v, ((lane & M) == 0) == down);
    if constexpr (M > 1) v = key_clean<M / 2>(v, lane, down);
    return v;
}
// A wave's 64 keys sorted by lane.
__device__ __forceinline__ uint64_t key_sort(uint64_t v, int lane, bool down) {
    v = key_clean<1>(v, lane, (lane & 2) == 0);
    v = key_clean<2>(v, lane, (lane & 4) == 0);
    v = key_clean<4>(v, lane, (lane & 8) == 0);
    v = key_clean<8>(v, lane, (lane & 16) == 0);
    v = key_clean<16>(v, lane, (lane & 32) == 0);
    return key_clean<32>(v, lane, down);
}
// The 64 largest of a descending list and of 64 more keys, descending: the lane-wise maximum of one list and the other
// reversed holds them and is bitonic.  empty: nothing is in the list yet.
__device__ __forceinline__ uint64_t key_merge(uint64_t best, uint64_t more, int lane, bool empty) {
    const uint64_t sorted = key_sort(more, lane, empty);
    return empty ? sorted : key_clean<32>(best > sorted ? best : sorted, lane, true);
}

// Where the 64 largest of the keys src[0 .. n) end: every wave of the workgroup takes chunks of 64, wave 0 joins them
// (tmp: 64 keys a wave).  Returns wave 0's list, descending.
template <int NW> __device__ __forceinline__ uint64_t keys_top(const uint64_t* src, int n, uint64_t* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t best = 0;
    for (int i = 64 * wave; i < n; i += 64 * NW) best = key_merge(best, i + lane < n ? src[i + lane] : 0, lane, i == 64 * wave);
    if (n <= 64) return best;                             // (wave 0 has had them all)
    __syncthreads();
    tmp[64 * wave + lane] = best;
    __syncthreads();
    if (wave == 0)
        for (int w = 1; w < NW && 64 * w < n; ++w) best = key_clean<32>(best > tmp[64 * w + 63 - lane] ? best : tmp[64 * w + 63 - lane], lane, true);
    return best;
}

// Logit of id v in row r as the sums count it; a NaN, the MASK id and what is no id are -inf.
template <typename T> __device__ __forceinline__ float lp_logit(const LogprobArgs& a, int r, int v) {
    float x = -INFINITY;
    if (v >= 0 && v < a.V && v != a.mask_id) x = elem_to_f32<T>(((const T*)a.logits)[(long)r * a.ld + v]);
    return x < FLT_MAX ? x : (x >= FLT_MAX ? FLT_MAX : -INFINITY);          // (a NaN is neither)
}
// Given token i of row `row`: -> whether it is that workgroup's (row 0's also has those of rows that there are not), and
// its logit.
template <typename T> __device__ __forceinline__ bool lp_token(const LogprobArgs& a, int row, int i, float& x) {
    const int r = a.tok_row ? a.tok_row[i] : i, v = a.tok[i];
    const bool there = r >= 0 && r < a.T;
    x = -INFINITY;
    if (there ? r != row : row != 0) return false;
    if (there) x = lp_logit<T>(a, row, v);
    return true;
}
// First token that a thread of row `row`'s workgroup looks at.  Without tok_row the row's own is the only one, else the
// workgroup looks at all of them (the launch rules bound how many).
__device__ __forceinline__ int lp_first(const LogprobArgs& a, int row) {
    return a.tok_row ? (int)threadIdx.x : (threadIdx.x == 0 ? row : a.n_tok);
}
// What a row's workgroup writes once its sums (in every thread) and best keys (in wave 0) are known.  mine, x0: lp_token of
// the thread's first token `first`, asked for before.
template <typename T, int NT>
__device__ __forceinline__ void lp_write(const LogprobArgs& a, int row, const LogStat& st, uint64_t best, int first, bool mine, float x0) {
    const int tid = threadIdx.x;
    const bool any = st.m > -INFINITY;
    const float lse = any ? logf(st.s) : 0.f;
    if (tid == 0 && a.entropy) a.entropy[row] = any ? lse - st.t / st.s : 0.f;
    if (tid < a.top) {                                    // (at most 64)
        a.top_id[(size_t)row * a.top + tid] = best ? id_of_key(best) : -1;
        a.top_logp[(size_t)row * a.top + tid] = best ? (value_of_key(best) - st.m) - lse : -INFINITY;
    }
    if (a.n_tok == 0) {
        if (tid == 0 && a.row_stat) a.row_stat[row] = make_float2(st.m, lse);
        return;
    }
    for (int i = first; i < a.n_tok; i += NT) {
        if (i != first) {
            if (!a.tok_row) break;
            mine = lp_token<T>(a, row, i, x0);
        }
        if (mine) a.logp[i] = any ? (x0 - st.m) - lse : -INFINITY;
    }
}

// The largest of 32 logits, two an instruction.  (In assembly: the compiler would quiet every operand first.  A signalling
// NaN may hide a larger logit here; whoever uses this looks for NaNs afterwards.)
__device__ __forceinline__ float max_of_block(const float (&x)[LP_PT]) {
    float m[2] = {x[0], x[1]};
#pragma unroll
    for (int i = 2; i < LP_PT; i += 4) {
        asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m[0]) : "v"(x[i]), "v"(x[i + 1]));
        if (i + 3 < LP_PT) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m[1]) : "v"(x[i + 2]), "v"(x[i + 3]));
    }
    return fmaxf(m[0], m[1]);
}

// A workgroup takes a part of a row, its waves blocks of 64 x 32 ids.  A lane holds 32 logits: their largest moves its
// reference m, then every logit costs a difference, an exponential and two sums.  (One multiply-add for difference and
// factor, with the reference's rounding taken back from the sums, is 0.7 us faster at 256 rows of 152064, but a row's own
// largest logit is no longer exactly e^0 = 1.)  A block with a NaN or an infinity is done again with a clamp a logit.
//
// The most probable ids: a wave keeps the 64 largest keys (logit, id) it has seen, a sorted list over its lanes, and the
// bound that a logit has to pass, the `top`-th of them.  In the first block that is the least of what the waves' top / NW-th
// largest lane maxima are, which `top` logits of the workgroup reach.  What passes goes to a buffer in LDS, by ballots, and
// 64 at a time are sorted and merged into the list.  Ids ascend from block to block, so an equal logit in a later block has
// lost: the bound is strict, but inside a block, whose ids are not taken in order.
//
// What bounds it: 256 rows of 152064 bf16 logits, 24 us and 5 for the merge, where reading takes 12 (at a plain read's 6.5 TB/s)
// and VALU issue 14: the start, the first bound and the last sorts of all waves, which run at once (256 of 126464 fp32 33 us in
// all, reading 20; 1024 rows, one part each, 87 and 79); few or short rows, latency: load, bound, sort, logarithm (16 rows of 1024
// 7 us, 32 of 126464 fp32 8 and 6).
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_NT) logprobs_kernel(LogprobArgs a) {
    constexpr int NL = 16 / (int)sizeof(T), U = LP_PT / NL, NW = LP_NT / 64;
    __shared__ uint64_t pend_all[TOP ? NW * 128 : 1], list_s[TOP ? NW * 64 : 1];
    __shared__ LogStat stat_s[NW];
    __shared__ uint32_t first_s[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = (int)(blockIdx.x % a.parts), row = (int)(blockIdx.x / a.parts);
    const int b0 = part * a.per, b1 = min(b0 + a.per, (a.V + LP_BLOCK - 1) / LP_BLOCK);
    const T* src = (const T*)a.logits + (long)row * a.ld;
    uint64_t* pend = pend_all + (TOP ? 128 * wave : 0);

    u32x4_t raw[U];
    // (32-bit byte offsets from the row: no address registers; rows start at any element; read once: not kept in the
    // caches, which is 4 to 7% faster)
    auto load = [&](int blk) {
        const uint32_t at = ((uint32_t)blk * LP_BLOCK + lane * NL) * sizeof(T);
        if ((blk + 1) * LP_BLOCK <= a.V) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = __builtin_nontemporal_load((const any_u32x4*)((const char*)src + (at + u * 1024u)));
        } else {
            const uint32_t last = (uint32_t)(a.V - 1) * sizeof(T);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                T x[NL];
#pragma unroll
                for (int j = 0; j < NL; ++j) __builtin_memcpy(&x[j], (const char*)src + min(at + u * 1024u + j * (uint32_t)sizeof(T), last), sizeof(T));
                __builtin_memcpy(&raw[u], x, 16);
            }
        }
    };

    LogStat st{-INFINITY, 0.f, 0.f, 0.f};
    uint64_t best = 0;                                     // TOP: the list
    float bound = -INFINITY;                               // a logit has to exceed it
    int n_pend = 0;
    bool empty = true;
    auto flush = [&](int n) {                              // the first n <= 64 of the buffer into the list
        __builtin_amdgcn_wave_barrier();                   // (a wave's LDS operations keep their order)
        best = key_merge(best, lane < n ? pend[lane] : 0, lane, empty);
        empty = false;
        const uint64_t more = pend[64 + lane];
        pend[lane] = more;
        n_pend -= n;
        __builtin_amdgcn_wave_barrier();
    };
    auto kth = [&]() {                                     // the list's top-th logit
        const uint32_t o = __builtin_amdgcn_readlane((uint32_t)(best >> 32), a.top - 1);
        return o ? of_order(o) : -INFINITY;
    };

    int blk = b0 + wave;
    if (blk < b1) load(blk);
    // (where this workgroup writes the row: a token's three loads, one after the other, beside the logits)
    float x0 = 0.f;
    const int tok0 = lp_first(a, row);
    const bool mine = a.parts == 1 && tok0 < a.n_tok && lp_token<T>(a, row, tok0, x0);
    // (every wave has a block, or its workgroup's first bound is each wave's own)
    const bool together = TOP && b1 - b0 >= NW;
    for (bool first = true; blk < b1; blk += NW, first = false) {
        float x[LP_PT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            T e[NL];
            __builtin_memcpy(e, &raw[u], 16);
#pragma unroll
            for (int j = 0; j < NL; ++j) x[u * NL + j] = elem_to_f32<T>(e[j]);
        }
        const int v0 = blk * LP_BLOCK + lane * NL;
        auto id_of = [&](int i) { return v0 + i / NL * 64 * NL + i % NL; };
        if ((blk + 1) * LP_BLOCK > a.V || (unsigned)(a.mask_id - blk * LP_BLOCK) < (unsigned)LP_BLOCK) {
#pragma unroll
            for (int i = 0; i < LP_PT; ++i)
                if (id_of(i) >= a.V || id_of(i) == a.mask_id) x[i] = -INFINITY;
        }
        if (blk + NW < b1) load(blk + NW);
        float mx = max_of_block(x);
        const float m = fmaxf(st.m, mx);
        bool plain = __builtin_amdgcn_ballot_w64(!(fabsf(m) <= FLT_MAX)) == 0;
        if (plain) {
            float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < LP_PT; ++i) {
                const float d = x[i] - m, e = lp_exp(d);
                s[i & 1] += e;
                t[i & 1] = fmaf(e, d, t[i & 1]);
            }
            t[0] += t[1];
            plain = __builtin_amdgcn_ballot_w64(!(t[0] <= 0.f)) == 0;      // (a NaN is not)
            if (plain) {
                stat_move(st, m);
                st.s += s[0] + s[1];
                st.t += t[0];
            }
        }
        if (!plain) {
            mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < LP_PT; ++i) mx = fmaxf(mx, x[i]);
            mx = fminf(mx, FLT_MAX);
            stat_move(st, fmaxf(st.m, mx));
#pragma unroll
            for (int i = 0; i < LP_PT; ++i) {
                const float d = __builtin_amdgcn_fmed3f(x[i] - st.m, LP_LEAST, 0.f);
                const float e = lp_exp(d);
                st.s += e;
                st.t = fmaf(e, d, st.t);
            }
        }
        if constexpr (TOP) {
            if (first) {
                // the k-th largest of the lanes' maxima, bit by bit (16-bit logits differ in the upper bits, of fp32 15 of 23 will do)
                const int k = together ? (a.top + NW - 1) / NW : a.top;
                const uint32_t o = order_of(mx);
                uint32_t t = 0;
                constexpr int LOW = sizeof(T) == 4 ? 8 : (std::is_same<T, __bf16>::value ? 16 : 13);
                for (int bit = 31; bit >= LOW; --bit) {
                    const uint32_t c = t | 1u << bit;
                    if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(o >= c)) >= k) t = c;
                }
                if (together) {
                    if (lane == 0) first_s[wave] = t;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < NW; ++w) t = min(t, first_s[w]);
                }
                // (a bound of no float's order, of the lowest bits cut off, is lower still)
                bound = t > order_of(-INFINITY) ? below(of_order(t)) : -INFINITY;
            }
            if (__builtin_amdgcn_ballot_w64(mx > bound) != 0) {
                float pass = bound;
#pragma unroll
                for (int i = 0; i < LP_PT; ++i) {
                    const bool in = x[i] > pass;
                    const uint64_t who = __builtin_amdgcn_ballot_w64(in);
                    if (who != 0) {
                        if (in) {
                            const int at = n_pend + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                            pend[at] = key_of_id(fminf(x[i], FLT_MAX), id_of(i));
                        }
                        n_pend += __builtin_popcountll(who);
                        if (n_pend >= 64) {
                            flush(64);
                            pass = fmaxf(pass, below(kth()));
                        }
                    }
                }
                bound = fmaxf(bound, kth());
            }
        }
    }
    if (TOP && n_pend > 0) flush(n_pend);
    st = wave_stat(st);
    if (a.parts > 1) {                                     // every wave's own, for the merge
        const size_t rec = ((size_t)row * a.parts + part) * NW + wave;
        if (lane == 0) a.stat[rec] = st;
        if (TOP && lane < a.top) a.keys[rec * a.top + lane] = best;
        return;
    }
    if (TOP && lane < a.top) list_s[wave * a.top + lane] = best;           // (as one list of NW * top keys)
    if (lane == 0) stat_s[wave] = st;
    __syncthreads();
    st = stat_s[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) st = stat_merge(st, stat_s[w]);
    if (TOP && b1 - b0 > 1) best = keys_top<NW>(list_s, NW * a.top, pend_all);      // (else wave 0 has them)
    lp_write<T, LP_NT>(a, row, st, best, tok0, mine, x0);
}

// Merge of a row's waves.
template <typename T>
__global__ void __launch_bounds__(LP_NT) logprobs_merge_kernel(LogprobArgs a) {
    constexpr int NW = LP_NT / 64;
    __shared__ uint64_t tmp[NW * 64];
    const int row = blockIdx.x, lane = threadIdx.x & 63, n = a.parts * NW;
    float x0 = 0.f;
    const int tok0 = lp_first(a, row);
    const bool mine = tok0 < a.n_tok && lp_token<T>(a, row, tok0, x0);
    LogStat st{-INFINITY, 0.f, 0.f, 0.f};
    for (int i = lane; i < n; i += 64) st = stat_merge(st, a.stat[(size_t)row * n + i]);
    st = wave_stat(st);                                   // (every wave for itself)
    uint64_t best = 0;
    if (a.top > 0) best = keys_top<NW>(a.keys + (size_t)row * n * a.top, n * a.top, tmp);
    lp_write<T, LP_NT>(a, row, st, best, tok0, mine, x0);
}

// Given tokens once the rows' sums are known, a thread each.
template <typename T>
__global__ void __launch_bounds__(LP_NT) logprobs_tokens_kernel(LogprobArgs a, int n_tok) {
    const int i = blockIdx.x * LP_NT + threadIdx.x;
    if (i >= n_tok) return;
    const int r = a.tok_row[i], v = a.tok[i];
    float lp = -INFINITY;
    if (r >= 0 && r < a.T) {
        const float2 st = a.row_stat[r];
        const float x = lp_logit<T>(a, r, v);
        if (st.x > -INFINITY) lp = (x - st.x) - st.y;
    }
    a.logp[i] = lp;
}

}  // namespace dllm
