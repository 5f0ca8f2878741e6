// Penalties, biases and masks on logits, then the id of the largest and its confidence.
#pragma once

#include <float.h>

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

// A logit after its sequence's penalties and bias.  Separate roundings (no fused
// multiply-add), so that equal logits with equal adjustments stay equal.
__device__ __forceinline__ float adjust_logit(float l, bool seen, int made, float bias, bool has_bias, float rep,
                                              float pres, float freq) {
#pragma clang fp contract(off)
    if (seen) l = l > 0.f ? __fdiv_rn(l, rep) : l * rep;
    const float f = freq * (float)made;
    l = l - f;
    if (made > 0) l = l - pres;
    if (has_bias) l = l + bias;
    return l != l ? -INFINITY : fminf(l, FLT_MAX);
}

// Simple form: a workgroup per row; every id scans its sequence's history and bias list.
template <typename T>
__global__ void __launch_bounds__(256) select_row_kernel(SelectArgs a) {
    __shared__ Best red[4];
    const int row = blockIdx.x;
    int b = 0;
    if (a.row0 != nullptr) {
        if (row < a.row0[0] || row >= a.row0[a.B]) return;
        while (b + 1 < a.B && a.row0[b + 1] <= row) ++b;
    }
    const T* src = (const T*)a.logits + row * a.ld;
    T* dst = a.out ? (T*)a.out + row * a.ld_out : nullptr;
    const float rep = a.rep ? a.rep[b] : 1.f, pres = a.pres ? a.pres[b] : 0.f, freq = a.freq ? a.freq[b] : 0.f;
    const int h0 = a.hist ? a.hist0[b] : 0, h1 = a.hist ? a.hist0[b + 1] : 0;
    const int hp = a.hist && a.n_prompt ? h0 + a.n_prompt[b] : h0;
    const int i0 = a.bias ? a.bias0[b] : 0, i1 = a.bias ? a.bias0[b + 1] : 0;
    const int ar = a.allow ? (a.allow_row ? a.allow_row[row] : row) : -1;
    Best best{-INFINITY, -1, 0.f};
    for (int v = threadIdx.x; v < a.V; v += 256) {
        int made = 0;
        bool seen = false, has = false;
        float bias = 0.f;
        for (int i = h0; i < h1; ++i)
            if (a.hist[i] == v) {
                seen = true;
                made += i >= hp;
            }
        for (int i = i0; i < i1; ++i)
            if (a.bias_id[i] == v) {
                has = true;
                bias = a.bias[i];
            }
        float l = adjust_logit(elem_to_f32<T>(src[v]), seen, made, bias, has, rep, pres, freq);
        bool drop = v == a.mask_id;
        if (a.allow && ar != -1)
            drop |= ar < 0 || ar >= a.n_allow || (v >> 5) >= a.allow_ld || !(a.allow[(size_t)ar * a.allow_ld + (v >> 5)] >> (v & 31) & 1);
        if (drop) l = -INFINITY;
        if (dst) dst[v] = (T)l;
        if (l > -INFINITY) best = best_merge(best, Best{l, v, 1.f});
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
        best = best_merge(best, Best{__shfl_xor(best.mx, o), __shfl_xor(best.id, o), __shfl_xor(best.s, o)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) best = best_merge(best, red[w]);
        a.out_id[row] = best.id;
        a.out_conf[row] = best.id >= 0 ? 1.f / best.s : 0.f;
    }
}

}  // namespace dllm
