// Norm of every query and key head, rotation and cache write in one pass.
#pragma once

#include "common.hpp"

namespace dllm {

// Element types of the batch operators.
struct ElemF32 { using T = float; };
struct ElemF16 { using T = _Float16; };
struct ElemBF16 { using T = __bf16; };

template <typename T> __device__ __forceinline__ float elem_to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T elem_from_f32(float v) { return (T)v; }
// fp16 saturates, as the library's caches do
template <> __device__ __forceinline__ _Float16 elem_from_f32<_Float16>(float v) {
    return (_Float16)(v != v ? v : fminf(fmaxf(v, -65504.f), 65504.f));
}

struct QkArgs {
    const void *q, *k, *v;
    long ld_q, ld_k, ld_v;
    const float *gq, *gk;
    const float2* rope;
    const int *pos, *slot;
    void *qo, *kp, *vp;
    int T, H, Hk, page_shift, n_pages, max_pos;
    float eps;
};

// Eight consecutive elements as fp32.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    T e[8];
    __builtin_memcpy(e, __builtin_assume_aligned(p, 16), sizeof(e));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = elem_to_f32<T>(e[i]);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = elem_from_f32<T>(x[i]);
    __builtin_memcpy(__builtin_assume_aligned(p, 16), e, sizeof(e));
}

// A head is taken by DH / 16 neighbouring lanes: lane i holds elements 8i .. 8i+7 of both halves,
// so that a rotation's pair is in one lane, loads and stores are 16 bytes and the sum of
// squares is a few lane swaps.  Items are (row, head) over the n_heads query and n_kv_heads
// key heads; V^T takes workgroups of its own behind them.
template <typename T, int DH>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkArgs a, int qk_wgs) {
    constexpr int LPH = DH / 16;                              // lanes per head
    if ((int)blockIdx.x < qk_wgs) {
        const long item = ((long)blockIdx.x * 256 + threadIdx.x) / LPH;
        const int i = threadIdx.x % LPH, HH = a.H + a.Hk;
        if (item >= (long)a.T * HH) return;                   // whole heads: the swaps below stay inside one
        const int row = (int)(item / HH), hh = (int)(item % HH);
        const bool is_q = hh < a.H;
        const int h = is_q ? hh : hh - a.H;
        const T* src = (is_q ? (const T*)a.q + row * a.ld_q : (const T*)a.k + row * a.ld_k) + h * DH + 8 * i;
        float x[8], y[8];
        load8<T>(src, x);
        load8<T>(src + DH / 2, y);
        const int pos = min(max(a.pos[row], 0), a.max_pos - 1);
        const float* gain = is_q ? a.gq : a.gk;
        if (gain != nullptr) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += x[e] * x[e] + y[e] * y[e];
#pragma unroll
            for (int o = 1; o < LPH; o <<= 1) s += __shfl_xor(s, o);
            const float rs = 1.0f / sqrtf(s / (float)DH + a.eps);
            float g0[8], g1[8];
            load8<float>(gain + 8 * i, g0);
            load8<float>(gain + DH / 2 + 8 * i, g1);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = x[e] * rs * g0[e];
                y[e] = y[e] * rs * g1[e];
            }
        }
        const float2* cs = a.rope + (size_t)pos * (DH / 2) + 8 * i;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 c = cs[e];
            const float u = x[e] * c.x - y[e] * c.y;
            y[e] = y[e] * c.x + x[e] * c.y;
            x[e] = u;
        }
        T* dst;
        if (is_q) {
            dst = (T*)a.qo + ((size_t)row * a.H + h) * DH + 8 * i;
        } else {
            const int slot = a.slot[row], pg = slot >> a.page_shift;
            if (slot < 0 || pg >= a.n_pages) return;
            const int off = slot & ((1 << a.page_shift) - 1);
            dst = (T*)a.kp + ((((size_t)pg * a.Hk + h) << a.page_shift) + off) * DH + 8 * i;
        }
        store8<T>(dst, x);
        store8<T>(dst + DH / 2, y);
        return;
    }
    // V^T: one element per thread
    const long u = (long)(blockIdx.x - qk_wgs) * 256 + threadIdx.x;
    const int n = a.Hk * DH;
    if (u >= (long)a.T * n) return;
    const int row = (int)(u / n), c = (int)(u % n);
    const int slot = a.slot[row], pg = slot >> a.page_shift;
    if (slot < 0 || pg >= a.n_pages) return;
    const int off = slot & ((1 << a.page_shift) - 1);
    const float v = elem_to_f32<T>(((const T*)a.v)[row * a.ld_v + c]);
    ((T*)a.vp)[((((size_t)pg * n) + c) << a.page_shift) + off] = elem_from_f32<T>(v);
}

}  // namespace dllm
