// The pieces of a model's forward around the batch operators: Q/K/V rows finished outside the QKV
// GEMM (norm of every head, paged cache), attention rows into the O projection's operand.
#pragma once

#include "common.hpp"
#include "qk_rope.hpp"

namespace dllm {

struct QkvRows {
    const float* P;          // [ks][rows][ldn] sums of the QKV GEMM, packed rows (a rotation's pair is adjacent)
    int ks;
    size_t slice;            // floats from slice to slice
    int ldn;
    const float* bias;       // packed order, or nullptr (already added, or none)
    int M, H, Hk;
    const float *gq, *gk;    // gains of the heads' norm, or nullptr
    float eps;
    const float2* rope;
    int max_pos, pos_base;
    const int* pos;          // row m's position, or nullptr: pos_base + m
    const int* slot;         // row m's cache slot, or nullptr: its position in one page of page_len
    int page_shift, page_len, n_pages;
    void* q;                 // fp32; or fp16: one plane (q_plane 0), or hi and lo
    size_t q_plane;
    void *K, *V;             // [n_pages][Hk][page_len][DH], [n_pages][Hk][DH][page_len]
};

// DH / 16 lanes per (row, Q or K head): lane i has pairs 8i .. 8i+7, which are dims 8i + e and 8i + e +
// DH / 2; the V values follow, one per thread.  Reads 4 bytes a value once, launch-bound at a window's rows
// (four layers of the 8B widths, 32 rows behind 512: the heads' norm through it 644 us against 639 without, where the GEMM's
// epilogue does the work).  V^T goes out in single elements a page or cache row apart: a prompt of 4096 rows 12.6
// against 12.1 ms.
template <bool XF32, int DH>
__global__ void __launch_bounds__(256) qkv_rows_kernel(QkvRows a, int qk_wgs) {
    using T = typename std::conditional<XF32, float, _Float16>::type;
    constexpr int LPH = DH / 16;
    const long u = (long)(blockIdx.x < (unsigned)qk_wgs ? blockIdx.x : blockIdx.x - qk_wgs) * 256 + threadIdx.x;
    const int HH = a.H + a.Hk;
    const bool is_v = blockIdx.x >= (unsigned)qk_wgs;
    const long item = is_v ? u : u / LPH;
    const int per_row = is_v ? a.Hk * DH : HH;
    if (item >= (long)a.M * per_row) return;                  // whole groups
    const int row = (int)(item / per_row), c = (int)(item % per_row);
    const int pos = a.pos ? a.pos[row] : a.pos_base + row;
    // cache page and offset
    int pg = 0, off = pos;
    bool cached = true;
    if (a.slot != nullptr) {
        const int slot = a.slot[row];
        pg = slot >> a.page_shift;
        off = slot & (a.page_len - 1);
        cached = slot >= 0 && pg < a.n_pages;
    }
    auto sum = [&](int col, auto& v) {                        // v = the row's values from packed column col on
        constexpr int N = sizeof(v) / sizeof(float);
        const float* p = a.P + (size_t)row * a.ldn + col;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = p[e];
        for (int k = 1; k < a.ks; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += p[k * a.slice + e];
        if (a.bias != nullptr)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += a.bias[col + e];
    };
    if (is_v) {
        if (!cached) return;
        float v[1];
        sum(HH * DH + c, v);
        ((T*)a.V)[((size_t)pg * a.Hk * DH + c) * a.page_len + off] = elem_from_f32<T>(v[0]);
        return;
    }
    const int i = threadIdx.x % LPH;
    const bool is_q = c < a.H;
    float p[16], x[8], y[8];
    sum(c * DH + 16 * i, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = p[2 * e]; y[e] = p[2 * e + 1]; }
    const float* gain = is_q ? a.gq : a.gk;
    if (gain != nullptr) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[e] * x[e] + y[e] * y[e];
#pragma unroll
        for (int o = 1; o < LPH; o <<= 1) s += __shfl_xor(s, o);
        const float rs = 1.0f / sqrtf(s / (float)DH + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = x[e] * rs * gain[8 * i + e];
            y[e] = y[e] * rs * gain[DH / 2 + 8 * i + e];
        }
    }
    const float2* cs = a.rope + (size_t)min(max(pos, 0), a.max_pos - 1) * (DH / 2) + 8 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 t = cs[e];
        const float w = x[e] * t.x - y[e] * t.y;
        y[e] = y[e] * t.x + x[e] * t.y;
        x[e] = w;
    }
    if (!is_q) {
        if (!cached) return;
        T* dst = (T*)a.K + (((size_t)pg * a.Hk + (c - a.H)) * a.page_len + off) * DH + 8 * i;
        store8<T>(dst, x);
        store8<T>(dst + DH / 2, y);
        return;
    }
    T* dst = (T*)a.q + ((size_t)row * a.H + c) * DH + 8 * i;
    store8<T>(dst, x);
    store8<T>(dst + DH / 2, y);
    if constexpr (!XF32) {
        if (a.q_plane != 0) {                                 // the lo plane: what fp16 rounding left of hi
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = fminf(fmaxf(x[e], -65504.f), 65504.f);
                y[e] = fminf(fmaxf(y[e], -65504.f), 65504.f);
                x[e] -= (float)(_Float16)x[e];
                y[e] -= (float)(_Float16)y[e];
            }
            store8<T>(dst + a.q_plane, x);
            store8<T>(dst + a.q_plane + DH / 2, y);
        }
    }
}

// Attention rows [M][d], floats, into the O projection's operand fragments; padding rows up to gridDim.x get zeros.
template <bool XF32>
__global__ void __launch_bounds__(256) attn_operand_kernel(const float* rows, int M, int d, void* frag, int KCx) {
    const int m = blockIdx.x;
    for (int n = 4 * threadIdx.x; n < d; n += 4 * 256) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (m < M) v = *(const float4*)(rows + (size_t)m * d + n);
        xfrag_store4<XF32>(frag, m, n, KCx, v);
    }
}

}  // namespace dllm
