// Norm of every query and key head, rotation and cache write in one pass.
#pragma once

#include "batch_rules.hpp"
#include "common.hpp"

namespace dllm {

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
// squares is a few lane swaps.  A lane group takes `hp` heads of one row one after another with the
// row's cosines and the gains in registers (one head a group re-read 1 KiB of them through the L1
// for every 256 bytes of a head).
//
// V is written transposed.  Workgroups behind the first qk_wgs take QK_VROWS rows of one K/V head
// through LDS, then a thread writes keys of one dim: 16 bytes where the rows' slots run on from
// an aligned one (groups are cut at the slots' alignment, taken from the tile's first row),
// else one by one.
//
// What bounds it: HBM, each element read and written once: 16384 rows of 28 + 2 x 4 fp16 heads of 128 in 65 us,
// 4.7 TB/s, the rate of a large copy (4.76).  A window's rows are launch and latency: 4 to 256 rows 6 to 7.5 us.
template <typename T, int DH>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkArgs a, int qk_wgs, int hp) {
    constexpr int ES = sizeof(T);
    constexpr int LPH = DH / 16;                              // lanes per head
    constexpr int VLD = DH + 8 / ES;                          // LDS row of a V tile: 8 bytes off a multiple of the banks
    __shared__ __attribute__((aligned(16))) T vt[QK_VROWS * VLD];
    __shared__ int slot_s[QK_VROWS];
    if ((int)blockIdx.x < qk_wgs) {
        const int nq = (a.H + hp - 1) / hp, nk = (a.Hk + hp - 1) / hp;
        const long item = ((long)blockIdx.x * 256 + threadIdx.x) / LPH;
        const int i = threadIdx.x % LPH;
        if (item >= (long)a.T * (nq + nk)) return;            // whole groups: the swaps below stay inside one
        const int row = (int)(item / (nq + nk)), ch = (int)(item % (nq + nk));
        const bool is_q = ch < nq;
        const int h0 = (is_q ? ch : ch - nq) * hp, h1 = min(h0 + hp, is_q ? a.H : a.Hk);
        const T* src = (is_q ? (const T*)a.q + row * a.ld_q : (const T*)a.k + row * a.ld_k) + 8 * i;
        T* dst;
        if (is_q) {
            dst = (T*)a.qo + (size_t)row * a.H * DH + 8 * i;
        } else {
            const int slot = a.slot[row], pg = slot >> a.page_shift;
            if (slot < 0 || pg >= a.n_pages) return;
            const int off = slot & ((1 << a.page_shift) - 1);
            dst = (T*)a.kp + (((size_t)pg * a.Hk << a.page_shift) + off) * DH + 8 * i;
        }
        const size_t dstep = is_q ? DH : (size_t)DH << a.page_shift;      // from head to head
        const int pos = min(max(a.pos[row], 0), a.max_pos - 1);
        const float* cs = (const float*)(a.rope + (size_t)pos * (DH / 2) + 8 * i);
        float c[16], g0[8], g1[8];
        load8<float>(cs, *(float(*)[8])c);
        load8<float>(cs + 8, *(float(*)[8])(c + 8));
        const float* gain = is_q ? a.gq : a.gk;
        if (gain != nullptr) {
            load8<float>(gain + 8 * i, g0);
            load8<float>(gain + DH / 2 + 8 * i, g1);
        }
        float x[8], y[8], nx[8], ny[8];
        load8<T>(src + h0 * DH, nx);
        load8<T>(src + h0 * DH + DH / 2, ny);
        for (int h = h0; h < h1; ++h) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = nx[e]; y[e] = ny[e]; }
            if (h + 1 < h1) {
                load8<T>(src + (h + 1) * DH, nx);
                load8<T>(src + (h + 1) * DH + DH / 2, ny);
            }
            if (gain != nullptr) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) s += x[e] * x[e] + y[e] * y[e];
#pragma unroll
                for (int o = 1; o < LPH; o <<= 1) s += __shfl_xor(s, o);
                const float rs = 1.0f / sqrtf(s / (float)DH + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = x[e] * rs * g0[e];
                    y[e] = y[e] * rs * g1[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = x[e] * c[2 * e] - y[e] * c[2 * e + 1];
                y[e] = y[e] * c[2 * e] + x[e] * c[2 * e + 1];
                x[e] = u;
            }
            store8<T>(dst + h * dstep, x);
            store8<T>(dst + h * dstep + DH / 2, y);
        }
        return;
    }
    constexpr int KPS = 16 / ES;                              // keys of a 16-byte store
    constexpr int NCH = DH * ES / 16;                         // 16-byte pieces of a row
    const int u = blockIdx.x - qk_wgs, h = u % a.Hk, r0 = u / a.Hk * QK_VROWS, n = min(QK_VROWS, a.T - r0);
    if (threadIdx.x < QK_VROWS) {
        const int slot = threadIdx.x < n ? a.slot[r0 + threadIdx.x] : -1;
        slot_s[threadIdx.x] = (slot >> a.page_shift) < a.n_pages ? slot : -1;
    }
    for (int j = threadIdx.x; j < n * NCH; j += 256) {
        const int row = j / NCH, cc = j % NCH;
        u32x4_t w = ldg16((const T*)a.v + (r0 + row) * a.ld_v + h * DH + cc * KPS);
        if constexpr (__is_same(T, _Float16)) {               // fp16 saturates: an infinity becomes the largest value
            const f16x8_t e = __builtin_bit_cast(f16x8_t, w);
            f16x8_t o;
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = elem_from_f32<_Float16>((float)e[k]);
            w = __builtin_bit_cast(u32x4_t, o);
        }
        u32x2_t* p = (u32x2_t*)(vt + row * VLD + cc * KPS);
        p[0] = u32x2_t{w[0], w[1]};
        p[1] = u32x2_t{w[2], w[3]};
    }
    __syncthreads();
    const int phase = max(slot_s[0], 0) % KPS;
    const int groups = QK_VROWS / KPS + 1;                    // of rows [KPS k - phase, + KPS)
    for (int j = threadIdx.x; j < groups * DH; j += 256) {
        // eight neighbouring lanes take neighbouring groups of a dim (one 64- or 128-byte run), the last group on its own
        const int k = j < (groups - 1) * DH ? j % (groups - 1) : groups - 1;
        const int dim = j < (groups - 1) * DH ? j / (groups - 1) : j - (groups - 1) * DH;
        const int ra = KPS * k - phase;
        if (ra >= n) continue;
        bool run = ra >= 0 && ra + KPS <= n && slot_s[ra] >= 0 && slot_s[ra] % KPS == 0;
        if (run)
            for (int e = 1; e < KPS; ++e) run &= slot_s[ra + e] == slot_s[ra] + e;
        auto at = [&](int slot) {
            const int pg = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
            return (T*)a.vp + ((((size_t)pg * a.Hk + h) * DH + dim) << a.page_shift) + off;
        };
        if (run) {
            T e[KPS];
#pragma unroll
            for (int q = 0; q < KPS; ++q) e[q] = vt[(ra + q) * VLD + dim];
            __builtin_memcpy(__builtin_assume_aligned(at(slot_s[ra]), 16), e, 16);
        } else {
            for (int q = 0; q < KPS; ++q) {
                const int row = ra + q;
                if (row >= 0 && row < n && slot_s[row] >= 0) *at(slot_s[row]) = vt[row * VLD + dim];
            }
        }
    }
}

}  // namespace dllm
