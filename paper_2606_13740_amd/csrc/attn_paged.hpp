// Attention of a batch of sequences that share a prefix, over a paged cache.
#pragma once

#include "common.hpp"
#include "qk_rope.hpp"

namespace dllm {

struct PagedArgs {
    const void* q;
    long ld_q;
    const void *kp, *vp;          // [n_pages][Hk][page][Dh], [n_pages][Hk][Dh][page]
    const int* table;
    int table_ld;
    const int *row0, *len, *lim;
    void* out;
    long ld_out;
    int T, B, H, Hk, page_shift, n_pages, shared, max_rows, max_len;
    float scale;
};

// Largest b with row0[b] <= r, or -1 where r is no row of a sequence.
__device__ __forceinline__ int row_seq(const int* row0, int B, int r) {
    if (r < row0[0] || r >= row0[B]) return -1;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row0[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One workgroup of 4 waves per (row, head): wave w takes the 64-key chunks w, w + 4, ...,
// scores with one key per lane, outputs with one dim (DH 128: two) per lane; the waves'
// (max, sum, output) are merged in wave order.
template <typename T, int DH>
__global__ void __launch_bounds__(256) attn_paged_row_kernel(PagedArgs a) {
    constexpr int NW = 4, ND = (DH + 63) / 64;
    __shared__ float q_s[DH], p_s[NW][64], o_s[NW][DH], m_s[NW], l_s[NW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x, h = blockIdx.y, hk = h / (a.H / a.Hk);
    const int b = row_seq(a.row0, a.B, row);
    if (b < 0) return;
    int n = min(min(a.len[b], a.max_len), a.table_ld << a.page_shift);
    if (a.lim != nullptr) n = min(n, a.lim[row]);
    if (threadIdx.x < DH) q_s[threadIdx.x] = elem_to_f32<T>(((const T*)a.q)[row * a.ld_q + h * DH + threadIdx.x]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = 0.f;
    const int mask = (1 << a.page_shift) - 1;
    for (int k0 = 64 * wave; k0 < n; k0 += 64 * NW) {
        const int key = k0 + lane;
        int pg = -1;
        if (key < n) pg = a.table[(size_t)(key < a.shared ? 0 : b) * a.table_ld + (key >> a.page_shift)];
        if (pg >= a.n_pages) pg = -1;
        float s = -INFINITY;
        if (pg >= 0) {
            const T* kr = (const T*)a.kp + ((((size_t)pg * a.Hk + hk) << a.page_shift) + (key & mask)) * DH;
            s = 0.f;
            for (int d = 0; d < DH; ++d) s = fmaf(q_s[d], elem_to_f32<T>(kr[d]), s);
            s *= a.scale;
        }
        const float mn = fmaxf(m, warp_max(s));
        if (mn == -INFINITY) continue;
        const float alpha = expf(m - mn), p = pg >= 0 ? expf(s - mn) : 0.f;
        l = l * alpha + warp_sum(p);
        m = mn;
        p_s[wave][lane] = p;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const int dim = min(lane + 64 * d, DH - 1);       // every lane stays: the pages come from all of them
            float acc = o[d] * alpha;
            for (int j = 0; j < 64; ++j) {
                const int pj = __shfl(pg, j);
                if (pj < 0) continue;
                const T v = ((const T*)a.vp)[((((size_t)pj * a.Hk + hk) * DH + dim) << a.page_shift) + ((k0 + j) & mask)];
                acc = fmaf(p_s[wave][j], elem_to_f32<T>(v), acc);
            }
            o[d] = acc;
        }
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
        if (lane + 64 * d < DH) o_s[wave][lane + 64 * d] = o[d];
    if (lane == 0) {
        m_s[wave] = m;
        l_s[wave] = l;
    }
    __syncthreads();
    if (threadIdx.x >= DH) return;
    float mx = m_s[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) mx = fmaxf(mx, m_s[w]);
    float L = 0.f, ov = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float e = m_s[w] == -INFINITY ? 0.f : expf(m_s[w] - mx);
        L += l_s[w] * e;
        ov += o_s[w][threadIdx.x] * e;
    }
    ((T*)a.out)[row * a.ld_out + h * DH + threadIdx.x] = elem_from_f32<T>(L > 0.f ? ov / L : 0.f);
}

}  // namespace dllm
