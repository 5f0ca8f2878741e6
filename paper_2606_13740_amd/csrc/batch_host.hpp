// Checks of arguments that the batch operators share (host).
#pragma once

#include <string>

#include "batch_rules.hpp"
#include "host.hpp"

namespace dllm {

inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline int check_dtype(int dtype) {
    if (dtype != DLLM_F32 && dtype != DLLM_BF16 && dtype != DLLM_F16)
        return fail(DLLM_E_DTYPE, "dtype must be DLLM_F32, DLLM_BF16 or DLLM_F16");
    return DLLM_OK;
}

// A page size and count: shift of the page size, or -1 (recorded).
inline int page_shift(int page, int n_pages) {
    if (page != 32 && page != 64 && page != 128 && page != 256) {
        fail(DLLM_E_INVAL, "page must be 32, 64, 128 or 256");
        return -1;
    }
    if (n_pages < 1 || (long)n_pages * page >= (1l << 31)) {
        fail(DLLM_E_INVAL, "n_pages must be >= 1 and n_pages * page < 2^31");
        return -1;
    }
    return page == 32 ? 5 : (page == 64 ? 6 : (page == 128 ? 7 : 8));
}

inline int check_heads(int H, int Hk, int Dh) {
    if (H < 1 || H > 1024 || Hk < 1 || Hk > H || H % Hk != 0)
        return fail(DLLM_E_INVAL, "n_heads must be in [1, 1024] and n_kv_heads divide it");
    if (Dh != 32 && Dh != 64 && Dh != 128) return fail(DLLM_E_DTYPE, "head_dim must be 32, 64 or 128");
    return DLLM_OK;
}

inline bool row_stride_ok(const void* p, int64_t ld, int64_t width, int es) {
    return aligned(p, 16) && ld >= width && ld <= (1ll << 40) && (ld * es) % 16 == 0;
}

// A launch has fewer than 2^32 threads (here with a workgroup to spare).
inline bool grid_ok(long wgs, int threads) { return wgs < ((1l << 32) - 1024) / threads; }

constexpr int MAX_BATCH_ROWS = 1 << 24;

}  // namespace dllm
