// libdllm: C ABI of the batch operators (several sequences over a paged K/V cache).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/dllm.h"
#include "attn_paged.hpp"
#include "batch_plan.hpp"
#include "batch_rules.hpp"
#include "common.hpp"
#include "host.hpp"
#include "qk_rope.hpp"
#include "select.hpp"

using namespace dllm;

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check_dtype(int dtype) {
    if (dtype != DLLM_F32 && dtype != DLLM_BF16 && dtype != DLLM_F16)
        return fail(DLLM_E_DTYPE, "dtype must be DLLM_F32, DLLM_BF16 or DLLM_F16");
    return DLLM_OK;
}

// A page size and count: shift of the page size, or -1 (recorded).
int page_shift(int page, int n_pages) {
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

int check_heads(int H, int Hk, int Dh) {
    if (H < 1 || H > 1024 || Hk < 1 || Hk > H || H % Hk != 0)
        return fail(DLLM_E_INVAL, "n_heads must be in [1, 1024] and n_kv_heads divide it");
    if (Dh != 32 && Dh != 64 && Dh != 128) return fail(DLLM_E_DTYPE, "head_dim must be 32, 64 or 128");
    return DLLM_OK;
}

bool row_stride_ok(const void* p, int64_t ld, int64_t width, int es) {
    return aligned(p, 16) && ld >= width && ld <= (1ll << 40) && (ld * es) % 16 == 0;
}

// A launch has fewer than 2^32 threads (here with a workgroup to spare).
bool grid_ok(long wgs, int threads) { return wgs < ((1l << 32) - 1024) / threads; }

constexpr int MAX_BATCH_ROWS = 1 << 24;

}  // namespace

extern "C" {

int dllm_batch_plan(const int32_t* d_len, const int32_t* d_new, const int32_t* d_owned, int32_t* d_owned_out,
                    int32_t n_seqs, int32_t* d_table, int32_t table_ld, int32_t* d_free, const int32_t* d_n_free,
                    int32_t* d_n_free_out, int32_t n_pages, int32_t page, int32_t shared_pages, int32_t max_rows,
                    int32_t* d_row0, int32_t* d_pos, int32_t* d_slot, int32_t* d_seq, int32_t* d_lim,
                    int32_t* d_status, dllm_stream stream) {
    const void* ptrs[] = {d_len, d_new, d_owned, d_owned_out, d_table, d_free, d_n_free, d_n_free_out,
                          d_row0, d_pos, d_slot, d_seq, d_lim, d_status};
    for (const void* p : ptrs) {
        if (!p) return fail(DLLM_E_INVAL, "NULL argument");
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "integer arrays must be 4-byte aligned");
    }
    if (d_owned_out == d_owned || d_n_free_out == d_n_free)
        return fail(DLLM_E_INVAL, "owned_out and n_free_out must be other memory than their inputs");
    if (n_seqs < 1 || n_seqs > DLLM_MAX_SEQS) return fail(DLLM_E_INVAL, "n_seqs must be in [1, DLLM_MAX_SEQS]");
    const int shift = page_shift(page, n_pages);
    if (shift < 0) return DLLM_E_INVAL;
    if (table_ld < 1 || table_ld > (1 << 18) || (long)table_ld * page >= (1l << 31))
        return fail(DLLM_E_INVAL, "table_ld must be in [1, 2^18] and table_ld * page < 2^31");
    if (shared_pages < 0 || shared_pages > table_ld) return fail(DLLM_E_INVAL, "shared_pages must be in [0, table_ld]");
    if (max_rows < 1 || max_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "max_rows must be in [1, 2^24]");
    PlanArgs a{d_len, d_new, d_owned, d_owned_out, n_seqs, d_table, table_ld, d_free, d_n_free, d_n_free_out,
               n_pages, shift, shared_pages, max_rows, d_row0, d_pos, d_slot, d_seq, d_lim, d_status};
    const int row_wgs = std::min(192, ceil_div(max_rows, PLAN_NT));
    const int seq_wgs = std::min(64, ceil_div(std::max(n_seqs, n_pages), PLAN_NT));   // a CU for every workgroup
    hipLaunchKernelGGL(batch_plan_kernel, dim3(row_wgs + seq_wgs), dim3(PLAN_NT), 0, (hipStream_t)stream, a, row_wgs);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

}  // extern "C"

namespace {

template <typename T>
void launch_qk(const QkArgs& a, int Dh, hipStream_t s) {
    const int hp = qk_heads_per(a.T, a.H, a.Hk), wgs = (int)qk_wgs(a.T, a.H, a.Hk, Dh);
    const dim3 grid((unsigned)qk_grid(a.T, a.H, a.Hk, Dh));
    if (Dh == 128) hipLaunchKernelGGL((qk_norm_rope_kernel<T, 128>), grid, dim3(256), 0, s, a, wgs, hp);
    else if (Dh == 64) hipLaunchKernelGGL((qk_norm_rope_kernel<T, 64>), grid, dim3(256), 0, s, a, wgs, hp);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<T, 32>), grid, dim3(256), 0, s, a, wgs, hp);
}

// Every check of an attention call's sizes.
int check_attn(const dllm_attn_args* g, int& shift) {
    if (!g) return fail(DLLM_E_INVAL, "args is NULL");
    if (int rc = check_dtype(g->dtype)) return rc;
    if (int rc = check_heads(g->n_heads, g->n_kv_heads, g->head_dim)) return rc;
    if (g->dtype != DLLM_F32 && g->head_dim == 32) return fail(DLLM_E_DTYPE, "head_dim 32 needs DLLM_F32");
    if (g->n_rows < 0 || g->n_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_rows must be in [0, 2^24]");
    if (g->n_seqs < 1 || g->n_seqs > DLLM_MAX_SEQS) return fail(DLLM_E_INVAL, "n_seqs must be in [1, DLLM_MAX_SEQS]");
    if ((shift = page_shift(g->page, g->n_pages)) < 0) return DLLM_E_INVAL;
    if (g->table_ld < 1 || (long)g->table_ld * g->page >= (1l << 31))
        return fail(DLLM_E_INVAL, "table_ld must be >= 1 and table_ld * page < 2^31");
    if (g->max_len < 0 || g->max_len > std::min(g->table_ld * g->page, 1 << 30))
        return fail(DLLM_E_INVAL, "max_len must be in [0, table_ld * page] and at most 2^30");
    if (g->max_rows < 0) return fail(DLLM_E_INVAL, "max_rows must be >= 0");
    if (g->shared_len < 0 || g->shared_len % g->page != 0 || g->shared_len > g->table_ld * g->page)
        return fail(DLLM_E_INVAL, "shared_len must be a multiple of page in [0, table_ld * page]");
    if (!std::isfinite(g->scale)) return fail(DLLM_E_INVAL, "scale must be finite");
    if ((long)g->n_rows * (g->n_heads / g->n_kv_heads) >= (1l << 31))
        return fail(DLLM_E_INVAL, "n_rows times the query heads of a K/V head must be < 2^31");
    const AttnPlan p = attn_plan(g);
    if (!grid_ok(p.wgs_s + p.wgs_o, 256) || !grid_ok((long)g->n_rows * g->n_heads, g->head_dim / 4))
        return fail(DLLM_E_INVAL, "n_seqs, max_rows and n_rows need too many workgroups");
    return DLLM_OK;
}

template <typename T, int DH>
void launch_attn_dh(PagedArgs a, const AttnPlan& p, hipStream_t s) {
    constexpr int SUB = sizeof(T) == 4 ? 1 : 2;
    const dim3 grid((unsigned)(p.wgs_s + p.wgs_o));
#define ATTN(QG_, RT_, KG_) \
    hipLaunchKernelGGL((attn_paged_kernel<T, DH, QG_, RT_, KG_, SUB>), grid, dim3(QG_ * KG_ * 64), 0, s, a)
    if constexpr (sizeof(T) == 2) {
        if (p.qt == 2) ATTN(4, 32, 1);
        else if (p.qg == 4) ATTN(4, 16, 1);
        else if (p.qg == 2) ATTN(2, 16, 2);
        else ATTN(1, 16, 2);
    } else {
        if (p.qg == 4) ATTN(4, 16, 1);
        else if (p.qg == 2) ATTN(2, 16, 1);
        else ATTN(1, 16, 1);
    }
#undef ATTN
    if (!a.direct)
        hipLaunchKernelGGL((attn_paged_merge_kernel<T, DH>), dim3(ceil_div((long)a.T * a.H, 256 / (DH / 4))), dim3(256), 0,
                           s, a);
}

template <typename T>
void launch_attn(const PagedArgs& a, const AttnPlan& p, int Dh, hipStream_t s) {
    if (Dh == 128) launch_attn_dh<T, 128>(a, p, s);
    else if (Dh == 64) launch_attn_dh<T, 64>(a, p, s);
    else if constexpr (sizeof(T) == 4) launch_attn_dh<T, 32>(a, p, s);
}

size_t select_ws_bytes(const dllm_select_args* g) {
    const int n = select_ranges(g->vocab);
    return n == 1 ? 0 : (size_t)g->n_rows * n * sizeof(SelectPart);
}

template <typename T>
void launch_select(const SelectArgs& a, SelectPart* part, hipStream_t s) {
    const int n = select_ranges(a.V), per = select_rows_per(a.T, n);
    const long wgs = select_wgs(a.T, n);
    if (select_four_waves(wgs)) hipLaunchKernelGGL((select_kernel<T, 3>), dim3((unsigned)wgs), dim3(SEL_NT), 0, s, a, part, n, per);
    else hipLaunchKernelGGL((select_kernel<T, 5>), dim3((unsigned)wgs), dim3(SEL_NT), 0, s, a, part, n, per);
    if (n > 1) hipLaunchKernelGGL(select_merge_kernel, dim3(ceil_div(a.T, 4)), dim3(256), 0, s, a, (const SelectPart*)part, n);
}

int check_select(const dllm_select_args* g) {
    if (!g) return fail(DLLM_E_INVAL, "args is NULL");
    if (int rc = check_dtype(g->dtype)) return rc;
    if (g->n_rows < 0 || g->n_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_rows must be in [0, 2^24]");
    if (g->vocab < 1 || g->vocab > (1 << 24)) return fail(DLLM_E_INVAL, "vocab must be in [1, 2^24]");
    if (g->mask_id < -1 || g->mask_id >= g->vocab) return fail(DLLM_E_INVAL, "mask_id must be -1 or an id");
    if (g->n_seqs < 1 || g->n_seqs > DLLM_MAX_SEQS) return fail(DLLM_E_INVAL, "n_seqs must be in [1, DLLM_MAX_SEQS]");
    return DLLM_OK;
}

}  // namespace

namespace dllm {

// Every check of a selection.
int select_check(const dllm_select_args* g) {
    if (int rc = check_select(g)) return rc;
    if (!g->d_logits || !g->d_out_id || !g->d_out_conf) return fail(DLLM_E_INVAL, "NULL argument");
    if (!g->d_row0 && g->n_seqs != 1) return fail(DLLM_E_INVAL, "row0 may be NULL only for one sequence");
    if (g->d_hist && !g->d_hist0) return fail(DLLM_E_INVAL, "hist needs hist0");
    if (!g->d_hist && (g->d_repetition || g->d_presence || g->d_frequency || g->d_n_prompt))
        return fail(DLLM_E_INVAL, "penalties need a history");
    if ((g->d_bias == nullptr) != (g->d_bias_id == nullptr) || (g->d_bias == nullptr) != (g->d_bias0 == nullptr))
        return fail(DLLM_E_INVAL, "bias, bias_id and bias0 must all be set or all be NULL");
    if (g->d_allow) {
        if (g->n_allow < 1 || g->allow_ld < 1) return fail(DLLM_E_INVAL, "n_allow and allow_ld must be >= 1");
        if ((long)g->allow_ld * 32 < g->vocab) return fail(DLLM_E_INVAL, "allow_ld words do not cover the vocabulary");
        if (!g->d_allow_row && g->n_allow < g->n_rows) return fail(DLLM_E_INVAL, "a mask per row needs n_allow >= n_rows");
    } else if (g->d_allow_row) {
        return fail(DLLM_E_INVAL, "allow_row needs allow");
    }
    const int es = esize(g->dtype);
    if (g->ld < g->vocab || g->ld > (1ll << 40) || !aligned(g->d_logits, es))
        return fail(DLLM_E_INVAL, "logits: stride of at least a row, pointer aligned to its elements");
    if (g->d_out_logits && (g->ld_out < g->vocab || g->ld_out > (1ll << 40) || !aligned(g->d_out_logits, es)))
        return fail(DLLM_E_INVAL, "out_logits: stride of at least a row, pointer aligned to its elements");
    if (g->d_out_logits == g->d_logits && g->ld_out != g->ld)
        return fail(DLLM_E_INVAL, "out_logits may be logits only with the same stride");
    const void* ints[] = {g->d_row0, g->d_hist, g->d_hist0, g->d_n_prompt, g->d_repetition, g->d_presence,
                          g->d_frequency, g->d_bias_id, g->d_bias, g->d_bias0, g->d_allow, g->d_allow_row,
                          g->d_out_id, g->d_out_conf};
    for (const void* p : ints)
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "arrays of 32-bit values must be 4-byte aligned");
    if (g->n_rows == 0) return DLLM_OK;               // (no workspace, no launch)
    const size_t need = select_ws_bytes(g);
    if (!grid_ok(select_wgs(g->n_rows, select_ranges(g->vocab)), SEL_NT))
        return fail(DLLM_E_INVAL, "n_rows and vocab need too many workgroups");
    if (need > 0 && (!g->d_ws || !aligned(g->d_ws, 16))) return fail(DLLM_E_INVAL, "workspace: NULL or not 16-byte aligned");
    if (need > g->ws_bytes)
        return fail(DLLM_E_CAPACITY, "the call needs " + std::to_string(need) + " bytes of workspace");
    return DLLM_OK;
}

int attention_paged(const dllm_attn_args* g, bool out_f32, hipStream_t s) {
    int shift = 0;
    if (int rc = check_attn(g, shift)) return rc;
    if (!g->d_q || !g->d_k_pages || !g->d_v_pages || !g->d_table || !g->d_row0 || !g->d_len || !g->d_out)
        return fail(DLLM_E_INVAL, "NULL argument");
    const int es = esize(g->dtype);
    const int64_t w = (int64_t)g->n_heads * g->head_dim;
    if (!row_stride_ok(g->d_q, g->ld_q, w, es) || !row_stride_ok(g->d_out, g->ld_out, w, out_f32 ? 4 : es))
        return fail(DLLM_E_INVAL, "q, out: pointers and row strides must be multiples of 16 bytes, strides at least a row");
    if (!aligned(g->d_k_pages, 16) || !aligned(g->d_v_pages, 16) || !aligned(g->d_table, 4) || !aligned(g->d_row0, 4) ||
        !aligned(g->d_len, 4) || !aligned(g->d_lim, 4))
        return fail(DLLM_E_INVAL, "pages must be 16-byte aligned, integer arrays 4-byte");
    if (g->n_rows == 0) return DLLM_OK;
    const AttnPlan p = attn_plan(g);
    const size_t need = attn_ws_bytes(g, p);
    if (need > 0 && (!g->d_ws || !aligned(g->d_ws, 16))) return fail(DLLM_E_INVAL, "workspace: NULL or not 16-byte aligned");
    if (need > g->ws_bytes)
        return fail(DLLM_E_CAPACITY, "the call needs " + std::to_string(need) + " bytes of workspace");
    PagedArgs a{};
    a.q = g->d_q; a.ld_q = g->ld_q; a.kp = g->d_k_pages; a.vp = g->d_v_pages; a.table = g->d_table; a.table_ld = g->table_ld;
    a.row0 = g->d_row0; a.len = g->d_len; a.lim = g->d_lim; a.out = g->d_out; a.ld_out = g->ld_out;
    a.T = g->n_rows; a.B = g->n_seqs; a.H = g->n_heads; a.Hk = g->n_kv_heads; a.G = a.H / a.Hk; a.page_shift = shift;
    a.n_pages = g->n_pages; a.shared = p.shared; a.max_rows = g->max_rows; a.max_len = g->max_len;
    a.sl2 = g->scale == 0.f ? 1.f : std::fabs(g->scale) * 1.4426950408889634f;
    a.qmul = g->scale == 0.f ? 0.f : (g->scale < 0.f ? -1.f : 1.f);
    a.opart = (float*)g->d_ws;
    a.mlpart = a.opart + (size_t)(p.ns_s + p.ns_o) * a.T * a.H * g->head_dim;
    a.ns_s = p.ns_s; a.nt_s = p.nt_s; a.ns_o = p.ns_o; a.nt_o = p.nt_o; a.n_s = (int)p.wgs_s;
    a.direct = p.direct();
    a.out_f32 = out_f32;
    if (g->dtype == DLLM_F32) launch_attn<float>(a, p, g->head_dim, s);
    else if (g->dtype == DLLM_F16) launch_attn<_Float16>(a, p, g->head_dim, s);
    else launch_attn<__bf16>(a, p, g->head_dim, s);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

}  // namespace dllm

extern "C" {

int dllm_qk_norm_rope(const dllm_qk_args* g, dllm_stream stream) {
    if (!g) return fail(DLLM_E_INVAL, "args is NULL");
    if (int rc = check_dtype(g->dtype)) return rc;
    if (int rc = check_heads(g->n_heads, g->n_kv_heads, g->head_dim)) return rc;
    if (g->n_rows < 0 || g->n_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_rows must be in [0, 2^24]");
    const int shift = page_shift(g->page, g->n_pages);
    if (shift < 0) return DLLM_E_INVAL;
    if (g->max_pos < 1) return fail(DLLM_E_INVAL, "max_pos must be >= 1");
    if (!(g->eps >= 0.f) || !std::isfinite(g->eps)) return fail(DLLM_E_INVAL, "eps must be finite and >= 0");
    if (!g->d_q || !g->d_k || !g->d_v || !g->d_rope || !g->d_pos || !g->d_slot || !g->d_q_out || !g->d_k_pages ||
        !g->d_v_pages)
        return fail(DLLM_E_INVAL, "NULL argument");
    const int es = esize(g->dtype);
    const int64_t wq = (int64_t)g->n_heads * g->head_dim, wk = (int64_t)g->n_kv_heads * g->head_dim;
    if (!row_stride_ok(g->d_q, g->ld_q, wq, es) || !row_stride_ok(g->d_k, g->ld_k, wk, es) ||
        !row_stride_ok(g->d_v, g->ld_v, wk, es))
        return fail(DLLM_E_INVAL, "q, k, v: pointers and row strides must be multiples of 16 bytes, strides at least a row");
    if (!aligned(g->d_q_out, 16) || !aligned(g->d_k_pages, 16) || !aligned(g->d_v_pages, 16) ||
        !aligned(g->d_rope, 16) || !aligned(g->d_q_gain, 16) || !aligned(g->d_k_gain, 16) || !aligned(g->d_pos, 4) ||
        !aligned(g->d_slot, 4))
        return fail(DLLM_E_INVAL, "pointers must be 16-byte aligned (integer arrays: 4)");
    if (g->d_q_out == g->d_q && g->ld_q != wq) return fail(DLLM_E_INVAL, "q_out may be q only if q is contiguous");
    if (!grid_ok(qk_grid(g->n_rows, g->n_heads, g->n_kv_heads, g->head_dim), 256))
        return fail(DLLM_E_INVAL, "n_rows and n_heads need too many workgroups");
    if (g->n_rows == 0) return DLLM_OK;
    QkArgs a{g->d_q, g->d_k, g->d_v, g->ld_q, g->ld_k, g->ld_v, g->d_q_gain, g->d_k_gain, (const float2*)g->d_rope,
             g->d_pos, g->d_slot, g->d_q_out, g->d_k_pages, g->d_v_pages, g->n_rows, g->n_heads, g->n_kv_heads, shift,
             g->n_pages, g->max_pos, g->eps};
    hipStream_t s = (hipStream_t)stream;
    if (g->dtype == DLLM_F32) launch_qk<float>(a, g->head_dim, s);
    else if (g->dtype == DLLM_F16) launch_qk<_Float16>(a, g->head_dim, s);
    else launch_qk<__bf16>(a, g->head_dim, s);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

int dllm_attention_paged_ws(const dllm_attn_args* g, size_t* bytes) {
    if (!bytes) return fail(DLLM_E_INVAL, "bytes is NULL");
    int shift = 0;
    if (int rc = check_attn(g, shift)) return rc;
    *bytes = attn_ws_bytes(g, attn_plan(g));
    return DLLM_OK;
}

int dllm_attention_paged(const dllm_attn_args* g, dllm_stream stream) { return attention_paged(g, false, (hipStream_t)stream); }

int dllm_select_ws(const dllm_select_args* g, size_t* bytes) {
    if (!bytes) return fail(DLLM_E_INVAL, "bytes is NULL");
    if (int rc = check_select(g)) return rc;
    *bytes = select_ws_bytes(g);
    return DLLM_OK;
}

int dllm_select(const dllm_select_args* g, dllm_stream stream) {
    if (int rc = select_check(g)) return rc;
    if (g->n_rows == 0) return DLLM_OK;
    SelectArgs a{g->d_logits, g->ld, g->n_rows, g->vocab, g->mask_id, g->n_seqs, g->d_row0, g->d_hist, g->d_hist0,
                 g->d_n_prompt, g->d_repetition, g->d_presence, g->d_frequency, g->d_bias_id, g->d_bias, g->d_bias0,
                 g->d_allow, g->n_allow, g->allow_ld, g->d_allow_row, g->d_out_logits, g->ld_out, g->d_out_id,
                 g->d_out_conf};
    hipStream_t s = (hipStream_t)stream;
    SelectPart* part = (SelectPart*)g->d_ws;
    if (g->dtype == DLLM_F32) launch_select<float>(a, part, s);
    else if (g->dtype == DLLM_F16) launch_select<_Float16>(a, part, s);
    else launch_select<__bf16>(a, part, s);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

}  // extern "C"
