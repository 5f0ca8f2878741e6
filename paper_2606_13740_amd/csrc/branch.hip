// libdllm: C ABI of the branching operators (trees of drafted rows, candidates, forks of sequences).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/dllm.h"
#include "batch_host.hpp"
#include "cache_move.hpp"
#include "logprobs.hpp"
#include "tree_plan.hpp"

using namespace dllm;

namespace {

int check_cache(const dllm_cache* c, int& shift) {
    if (!c || !c->d_pages) return fail(DLLM_E_INVAL, "NULL argument");
    if (int rc = check_dtype(c->dtype)) return rc;
    if (int rc = check_heads(c->n_kv_heads, c->n_kv_heads, c->head_dim)) return rc;
    if (c->n_layers < 1 || c->n_layers > 4096) return fail(DLLM_E_INVAL, "n_layers must be in [1, 4096]");
    if ((shift = page_shift(c->page, c->n_pages)) < 0) return DLLM_E_INVAL;
    if (!aligned(c->d_pages, 16)) return fail(DLLM_E_INVAL, "pages must be 16-byte aligned");
    return DLLM_OK;
}

CacheArgs cache_args(const dllm_cache* c, int shift) {
    return CacheArgs{(char*)c->d_pages, c->n_layers, c->n_kv_heads, c->head_dim, shift, c->n_pages};
}

int check_table(int table_ld, int page) {
    if (table_ld < 1 || table_ld > (1 << 18) || (long)table_ld * page >= (1l << 31))
        return fail(DLLM_E_INVAL, "table_ld must be in [1, 2^18] and table_ld * page < 2^31");
    return DLLM_OK;
}

int check_seqs(int n_seqs) {
    if (n_seqs < 1 || n_seqs > DLLM_MAX_SEQS) return fail(DLLM_E_INVAL, "n_seqs must be in [1, DLLM_MAX_SEQS]");
    return DLLM_OK;
}

// Every check of a log probability call's sizes.
int check_logprobs(const dllm_logprobs_args* g) {
    if (!g) return fail(DLLM_E_INVAL, "args is NULL");
    if (int rc = check_dtype(g->dtype)) return rc;
    if (g->n_rows < 0 || g->n_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_rows must be in [0, 2^24]");
    if (g->vocab < 1 || g->vocab > (1 << 24)) return fail(DLLM_E_INVAL, "vocab must be in [1, 2^24]");
    if (g->mask_id < -1 || g->mask_id >= g->vocab) return fail(DLLM_E_INVAL, "mask_id must be -1 or an id");
    if (g->top < 0 || g->top > DLLM_MAX_TOP) return fail(DLLM_E_INVAL, "top must be in [0, DLLM_MAX_TOP]");
    if (g->n_tok < 0 || g->n_tok > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_tok must be in [0, 2^24]");
    return DLLM_OK;
}

// apart: given tokens that get a launch of their own.
template <typename T>
void launch_logprobs(const LogprobArgs& a, int apart, hipStream_t s) {
    const dim3 grid((unsigned)((long)a.T * a.parts));
    if (a.top > 0) hipLaunchKernelGGL((logprobs_kernel<T, true>), grid, dim3(LP_NT), 0, s, a);
    else hipLaunchKernelGGL((logprobs_kernel<T, false>), grid, dim3(LP_NT), 0, s, a);
    if (a.parts > 1) hipLaunchKernelGGL((logprobs_merge_kernel<T>), dim3(a.T), dim3(LP_NT), 0, s, a);
    if (apart > 0) hipLaunchKernelGGL((logprobs_tokens_kernel<T>), dim3(ceil_div(apart, LP_NT)), dim3(LP_NT), 0, s, a, apart);
}

// Tokens of a call that get a launch of their own: all or none.
int tokens_apart(const dllm_logprobs_args* g) {
    return lp_tokens_apart(g->n_rows, g->n_tok, g->d_tok_row != nullptr) ? g->n_tok : 0;
}

size_t logprobs_ws(const dllm_logprobs_args* g) {
    return lp_ws_bytes(g->n_rows, g->vocab, g->top) + (tokens_apart(g) > 0 ? (size_t)g->n_rows * sizeof(float2) : 0);
}

template <typename E>
void launch_compact(const CompactArgs& a, hipStream_t s) {
    const int hp = compact_heads_per(a.B, a.c.L, a.c.Hk);
    const dim3 grid((unsigned)compact_wgs(a.B, a.c.L, a.c.Hk, a.c.Dh, sizeof(E)));
    if (a.c.Dh == 128) hipLaunchKernelGGL((cache_compact_kernel<E, 128>), grid, dim3(COMPACT_NT), 0, s, a, hp);
    else if (a.c.Dh == 64) hipLaunchKernelGGL((cache_compact_kernel<E, 64>), grid, dim3(COMPACT_NT), 0, s, a, hp);
    else hipLaunchKernelGGL((cache_compact_kernel<E, 32>), grid, dim3(COMPACT_NT), 0, s, a, hp);
}

template <typename E>
void launch_copies(const CacheArgs& c, const ForkArgs& a, int* table_out, hipStream_t s) {
    // (tables are vectors where the rows of both are)
    const bool vec = a.vec && aligned(table_out, 16);
    const dim3 grid((unsigned)std::min<long>((long)a.B * c.L * 2 * c.Hk, 8 * N_CU));
#define COPY(DH_) \
    hipLaunchKernelGGL((fork_copy_kernel<E, DH_>), grid, dim3(256), 0, s, c, a.n_copies, a.copies, a.rows, a.B, a.table, table_out, a.ld, vec)
    if (c.Dh == 128) COPY(128);
    else if (c.Dh == 64) COPY(64);
    else COPY(32);
#undef COPY
}

}  // namespace

extern "C" {

int dllm_tree_plan(const int32_t* d_parent, const int32_t* d_row0, const int32_t* d_len, int32_t n_rows, int32_t n_seqs,
                   int32_t* d_pos, uint32_t* d_mask, int32_t mask_ld, dllm_stream stream) {
    const void* ptrs[] = {d_parent, d_row0, d_len, d_pos, d_mask};
    for (const void* p : ptrs) {
        if (!p) return fail(DLLM_E_INVAL, "NULL argument");
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "integer arrays must be 4-byte aligned");
    }
    if (d_pos == d_parent) return fail(DLLM_E_INVAL, "pos must be other memory than parent");
    if (n_rows < 0 || n_rows > MAX_BATCH_ROWS) return fail(DLLM_E_INVAL, "n_rows must be in [0, 2^24]");
    if (int rc = check_seqs(n_seqs)) return rc;
    if (mask_ld < 1 || mask_ld > TREE_MAX_LD) return fail(DLLM_E_INVAL, "mask_ld must be in [1, 32]");
    if (n_rows == 0) return DLLM_OK;
    TreeArgs a{d_parent, d_row0, d_len, n_rows, n_seqs, d_pos, d_mask, mask_ld};
    hipLaunchKernelGGL(tree_plan_kernel, dim3(n_seqs), dim3(TREE_NT), 0, (hipStream_t)stream, a);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

int dllm_attention_tree(const dllm_attn_args* g, const uint32_t* d_mask, int32_t mask_ld, dllm_stream stream) {
    if (!d_mask || !aligned(d_mask, 4)) return fail(DLLM_E_INVAL, "mask: NULL or not 4-byte aligned");
    if (mask_ld < 1 || mask_ld > (1 << 24)) return fail(DLLM_E_INVAL, "mask_ld must be in [1, 2^24]");
    if (g && (int64_t)g->n_rows * mask_ld >= (1ll << 29)) return fail(DLLM_E_INVAL, "n_rows * mask_ld must be < 2^29");
    return attention_paged(g, d_mask, mask_ld, false, (hipStream_t)stream);
}

int dllm_attention_tree_ws(const dllm_attn_args* g, size_t* bytes) { return attention_ws(g, true, bytes); }

int dllm_logprobs_ws(const dllm_logprobs_args* g, size_t* bytes) {
    if (!bytes) return fail(DLLM_E_INVAL, "bytes is NULL");
    if (int rc = check_logprobs(g)) return rc;
    *bytes = logprobs_ws(g);
    return DLLM_OK;
}

int dllm_logprobs(const dllm_logprobs_args* g, dllm_stream stream) {
    if (int rc = check_logprobs(g)) return rc;
    if (!g->d_logits) return fail(DLLM_E_INVAL, "NULL argument");
    if (g->n_tok > 0 && (!g->d_tok || !g->d_logp)) return fail(DLLM_E_INVAL, "tokens need tok and logp");
    if (!g->d_tok_row && g->n_tok > g->n_rows) return fail(DLLM_E_INVAL, "without tok_row there is a token per row at most");
    if (g->top > 0 && (!g->d_top_id || !g->d_top_logp)) return fail(DLLM_E_INVAL, "top needs top_id and top_logp");
    if (g->ld < g->vocab || g->ld > (1ll << 40) || !aligned(g->d_logits, esize(g->dtype)))
        return fail(DLLM_E_INVAL, "logits: stride of at least a row, pointer aligned to its elements");
    const void* ints[] = {g->d_tok, g->d_tok_row, g->d_logp, g->d_entropy, g->d_top_id, g->d_top_logp};
    for (const void* p : ints)
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "arrays of 32-bit values must be 4-byte aligned");
    if (g->n_rows == 0) return g->n_tok == 0 ? DLLM_OK : fail(DLLM_E_INVAL, "tokens need rows");
    const int parts = lp_parts(g->n_rows, g->vocab);
    if (!grid_ok((long)g->n_rows * parts, LP_NT)) return fail(DLLM_E_INVAL, "n_rows and vocab need too many workgroups");
    const size_t need = logprobs_ws(g);
    if (need > 0 && (!g->d_ws || !aligned(g->d_ws, 16))) return fail(DLLM_E_INVAL, "workspace: NULL or not 16-byte aligned");
    if (need > g->ws_bytes)
        return fail(DLLM_E_CAPACITY, "the call needs " + std::to_string(need) + " bytes of workspace");
    const int apart = tokens_apart(g);
    LogprobArgs a{g->d_logits, g->ld, g->n_rows, g->vocab, g->mask_id, g->n_tok - apart, g->top, g->d_tok, g->d_tok_row, g->d_logp,
                  g->d_entropy, g->d_top_id, g->d_top_logp, parts, lp_per(g->n_rows, g->vocab), (LogStat*)g->d_ws, nullptr, nullptr};
    a.keys = (uint64_t*)((char*)g->d_ws + (size_t)a.T * parts * (LP_NT / 64) * sizeof(LogStat));
    if (apart > 0) a.row_stat = (float2*)((char*)g->d_ws + lp_ws_bytes(a.T, a.V, a.top));
    hipStream_t s = (hipStream_t)stream;
    if (g->dtype == DLLM_F32) launch_logprobs<float>(a, apart, s);
    else if (g->dtype == DLLM_F16) launch_logprobs<_Float16>(a, apart, s);
    else launch_logprobs<__bf16>(a, apart, s);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

int dllm_cache_compact(const dllm_cache* cache, const int32_t* d_table, int32_t table_ld, const int32_t* d_base,
                       const int32_t* d_path, int32_t path_ld, const int32_t* d_n, int32_t n_seqs, dllm_stream stream) {
    int shift = 0;
    if (int rc = check_cache(cache, shift)) return rc;
    const void* ptrs[] = {d_table, d_base, d_path, d_n};
    for (const void* p : ptrs) {
        if (!p) return fail(DLLM_E_INVAL, "NULL argument");
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "integer arrays must be 4-byte aligned");
    }
    if (int rc = check_seqs(n_seqs)) return rc;
    if (int rc = check_table(table_ld, cache->page)) return rc;
    if (path_ld < 1 || path_ld > 32 * TREE_MAX_LD) return fail(DLLM_E_INVAL, "path_ld must be in [1, 1024]");
    CompactArgs a{cache_args(cache, shift), d_table, table_ld, d_base, d_path, path_ld, d_n, n_seqs};
    if (!grid_ok(compact_wgs(n_seqs, a.c.L, a.c.Hk, a.c.Dh, esize(cache->dtype)), COMPACT_NT)) return fail(DLLM_E_INVAL, "the cache and n_seqs need too many workgroups");
    if (cache->dtype == DLLM_F32) launch_compact<uint32_t>(a, (hipStream_t)stream);
    else launch_compact<uint16_t>(a, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

int dllm_batch_fork_ws(int32_t n_seqs, int32_t n_pages, size_t* bytes) {
    if (!bytes) return fail(DLLM_E_INVAL, "bytes is NULL");
    if (int rc = check_seqs(n_seqs)) return rc;
    if (page_shift(32, n_pages) < 0) return DLLM_E_INVAL;
    *bytes = fork_ws_bytes(n_seqs, n_pages);
    return DLLM_OK;
}

int dllm_batch_fork(const dllm_cache* cache, const dllm_fork_args* g, dllm_stream stream) {
    int shift = 0;
    if (!g) return fail(DLLM_E_INVAL, "args is NULL");
    if (int rc = check_cache(cache, shift)) return rc;
    const void* ptrs[] = {g->d_src, g->d_keep, g->d_owned, g->d_owned_out, g->d_table, g->d_table_out, g->d_free, g->d_n_free,
                          g->d_n_free_out, g->d_status};
    for (const void* p : ptrs) {
        if (!p) return fail(DLLM_E_INVAL, "NULL argument");
        if (!aligned(p, 4)) return fail(DLLM_E_INVAL, "integer arrays must be 4-byte aligned");
    }
    if (g->d_owned_out == g->d_owned || g->d_n_free_out == g->d_n_free || g->d_table_out == g->d_table)
        return fail(DLLM_E_INVAL, "owned_out, table_out and n_free_out must be other memory than their inputs");
    if (int rc = check_seqs(g->n_seqs)) return rc;
    if (int rc = check_table(g->table_ld, cache->page)) return rc;
    if (g->shared_pages < 0 || g->shared_pages > g->table_ld) return fail(DLLM_E_INVAL, "shared_pages must be in [0, table_ld]");
    const size_t need = fork_ws_bytes(g->n_seqs, cache->n_pages);
    if (!g->d_ws || !aligned(g->d_ws, 16)) return fail(DLLM_E_INVAL, "workspace: NULL or not 16-byte aligned");
    if (need > g->ws_bytes)
        return fail(DLLM_E_CAPACITY, "the call needs " + std::to_string(need) + " bytes of workspace");
    int4* copies = (int4*)((char*)g->d_ws + 16);
    uint2* rows = (uint2*)(copies + g->n_seqs);
    ForkArgs a{g->d_src, g->d_keep, g->d_owned, g->d_owned_out, g->d_table, g->table_ld,
               g->table_ld % 4 == 0 && aligned(g->d_table, 16), g->d_free, g->d_n_free, g->d_n_free_out, g->d_status, g->n_seqs,
               cache->n_pages, shift, g->shared_pages, (int*)g->d_ws, copies, rows, (uint32_t*)(rows + g->n_seqs)};
    const CacheArgs c = cache_args(cache, shift);
    hipStream_t s = (hipStream_t)stream;
    if (cache->n_pages <= FORK_LDS_PAGES)
        hipLaunchKernelGGL((batch_fork_kernel<true>), dim3(1), dim3(FORK_NT), (size_t)cache->n_pages * 4, s, a);
    else hipLaunchKernelGGL((batch_fork_kernel<false>), dim3(1), dim3(FORK_NT), 0, s, a);
    HIP_TRY(hipGetLastError());
    if (cache->dtype == DLLM_F32) launch_copies<uint32_t>(c, a, g->d_table_out, s);
    else launch_copies<uint16_t>(c, a, g->d_table_out, s);
    HIP_TRY(hipGetLastError());
    return DLLM_OK;
}

}  // extern "C"
