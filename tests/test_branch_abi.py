"""Refusals of the branching operators on the host, and the launch rules of their kernels (no GPU here)."""
import ctypes

import pytest

from test_batch_abi import ATTN, P, dl, fill  # noqa: F401
from test_batch_rules import run_cpp

TREE = dict(d_parent=P, d_row0=P, d_len=P, n_rows=8, n_seqs=2, d_pos=2 * P, d_mask=P, mask_ld=1)


@pytest.mark.parametrize("change", [dict(d_parent=None), dict(d_mask=None), dict(d_pos=P + 2), dict(d_pos=P), dict(n_rows=-1),
                                    dict(n_rows=(1 << 24) + 1), dict(n_seqs=0), dict(n_seqs=4097), dict(mask_ld=0), dict(mask_ld=33)])
def test_tree_plan_refusals(dl, change):  # noqa: F811
    a = dict(TREE, **change)
    assert dl.lib().dllm_tree_plan(*a.values(), None) == dl.DLLM_E_INVAL and dl.lib().dllm_last_error()


@pytest.mark.parametrize("change,mask,ld,code", [
    ({}, None, 1, -1), ({}, P + 2, 1, -1), ({}, P, 0, -1), ({}, P, (1 << 24) + 1, -1), (dict(dtype=3), P, 1, -3),
    (dict(head_dim=96), P, 1, -3), (dict(d_q=None), P, 1, -1), (dict(max_len=129), P, 1, -1), (dict(ld_out=258), P, 1, -1)])
def test_attention_tree_refusals(dl, change, mask, ld, code):  # noqa: F811
    a = fill(dl.dllm_attn_args, **dict(ATTN, **change))
    assert dl.lib().dllm_attention_tree(ctypes.byref(a), mask, ld, None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_attention_tree(None, P, 1, None) == dl.DLLM_E_INVAL
    n = ctypes.c_size_t()
    assert dl.lib().dllm_attention_tree_ws(None, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert dl.lib().dllm_attention_tree_ws(ctypes.byref(a), None) == dl.DLLM_E_INVAL


def test_batch_step_tree_refusals(dl):  # noqa: F811
    for tree, ld in ((None, 1), (P + 1, 1), (P, 0), (P, 1)):           # (the last: no model)
        assert dl.lib().dllm_batch_step_tree(None, P, 1 << 20, None, tree, ld, P, None, None, None, None, None) == dl.DLLM_E_INVAL


LOGP = dict(dtype=0, n_rows=4, vocab=5000, mask_id=99, n_tok=3, top=2, d_logits=P, ld=5000, d_tok=P, d_tok_row=P, d_logp=P,
            d_entropy=P, d_top_id=P, d_top_logp=P, d_ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -3), (dict(n_rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=(1 << 24) + 1), -1), (dict(mask_id=-2), -1),
    (dict(mask_id=5000), -1), (dict(top=-1), -1), (dict(top=65), -1), (dict(n_tok=-1), -1), (dict(n_tok=(1 << 24) + 1), -1),
    (dict(d_logits=None), -1), (dict(d_tok=None), -1), (dict(d_logp=None), -1), (dict(d_tok_row=None, n_tok=5), -1),
    (dict(d_top_id=None), -1), (dict(d_top_logp=None), -1), (dict(ld=4999), -1), (dict(d_logits=P + 2), -1), (dict(d_tok=P + 1), -1),
    (dict(d_entropy=P + 2), -1), (dict(n_rows=0), -1)])
def test_logprobs_refusals(dl, change, code):  # noqa: F811
    a = fill(dl.dllm_logprobs_args, **dict(LOGP, **change))
    assert dl.lib().dllm_logprobs(ctypes.byref(a), None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_logprobs(None, None) == dl.DLLM_E_INVAL


def test_workspaces_are_checked(dl):  # noqa: F811
    L, n = dl.lib(), ctypes.c_size_t()
    assert L.dllm_logprobs_ws(None, ctypes.byref(n)) == dl.DLLM_E_INVAL
    a = fill(dl.dllm_logprobs_args, **dict(LOGP, vocab=50000, ld=50000, d_ws=None, ws_bytes=0))
    assert L.dllm_logprobs_ws(ctypes.byref(a), None) == dl.DLLM_E_INVAL
    assert L.dllm_logprobs_ws(ctypes.byref(a), ctypes.byref(n)) == 0 and n.value > 0
    assert L.dllm_logprobs(ctypes.byref(a), None) == dl.DLLM_E_INVAL
    a.d_ws, a.ws_bytes = P, n.value - 1
    assert L.dllm_logprobs(ctypes.byref(a), None) == dl.DLLM_E_CAPACITY
    a.d_ws, a.ws_bytes = P + 8, n.value
    assert L.dllm_logprobs(ctypes.byref(a), None) == dl.DLLM_E_INVAL
    assert L.dllm_batch_fork_ws(0, 8, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert L.dllm_batch_fork_ws(4, 0, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert L.dllm_batch_fork_ws(4, 8, None) == dl.DLLM_E_INVAL
    assert L.dllm_batch_fork_ws(FORK["n_seqs"], CACHE["n_pages"], ctypes.byref(n)) == 0 and n.value > 0
    c, f = fill(dl.dllm_cache, **CACHE), fill(dl.dllm_fork_args, **dict(FORK, ws_bytes=n.value - 1))
    assert L.dllm_batch_fork(ctypes.byref(c), ctypes.byref(f), None) == dl.DLLM_E_CAPACITY


CACHE = dict(dtype=4, n_layers=2, n_kv_heads=2, head_dim=64, page=32, n_pages=8, d_pages=P)
BAD_CACHE = [(dict(dtype=2), -3), (dict(n_layers=0), -1), (dict(n_layers=4097), -1), (dict(n_kv_heads=0), -1), (dict(n_kv_heads=1025), -1),
             (dict(head_dim=48), -3), (dict(page=16), -1), (dict(n_pages=0), -1), (dict(n_pages=1 << 26), -1), (dict(d_pages=None), -1),
             (dict(d_pages=P + 8), -1)]
COMPACT = dict(d_table=P, table_ld=4, d_base=P, d_path=P, path_ld=8, d_n=P, n_seqs=3)


@pytest.mark.parametrize("change,code", BAD_CACHE)
def test_cache_refusals(dl, change, code):  # noqa: F811
    c, f = fill(dl.dllm_cache, **dict(CACHE, **change)), fill(dl.dllm_fork_args, **FORK)
    assert dl.lib().dllm_cache_compact(ctypes.byref(c), *COMPACT.values(), None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_batch_fork(ctypes.byref(c), ctypes.byref(f), None) == code


@pytest.mark.parametrize("change", [dict(d_table=None), dict(d_n=None), dict(d_base=P + 2), dict(table_ld=0), dict(table_ld=(1 << 18) + 1),
                                    dict(path_ld=0), dict(path_ld=1025), dict(n_seqs=0), dict(n_seqs=4097)])
def test_compact_refusals(dl, change):  # noqa: F811
    c, a = fill(dl.dllm_cache, **CACHE), dict(COMPACT, **change)
    assert dl.lib().dllm_cache_compact(ctypes.byref(c), *a.values(), None) == dl.DLLM_E_INVAL
    assert dl.lib().dllm_cache_compact(None, *COMPACT.values(), None) == dl.DLLM_E_INVAL


FORK = dict(n_seqs=3, table_ld=4, shared_pages=1, d_src=P, d_keep=P, d_owned=P, d_owned_out=2 * P, d_table=P, d_table_out=2 * P,
            d_free=P, d_n_free=P, d_n_free_out=2 * P, d_status=P, d_ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("change", [
    dict(n_seqs=0), dict(n_seqs=4097), dict(table_ld=0), dict(table_ld=(1 << 18) + 1), dict(shared_pages=-1), dict(shared_pages=5),
    dict(d_src=None), dict(d_status=None), dict(d_keep=P + 2), dict(d_owned_out=P), dict(d_table_out=P), dict(d_n_free_out=P),
    dict(d_ws=None), dict(d_ws=P + 8)])
def test_fork_refusals(dl, change):  # noqa: F811
    c, f = fill(dl.dllm_cache, **CACHE), fill(dl.dllm_fork_args, **dict(FORK, **change))
    assert dl.lib().dllm_batch_fork(ctypes.byref(c), ctypes.byref(f), None) == dl.DLLM_E_INVAL and dl.lib().dllm_last_error()
    assert dl.lib().dllm_batch_fork(ctypes.byref(c), None, None) == dl.DLLM_E_INVAL


def test_rules_of_the_branching_operators(tmp_path):
    """Parts of a row: every block in exactly one, none empty, whole rounds of a workgroup's waves; LDS within a CU's 160 KB."""
    out = run_cpp(tmp_path, r"""
int main() {
    long n = 0;
    for (int T : {0, 1, 2, 7, 32, 256, 1024, 1025, 4096, 1 << 24})
        for (int V : {1, 2, 2047, 2048, 2049, 8192, 8193, 126464, 152064, 1 << 24}) {
            const int blocks = (V + LP_BLOCK - 1) / LP_BLOCK, per = lp_per(T, V), parts = lp_parts(T, V);
            if (per < 1 || per % (LP_NT / 64) || (long)parts * per < blocks || (long)(parts - 1) * per >= blocks) return 1;
            if (T >= 4 * N_CU && parts != 1) return 2;
            if (lp_ws_bytes(T, V, 64) != (parts == 1 ? 0 : (size_t)T * parts * 4 * 528)) return 3;
            ++n;
        }
    if ((size_t)FORK_LDS_PAGES * 4 + 3 * 4 * DLLM_MAX_SEQS + 1024 > 160 * 1024) return 5;
    if (fork_ws_bytes(3, FORK_LDS_PAGES) != 88 || fork_ws_bytes(3, FORK_LDS_PAGES + 1) != 88 + 4 * (FORK_LDS_PAGES + 1)) return 6;
    std::printf("%ld", n);
}
""")
    assert out == "100"


def test_rules_of_the_attention_with_masks(tmp_path):
    """Groups of tiles for every sequence, head and split, the same number for each XCD; splits that cover the keys, none
    empty; the paged attention's launches as they were."""
    out = run_cpp(tmp_path, r"""
int main() {
    long n = 0;
    for (int dtype : {DLLM_F32, DLLM_F16})
        for (int B : {1, 3, 16, 256, 300, 4096})
            for (int rows : {1, 5, 64, 1000})
                for (int share : {0, 1024, 8192})
                    for (int own : {0, 1, 900, 30000}) {
                        dllm_attn_args g{};
                        g.dtype = dtype; g.n_seqs = B; g.max_rows = rows; g.n_rows = (int)((long)B * rows * 2 / 3 + 1);
                        g.n_heads = 28; g.n_kv_heads = 4; g.head_dim = 128; g.page = 64; g.shared_len = share; g.max_len = share + own;
                        const AttnPlan p = attn_plan(&g, true), q = attn_plan(&g);
                        const int step = dtype == DLLM_F32 ? 32 : 64, steps = own + (share - p.shared);
                        if (p.wgs_o % (8 * p.nt_o) || p.wgs_o < (long)B * 4 * p.ns_o * p.nt_o || p.wgs_o >= (long)(B * 4 * p.ns_o + 8) * p.nt_o) return 1;
                        if (p.nt_o * 16l * p.qg * p.qt < (long)(rows < g.n_rows ? rows : g.n_rows) * 7) return 2;
                        if (p.ns_o < 1 || p.ns_o > MAX_ATTN_SPLITS || p.ns_s > MAX_ATTN_SPLITS || (p.shared > 0) != (p.ns_s > 0)) return 3;
                        if (steps > 0 && (p.ns_o - 1) * (long)ceil_div(ceil_div(steps, step), p.ns_o) >= ceil_div(steps, step)) return 4;
                        if (p.shared != q.shared || q.wgs_o != (long)B * 4 * q.nt_o * q.ns_o || p.wgs_s != (p.shared ? 4l * p.nt_s * p.ns_s : 0)) return 5;
                        ++n;
                    }
    std::printf("%ld", n);
}
""")
    assert out == "576"


def test_work_of_the_given_tokens_is_bounded(dl, tmp_path):  # noqa: F811
    """No launch in which every row looks through a long list: at most 1024 tokens a row and 2^20 in all; longer lists get a
    launch of their own and the rows' sums 8 bytes each in the workspace.  Without a list of rows a token is its row's."""
    out = run_cpp(tmp_path, r"""
int main() {
    long n = 0;
    for (int T : {0, 1, 5, 256, 1024, 1025, 2048, 16384, 1 << 20, 1 << 24})
        for (int k : {0, 1, 64, 512, 1024, 1025, 4096, 1 << 20, 1 << 24}) {
            if (lp_tokens_apart(T, k, false)) return 1;
            if (!lp_tokens_apart(T, k, true) && (k > 1024 || (long)T * k > 1l << 20)) return 2;
            n += lp_tokens_apart(T, k, true);
        }
    if (lp_tokens_apart(256, 512, true) || !lp_tokens_apart(16384, 256, true)) return 3;
    std::printf("%ld", n);
}
""")
    assert int(out) > 0
    L, n = dl.lib(), ctypes.c_size_t()
    size = lambda **kw: L.dllm_logprobs_ws(ctypes.byref(fill(dl.dllm_logprobs_args, **dict(LOGP, **kw))), ctypes.byref(n)) or n.value  # noqa: E731
    few, many = dict(n_rows=3000, n_tok=300), dict(n_rows=3000, n_tok=3000)
    assert size(**few) == 0 and size(**many, d_tok_row=None) == 0 and size(**many) == 3000 * 8
    assert size(vocab=50000, ld=50000, n_tok=2000) == size(vocab=50000, ld=50000) + 4 * 8
    a = fill(dl.dllm_logprobs_args, **dict(LOGP, **many, ws_bytes=3000 * 8 - 1))
    assert L.dllm_logprobs(ctypes.byref(a), None) == dl.DLLM_E_CAPACITY
    a.d_ws = None
    assert L.dllm_logprobs(ctypes.byref(a), None) == dl.DLLM_E_INVAL


def test_sizes_of_the_gpu_tests_reach_their_launches(tmp_path):
    """test_gpu_branch_sizes.py: several blocks a wave with several parts a row and with one; two, three and eight heads of V^T a
    workgroup, the last one with fewer; the measured compaction's two."""
    out = run_cpp(tmp_path, r"""
int main() {
    if (lp_per(256, 70001) <= 4 || lp_parts(256, 70001) <= 1 || lp_per(300, 152064) <= 4 || lp_parts(300, 152064) <= 1) return 1;
    if (lp_parts(1100, 70001) != 1 || lp_per(1100, 70001) < 35) return 2;
    if (compact_heads_per(64, 7, 7) != 2 || compact_heads_per(60, 4, 13) != 2 || compact_heads_per(34, 13, 7) != 2) return 3;
    if (compact_heads_per(96, 7, 7) != 3 || compact_heads_per(96, 11, 12) != 8 || compact_heads_per(100, 11, 13) != 8) return 4;
    if (49 % 2 != 1 || 49 % 3 != 1 || 132 % 8 != 4 || 143 % 8 != 7 || compact_heads_per(32, 28, 4) != 2) return 5;
    std::printf("ok");
}
""")
    assert out == "ok"
