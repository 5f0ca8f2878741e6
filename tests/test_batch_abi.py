"""Refusals of the batch operators: every bad argument is turned down on the host, before any GPU work (no GPU here)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    try:
        pkg.lib()
    except ImportError:
        pytest.skip("libdllm.so not built")
    return pkg


P = 0x10000          # a 16-byte aligned address; nothing is read through it


PLAN = dict(d_len=P, d_new=P, d_owned=P, d_owned_out=2 * P, n_seqs=4, d_table=P, table_ld=8, d_free=P, d_n_free=P,
            d_n_free_out=2 * P, n_pages=64, page=32, shared_pages=0, max_rows=16, d_row0=P, d_pos=P, d_slot=P, d_seq=P,
            d_lim=P, d_status=P)


@pytest.mark.parametrize("change", [
    dict(d_len=None), dict(d_status=None), dict(d_slot=P + 2), dict(d_owned_out=P), dict(d_n_free_out=P),
    dict(n_seqs=0), dict(n_seqs=4097), dict(page=16), dict(page=48), dict(page=512), dict(n_pages=0),
    dict(n_pages=1 << 26), dict(table_ld=0), dict(table_ld=(1 << 18) + 1), dict(shared_pages=-1), dict(shared_pages=9),
    dict(max_rows=0), dict(max_rows=(1 << 24) + 1)])
def test_plan_refusals(dl, change):
    a = dict(PLAN, **change)
    assert dl.lib().dllm_batch_plan(*a.values(), None) == dl.DLLM_E_INVAL and dl.lib().dllm_last_error()


@pytest.mark.parametrize("args", [(None, 8, 64, 1e4), (P, 0, 64, 1e4), (P, 8, 63, 1e4), (P, 8, 0, 1e4), (P + 4, 8, 64, 1e4),
                                  (P, 1 << 30, 64, 1e4), (P, 8, 64, 1.0), (P, 8, 64, float("inf"))])
def test_rope_table_refusals(dl, args):
    assert dl.lib().dllm_rope_table(*args, None) == dl.DLLM_E_INVAL


def fill(cls, **values):
    a = cls()
    for k, v in values.items():
        setattr(a, k, v)
    return a


QK = dict(dtype=1, n_rows=4, n_heads=4, n_kv_heads=2, head_dim=64, page=32, n_pages=8, max_pos=16, eps=1e-6, d_q=P, d_k=P,
          d_v=P, ld_q=256, ld_k=128, ld_v=128, d_q_gain=P, d_k_gain=P, d_rope=P, d_pos=P, d_slot=P, d_q_out=2 * P,
          d_k_pages=P, d_v_pages=P)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -3), (dict(dtype=9), -3), (dict(head_dim=48), -3), (dict(head_dim=256), -3), (dict(n_rows=-1), -1),
    (dict(n_heads=3), -1), (dict(n_kv_heads=0), -1), (dict(n_heads=2048), -1), (dict(page=8), -1), (dict(n_pages=-1), -1),
    (dict(max_pos=0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(d_q=None), -1), (dict(d_rope=None), -1),
    (dict(d_k_pages=None), -1), (dict(d_k=P + 8), -1), (dict(ld_q=255), -1), (dict(ld_q=260), -1), (dict(ld_v=64), -1),
    (dict(d_v_pages=P + 2), -1), (dict(d_q_gain=P + 4), -1), (dict(d_pos=P + 1), -1), (dict(d_q_out=P, ld_q=512), -1)])
def test_qk_refusals(dl, change, code):
    a = fill(dl.dllm_qk_args, **dict(QK, **change))
    assert dl.lib().dllm_qk_norm_rope(ctypes.byref(a), None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_qk_norm_rope(None, None) == dl.DLLM_E_INVAL


ATTN = dict(dtype=4, n_rows=4, n_seqs=2, n_heads=4, n_kv_heads=2, head_dim=64, page=32, n_pages=8, table_ld=4, shared_len=32,
            max_rows=2, max_len=100, scale=0.1, d_q=P, ld_q=256, d_k_pages=P, d_v_pages=P, d_table=P, d_row0=P, d_len=P,
            d_lim=None, d_out=P, ld_out=256, d_ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), -3), (dict(head_dim=96), -3), (dict(head_dim=32, ld_q=128, ld_out=128), -3), (dict(n_rows=-2), -1),
    (dict(n_seqs=0), -1), (dict(n_seqs=5000), -1), (dict(n_kv_heads=3), -1), (dict(page=33), -1), (dict(n_pages=0), -1),
    (dict(table_ld=0), -1), (dict(table_ld=1 << 27), -1), (dict(max_len=-1), -1), (dict(max_len=129), -1),
    (dict(max_rows=-1), -1), (dict(shared_len=33), -1), (dict(shared_len=-32), -1), (dict(shared_len=160), -1),
    (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(d_q=None), -1), (dict(d_table=None), -1),
    (dict(d_out=None), -1), (dict(ld_q=248), -1), (dict(ld_out=258), -1), (dict(d_q=P + 2), -1), (dict(d_lim=P + 2), -1),
    (dict(d_v_pages=P + 4), -1)])
def test_attention_refusals(dl, change, code):
    a = fill(dl.dllm_attn_args, **dict(ATTN, **change))
    assert dl.lib().dllm_attention_paged(ctypes.byref(a), None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_attention_paged(None, None) == dl.DLLM_E_INVAL
    n = ctypes.c_size_t()
    assert dl.lib().dllm_attention_paged_ws(None, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert dl.lib().dllm_attention_paged_ws(ctypes.byref(a), None) == dl.DLLM_E_INVAL


SELECT = dict(dtype=0, n_rows=4, vocab=100, mask_id=99, n_seqs=2, d_logits=P, ld=100, d_row0=P, d_hist=P, d_hist0=P,
              d_n_prompt=P, d_repetition=P, d_presence=P, d_frequency=P, d_bias_id=P, d_bias=P, d_bias0=P, d_allow=P,
              n_allow=2, allow_ld=4, d_allow_row=P, d_out_logits=None, ld_out=0, d_out_id=P, d_out_conf=P, d_ws=P,
              ws_bytes=1 << 40)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -3), (dict(n_rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=(1 << 24) + 1), -1), (dict(mask_id=-2), -1),
    (dict(mask_id=100), -1), (dict(n_seqs=0), -1), (dict(n_seqs=4097), -1), (dict(d_logits=None), -1), (dict(d_out_id=None), -1),
    (dict(d_out_conf=None), -1), (dict(d_row0=None), -1), (dict(d_hist0=None), -1), (dict(d_hist=None), -1),
    (dict(d_bias=None), -1), (dict(d_bias0=None), -1), (dict(n_allow=0), -1), (dict(allow_ld=3), -1),
    (dict(d_allow_row=None), -1), (dict(d_allow=None), -1), (dict(ld=99), -1), (dict(d_logits=P + 2), -1),
    (dict(d_out_logits=P, ld_out=104), -1), (dict(d_out_logits=2 * P, ld_out=99), -1), (dict(d_out_logits=P + 1, ld_out=100), -1),
    (dict(d_hist=P + 2), -1), (dict(d_out_conf=P + 1), -1)])
def test_select_refusals(dl, change, code):
    a = fill(dl.dllm_select_args, **dict(SELECT, **change))
    assert dl.lib().dllm_select(ctypes.byref(a), None) == code and dl.lib().dllm_last_error()
    assert dl.lib().dllm_select(None, None) == dl.DLLM_E_INVAL
    n = ctypes.c_size_t()
    assert dl.lib().dllm_select_ws(None, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert dl.lib().dllm_select_ws(ctypes.byref(a), None) == dl.DLLM_E_INVAL


def test_workspace_is_checked(dl):
    L, n = dl.lib(), ctypes.c_size_t()
    a = fill(dl.dllm_attn_args, **dict(ATTN, table_ld=200, max_len=6000, n_pages=4000, shared_len=0, d_ws=None, ws_bytes=0))
    assert L.dllm_attention_paged_ws(ctypes.byref(a), ctypes.byref(n)) == 0 and n.value > 0
    assert L.dllm_attention_paged(ctypes.byref(a), None) == dl.DLLM_E_INVAL             # NULL
    a.d_ws, a.ws_bytes = P, n.value - 1
    assert L.dllm_attention_paged(ctypes.byref(a), None) == dl.DLLM_E_CAPACITY
    a.d_ws, a.ws_bytes = P + 8, n.value
    assert L.dllm_attention_paged(ctypes.byref(a), None) == dl.DLLM_E_INVAL             # misaligned
    s = fill(dl.dllm_select_args, **dict(SELECT, vocab=5000, mask_id=-1, ld=5000, allow_ld=200, d_ws=None, ws_bytes=0))
    assert L.dllm_select_ws(ctypes.byref(s), ctypes.byref(n)) == 0 and n.value > 0
    assert L.dllm_select(ctypes.byref(s), None) == dl.DLLM_E_INVAL
    s.d_ws, s.ws_bytes = P, n.value - 1
    assert L.dllm_select(ctypes.byref(s), None) == dl.DLLM_E_CAPACITY


@pytest.mark.parametrize("change", [dict(n_rows=1 << 24, n_heads=1024, n_kv_heads=1, ld_q=1 << 16, ld_out=1 << 16),
                                    dict(n_seqs=4096, max_rows=1 << 24, n_rows=1 << 24, n_heads=32, n_kv_heads=32, ld_q=2048, ld_out=2048),
                                    dict(table_ld=1 << 25, max_len=(1 << 30) + 1), dict(n_rows=1 << 24, max_rows=1, n_heads=512, n_kv_heads=64, ld_q=1 << 16, ld_out=1 << 16)])
def test_attention_refuses_launches_past_the_grid(dl, change):
    a, n = fill(dl.dllm_attn_args, **dict(ATTN, **change)), ctypes.c_size_t()
    assert dl.lib().dllm_attention_paged_ws(ctypes.byref(a), ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert dl.lib().dllm_attention_paged(ctypes.byref(a), None) == dl.DLLM_E_INVAL


def test_qk_refuses_launches_past_the_grid(dl):
    wide = dict(n_rows=1 << 24, n_heads=1024, n_kv_heads=1024, ld_q=1 << 16, ld_k=1 << 16, ld_v=1 << 16)
    assert dl.lib().dllm_qk_norm_rope(ctypes.byref(fill(dl.dllm_qk_args, **dict(QK, **wide))), None) == dl.DLLM_E_INVAL


def test_binding_refuses_tensors_that_are_not_on_the_gpu(dl):
    import torch
    z = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(dl.DllmError):
        dl.dllm_batch_plan(z(2), z(2), z(2), z(2), z(8).view(2, 4), z(9), z(1), z(1), 32, 0, z(3), z(5), z(5), z(5), z(5), z(3))
    with pytest.raises(dl.DllmError):
        dl.dllm_select(torch.zeros(2, 9), z(2), torch.zeros(2))


def test_packed_arguments_are_the_structs_bytes(dl):
    for cls, pack in ((dl.dllm_qk_args, dl._pack_qk), (dl.dllm_attn_args, dl._pack_attn), (dl.dllm_select_args, dl._pack_select)):
        v = [i + 0.5 if t is ctypes.c_float else i + 1 for i, (_, t) in enumerate(cls._fields_)]
        assert pack(*v) == bytes(cls(*v))


def test_argument_structs_have_the_headers_layout(dl, tmp_path):
    """The binding's structs against the header's, field by field, through the host compiler."""
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines, want = [], []
    for name in ("dllm_qk_args", "dllm_attn_args", "dllm_select_args", "dllm_batch_rows"):
        cls = getattr(dl, name)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "dllm.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call([cc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")])
    assert [int(x) for x in subprocess.check_output([str(tmp_path / "layout")]).split()] == want


def test_batch_step_refuses_null(dl):
    L = dl.lib()
    n = ctypes.c_size_t()
    rows = dl.dllm_batch_rows()
    ptrs = (ctypes.c_void_p * 1)(P)
    assert L.dllm_batch_bytes(None, 8, 32, ctypes.byref(n)) == dl.DLLM_E_INVAL
    assert L.dllm_batch_step(None, P, 1 << 40, ctypes.byref(rows), P, None, None, None, None, None) == dl.DLLM_E_INVAL
    assert L.dllm_model_set_qk_norm(None, ptrs, ptrs, None) == dl.DLLM_E_INVAL
