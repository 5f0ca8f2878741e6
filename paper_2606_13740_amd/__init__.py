"""Python binding of libdllm, the gfx950 denoising-step library.

Argument marshalling only: every function below forwards to the C ABI entry
point of the same name (see include/dllm.h) and every step runs in the HIP
kernels of ``csrc/``.  PyTorch supplies device memory and the stream.  There is
no fallback: if ``libdllm.so`` has not been built, importing the library fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdllm.so")

DLLM_OK, DLLM_E_INVAL, DLLM_E_CAPACITY, DLLM_E_DTYPE, DLLM_E_HIP, DLLM_E_UNIMPL, DLLM_E_NOMEM = 0, -1, -2, -3, -4, -5, -6
DLLM_F32, DLLM_BF16, DLLM_W8, DLLM_Q4 = 0, 1, 2, 3
DLLM_F16 = 4                      # element type of the batch operators
DLLM_MAX_SEQS = 4096
DLLM_MAX_TOP, DLLM_MAX_TREE = 64, 1024
K_QKV, K_ATTN, K_OPROJ, K_GATEUP, K_DOWN, K_LMHEAD = range(6)
KERNEL_CLASSES = {"qkv": K_QKV, "attn": K_ATTN, "oproj": K_OPROJ, "gateup": K_GATEUP, "down": K_DOWN,
                  "lmhead": K_LMHEAD}


class DllmError(RuntimeError):
    def __init__(self, code: int, func: str, msg: str):
        super().__init__(f"{func} failed with {code}: {msg}")
        self.code = code


class dllm_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("mask_id", ctypes.c_int32), ("block", ctypes.c_int32), ("eps", ctypes.c_float),
                ("rope_base", ctypes.c_float), ("dtype", ctypes.c_int32), ("max_window", ctypes.c_int32),
                ("max_pos", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("qkv_bias", ctypes.c_int32)]


class dllm_layer_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "attn_norm", "ffn_norm",
                                               "bq", "bk", "bv")]


class dllm_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("layers", ctypes.POINTER(dllm_layer_weights))]


_lib = None
_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_i64, _f32 = ctypes.c_int64, ctypes.c_float


def _fields(ctype, names):
    return [(n, ctype) for n in names.split()]


class dllm_qk_args(ctypes.Structure):
    _fields_ = (_fields(_i32, "dtype n_rows n_heads n_kv_heads head_dim page n_pages max_pos") + [("eps", _f32)] +
                _fields(_vp, "d_q d_k d_v") + _fields(_i64, "ld_q ld_k ld_v") +
                _fields(_vp, "d_q_gain d_k_gain d_rope d_pos d_slot d_q_out d_k_pages d_v_pages"))


class dllm_attn_args(ctypes.Structure):
    _fields_ = (_fields(_i32, "dtype n_rows n_seqs n_heads n_kv_heads head_dim page n_pages table_ld shared_len "
                              "max_rows max_len") +
                [("scale", _f32), ("d_q", _vp), ("ld_q", _i64)] +
                _fields(_vp, "d_k_pages d_v_pages d_table d_row0 d_len d_lim d_out") +
                [("ld_out", _i64), ("d_ws", _vp), ("ws_bytes", _sz)])


class dllm_batch_rows(ctypes.Structure):
    _fields_ = (_fields(_i32, "n_rows n_seqs page n_pages table_ld shared_len max_rows max_len") +
                _fields(_vp, "d_table d_row0 d_pos d_slot d_len d_lim"))


class dllm_select_args(ctypes.Structure):
    _fields_ = (_fields(_i32, "dtype n_rows vocab mask_id n_seqs") + [("d_logits", _vp), ("ld", _i64)] +
                _fields(_vp, "d_row0 d_hist d_hist0 d_n_prompt d_repetition d_presence d_frequency d_bias_id d_bias "
                             "d_bias0 d_allow") +
                _fields(_i32, "n_allow allow_ld") + _fields(_vp, "d_allow_row d_out_logits") + [("ld_out", _i64)] +
                _fields(_vp, "d_out_id d_out_conf d_ws") + [("ws_bytes", _sz)])


class dllm_logprobs_args(ctypes.Structure):
    _fields_ = (_fields(_i32, "dtype n_rows vocab mask_id n_tok top") + [("d_logits", _vp), ("ld", _i64)] +
                _fields(_vp, "d_tok d_tok_row d_logp d_entropy d_top_id d_top_logp d_ws") + [("ws_bytes", _sz)])


class dllm_cache(ctypes.Structure):
    _fields_ = _fields(_i32, "dtype n_layers n_kv_heads head_dim page n_pages") + [("d_pages", _vp)]


class dllm_fork_args(ctypes.Structure):
    _fields_ = (_fields(_i32, "n_seqs table_ld shared_pages") +
                _fields(_vp, "d_src d_keep d_owned d_owned_out d_table d_table_out d_free d_n_free d_n_free_out d_status d_ws") +
                [("ws_bytes", _sz)])


def _packer(cls):
    """Packs values, in the order of the fields, into the bytes of a struct: a quarter of its constructor's time."""
    fmt = "@" + "".join({_i32: "i", _f32: "f", _i64: "q", _vp: "P", _sz: "N"}[t] for _, t in cls._fields_)
    return struct.Struct(fmt + "x" * (ctypes.sizeof(cls) - struct.calcsize(fmt))).pack


_pack_qk, _pack_attn, _pack_select = _packer(dllm_qk_args), _packer(dllm_attn_args), _packer(dllm_select_args)
_pack_rows = _packer(dllm_batch_rows)
_pack_logprobs, _pack_cache, _pack_fork = _packer(dllm_logprobs_args), _packer(dllm_cache), _packer(dllm_fork_args)
_pack_ws = struct.Struct("@PN").pack          # the last two fields of every struct with a workspace
_pack_2i = struct.Struct("@2i").pack

# (the batch operators' args are pointers to their structs: a struct by reference, or its bytes)
_SIGNATURES = {
    "dllm_last_error": ([], ctypes.c_char_p),
    "dllm_version": ([], ctypes.c_char_p),
    "dllm_model_create": ([ctypes.POINTER(dllm_config), ctypes.POINTER(dllm_weights), _vp, ctypes.POINTER(_vp)],
                          ctypes.c_int),
    "dllm_model_destroy": ([_vp], ctypes.c_int),
    "dllm_kv_bytes": ([_vp, _i32, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_kv_create": ([_vp, _vp, _sz, _i32, ctypes.POINTER(_vp)], ctypes.c_int),
    "dllm_kv_destroy": ([_vp], ctypes.c_int),
    "dllm_kv_prefix_len": ([_vp, ctypes.POINTER(_i32), ctypes.POINTER(_i32)], ctypes.c_int),
    "dllm_kv_set_prefix_len": ([_vp, _i32], ctypes.c_int),
    "dllm_prefill": ([_vp, _vp, _vp, _i32, _vp], ctypes.c_int),
    "dllm_denoise_step": ([_vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_commit": ([_vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_append_prefix_kv": ([_vp, _vp, _vp, _i32, _vp], ctypes.c_int),
    "dllm_refresh_kv": ([_vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_denoise_step_noalloc": ([_vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_denoise_window": ([_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_denoise_window_sls": ([_vp, _vp, _i32, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_accept_drafts": ([_vp, _vp, _vp, _vp, _vp, _i32, ctypes.c_float, _vp, _vp, _vp], ctypes.c_int),
    "dllm_record_drafts": ([_vp, _vp, _vp, _i32, _vp], ctypes.c_int),
    "dllm_step_merged": ([_vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp],
                         ctypes.c_int),
    "dllm_debug_logits": ([_vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp], ctypes.c_int),
    "dllm_debug_hidden": ([_vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp], ctypes.c_int),
    "dllm_probe_enable": ([_vp, _i32, _i32], ctypes.c_int),
    "dllm_probe_read": ([_vp, ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_double)], ctypes.c_int),
    "dllm_kernel_bytes": ([_vp, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_double)], ctypes.c_int),
    "dllm_kernel_replay": ([_vp, _vp, _i32, _i32, _i32, _vp], ctypes.c_int),
    "dllm_read_bandwidth": ([_vp, ctypes.c_size_t, _vp, _vp], ctypes.c_int),
    "dllm_quantize_q4_0": ([_vp, _i32, _i32, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_quantize_int8": ([_vp, _i32, _i32, _i32, _vp, _vp, _vp], ctypes.c_int),
    "dllm_batch_plan": ([_vp] * 4 + [_i32, _vp, _i32] + [_vp] * 3 + [_i32] * 4 + [_vp] * 7, ctypes.c_int),
    "dllm_rope_table": ([_vp, _i32, _i32, _f32, _vp], ctypes.c_int),
    "dllm_qk_norm_rope": ([_vp, _vp], ctypes.c_int),
    "dllm_attention_paged_ws": ([_vp, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_attention_paged": ([_vp, _vp], ctypes.c_int),
    "dllm_select_ws": ([_vp, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_select": ([_vp, _vp], ctypes.c_int),
    "dllm_model_set_qk_norm": ([_vp, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp], ctypes.c_int),
    "dllm_batch_bytes": ([_vp, _i32, _i32, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_batch_step": ([_vp, _vp, _sz, _vp, _vp, _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "dllm_tree_plan": ([_vp, _vp, _vp, _i32, _i32, _vp, _vp, _i32, _vp], ctypes.c_int),
    "dllm_attention_tree_ws": ([_vp, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_attention_tree": ([_vp, _vp, _i32, _vp], ctypes.c_int),
    "dllm_batch_step_tree": ([_vp, _vp, _sz, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "dllm_logprobs_ws": ([_vp, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_logprobs": ([_vp, _vp], ctypes.c_int),
    "dllm_cache_compact": ([_vp, _vp, _i32, _vp, _vp, _i32, _vp, _i32, _vp], ctypes.c_int),
    "dllm_batch_fork_ws": ([_i32, _i32, ctypes.POINTER(_sz)], ctypes.c_int),
    "dllm_batch_fork": ([_vp, _vp, _vp], ctypes.c_int),
    "dllm_commit_staged": ([_vp, _vp, _vp, _vp, _vp, _i32, _i32, ctypes.c_float, ctypes.c_float, _vp, _vp, _vp],
                           ctypes.c_int),
}


def lib():
    """The loaded libdllm.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGNATURES.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def _check(rc: int, func: str):
    if rc != DLLM_OK:
        raise DllmError(rc, func, lib().dllm_last_error().decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


_raw_stream = None


def _current_device() -> int:
    import torch
    return torch.cuda.current_device()


def _stream(stream, device: Optional[int] = None):
    """The stream's handle; None: the current stream of the current device (`device`, where the caller knows it)."""
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            # the handle without the Stream object around it (2.7 us a call), where torch has it
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
                lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        return _raw_stream(_current_device() if device is None else device)
    return stream if isinstance(stream, int) else stream.cuda_stream


# ----------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# ----------------------------------------------------------------------------


_gain_sizes = {}          # of a model's handle: (layers, head_dim), what dllm_model_set_qk_norm reads


def dllm_model_create(cfg: dllm_config, weights: dllm_weights, stream=None) -> int:
    h = _vp()
    _check(lib().dllm_model_create(ctypes.byref(cfg), ctypes.byref(weights), _stream(stream), ctypes.byref(h)),
           "dllm_model_create")
    _gain_sizes[h.value] = (cfg.n_layers, cfg.head_dim)
    return h.value


def dllm_model_destroy(model: int):
    _gain_sizes.pop(model, None)
    _check(lib().dllm_model_destroy(model), "dllm_model_destroy")


def dllm_kv_bytes(model: int, capacity: int) -> int:
    n = _sz()
    _check(lib().dllm_kv_bytes(model, capacity, ctypes.byref(n)), "dllm_kv_bytes")
    return n.value


def dllm_kv_create(model: int, buf, nbytes: int, capacity: int) -> int:
    h = _vp()
    _check(lib().dllm_kv_create(model, _ptr(buf), nbytes, capacity, ctypes.byref(h)), "dllm_kv_create")
    return h.value


def dllm_kv_destroy(kv: int):
    _check(lib().dllm_kv_destroy(kv), "dllm_kv_destroy")


def dllm_kv_prefix_len(kv: int):
    p, q = _i32(), _i32()
    _check(lib().dllm_kv_prefix_len(kv, ctypes.byref(p), ctypes.byref(q)), "dllm_kv_prefix_len")
    return p.value, q.value


def dllm_kv_set_prefix_len(kv: int, n: int):
    _check(lib().dllm_kv_set_prefix_len(kv, n), "dllm_kv_set_prefix_len")


def dllm_prefill(model: int, kv: int, ids, n: int, stream=None):
    _check(lib().dllm_prefill(model, kv, _ptr(ids), n, _stream(stream)), "dllm_prefill")


def dllm_denoise_step(model: int, kv: int, tok, mask, W: int, out_id, out_conf, stream=None):
    _check(lib().dllm_denoise_step(model, kv, _ptr(tok), _ptr(mask), W, _ptr(out_id), _ptr(out_conf),
                                   _stream(stream)), "dllm_denoise_step")


def dllm_denoise_step_noalloc(model: int, kv: int, tok, mask, W: int, out_id, out_conf, stream=None):
    _check(lib().dllm_denoise_step_noalloc(model, kv, _ptr(tok), _ptr(mask), W, _ptr(out_id), _ptr(out_conf),
                                           _stream(stream)), "dllm_denoise_step_noalloc")


def dllm_commit(conf, ids, tok, mask, seg_begin: int, seg_len: int, k: int, committed_pos=None,
                n_committed=None, stream=None):
    _check(lib().dllm_commit(_ptr(conf), _ptr(ids), _ptr(tok), _ptr(mask), seg_begin, seg_len, k,
                             _ptr(committed_pos), _ptr(n_committed), _stream(stream)), "dllm_commit")


def dllm_append_prefix_kv(model: int, kv: int, block_tok, n: int, stream=None):
    _check(lib().dllm_append_prefix_kv(model, kv, _ptr(block_tok), n, _stream(stream)), "dllm_append_prefix_kv")


def dllm_refresh_kv(model: int, kv: int, pos, new_ids, n: int, out_id=None, out_conf=None, stream=None):
    _check(lib().dllm_refresh_kv(model, kv, _ptr(pos), _ptr(new_ids), n, _ptr(out_id), _ptr(out_conf),
                                 _stream(stream)), "dllm_refresh_kv")


def dllm_denoise_window(model: int, kv: int, w0: int, tok, mask, W: int, out_id, out_conf, stream=None):
    _check(lib().dllm_denoise_window(model, kv, w0, _ptr(tok), _ptr(mask), W, _ptr(out_id), _ptr(out_conf),
                                     _stream(stream)), "dllm_denoise_window")


def dllm_denoise_window_sls(model: int, kv: int, w0: int, tok, mask, need, n_need: int, W: int, out_id, out_conf,
                            stream=None):
    _check(lib().dllm_denoise_window_sls(model, kv, w0, _ptr(tok), _ptr(mask), _ptr(need), n_need, W, _ptr(out_id),
                                         _ptr(out_conf), _stream(stream)), "dllm_denoise_window_sls")


def dllm_accept_drafts(conf, ids, draft_ids, tok, mask, n: int, theta: float, accepted_pos=None, n_accepted=None,
                       stream=None):
    _check(lib().dllm_accept_drafts(_ptr(conf), _ptr(ids), _ptr(draft_ids), _ptr(tok), _ptr(mask), n, float(theta),
                                    _ptr(accepted_pos), _ptr(n_accepted), _stream(stream)), "dllm_accept_drafts")


def dllm_record_drafts(ids, mask, draft_ids, n: int, stream=None):
    _check(lib().dllm_record_drafts(_ptr(ids), _ptr(mask), _ptr(draft_ids), n, _stream(stream)),
           "dllm_record_drafts")


def dllm_step_merged(model: int, kv: int, ref_pos, ref_ids, n_ref: int, block_tok, n_block: int, tok, mask,
                     W: int, out_id=None, out_conf=None, ref_out_id=None, ref_out_conf=None, stream=None):
    _check(lib().dllm_step_merged(model, kv, _ptr(ref_pos), _ptr(ref_ids), n_ref, _ptr(block_tok), n_block,
                                  _ptr(tok), _ptr(mask), W, _ptr(out_id), _ptr(out_conf), _ptr(ref_out_id),
                                  _ptr(ref_out_conf), _stream(stream)), "dllm_step_merged")


def dllm_debug_logits(model: int, kv: int, tok, mask, W: int, logits, out_id=None, out_conf=None, stream=None):
    _check(lib().dllm_debug_logits(model, kv, _ptr(tok), _ptr(mask), W, _ptr(logits), _ptr(out_id),
                                   _ptr(out_conf), _stream(stream)), "dllm_debug_logits")


def dllm_debug_hidden(model: int, kv: int, tok, mask, W: int, n_layers: int, x, stream=None):
    _check(lib().dllm_debug_hidden(model, kv, _ptr(tok), _ptr(mask), W, n_layers, _ptr(x), _stream(stream)),
           "dllm_debug_hidden")


def dllm_probe_enable(model: int, kernel_class: int, max_records: int):
    _check(lib().dllm_probe_enable(model, kernel_class, max_records), "dllm_probe_enable")


def dllm_probe_read(model: int):
    n, ms = _i32(), ctypes.c_double()
    _check(lib().dllm_probe_read(model, ctypes.byref(n), ctypes.byref(ms)), "dllm_probe_read")
    return n.value, ms.value


def dllm_kernel_replay(model: int, kv: int, kernel_class: int, W: int, n_launches: int, stream=None):
    _check(lib().dllm_kernel_replay(model, kv, kernel_class, W, n_launches, _stream(stream)), "dllm_kernel_replay")


def dllm_kernel_bytes(model: int, kernel_class: int, W: int, P: int) -> float:
    b = ctypes.c_double()
    _check(lib().dllm_kernel_bytes(model, kernel_class, W, P, ctypes.byref(b)), "dllm_kernel_bytes")
    return b.value


DLLM_TOKEN_INVISIBLE, DLLM_TOKEN_VISIBLE, DLLM_TOKEN_STABLE = 0, 1, 2


def dllm_commit_staged(conf, ids, tok, mask, state, seg_begin: int, seg_len: int, theta_visible: float,
                       theta_stable: float, promoted_pos=None, n_promoted=None, stream=None):
    _check(lib().dllm_commit_staged(_ptr(conf), _ptr(ids), _ptr(tok), _ptr(mask), _ptr(state), seg_begin, seg_len,
                                    theta_visible, theta_stable, _ptr(promoted_pos), _ptr(n_promoted),
                                    _stream(stream)), "dllm_commit_staged")


def dllm_quantize_q4_0(src, src_dtype: int, rows: int, K: int, codes, scales, stream=None):
    _check(lib().dllm_quantize_q4_0(_ptr(src), src_dtype, rows, K, _ptr(codes), _ptr(scales), _stream(stream)),
           "dllm_quantize_q4_0")


def dllm_quantize_int8(src, src_dtype: int, rows: int, K: int, codes, scales, stream=None):
    _check(lib().dllm_quantize_int8(_ptr(src), src_dtype, rows, K, _ptr(codes), _ptr(scales), _stream(stream)),
           "dllm_quantize_int8")


def dllm_read_bandwidth(buf, nbytes: int, sink, stream=None):
    _check(lib().dllm_read_bandwidth(_ptr(buf), nbytes, _ptr(sink), _stream(stream)), "dllm_read_bandwidth")


# ----------------------------------------------------------------------------
# Batch operators: sizes, types and row strides come from the tensors; workspaces,
# where none is given, from torch's allocator on the current stream
# ----------------------------------------------------------------------------

class _Types:
    """torch and its element types, looked up at the first batch call (torch is not imported with this module)."""

    torch = None

    @classmethod
    def load(cls):
        import torch
        cls.i32, cls.f32 = torch.int32, torch.float32
        cls.elem = {torch.float32: DLLM_F32, torch.bfloat16: DLLM_BF16, torch.float16: DLLM_F16}
        # (the index without torch's check for its first use, which a tensor on a GPU has made: 0.2 us a call)
        cls.device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        cls.torch = torch


def _refuse(func: str, msg: str):
    raise DllmError(DLLM_E_INVAL, func, msg)


_NO_SHAPE = (ValueError, IndexError, ZeroDivisionError)
_NO_FIT = (struct.error, OverflowError)
_NO_FIT_MSG = "an argument is no number of its field's range"


def _gpu(func: str, ref) -> int:
    """The current GPU's index, which ref must be on."""
    if _Types.torch is None:
        _Types.load()
    dev = ref.get_device()
    if dev < 0 or dev != _Types.device():
        _refuse(func, "tensors must be on the current GPU")
    return dev


def _fits(func: str, a, b):
    """Two numbers that go through ctypes, which cuts them to 32 bits without a word."""
    try:
        _pack_2i(a, b)
    except _NO_FIT:
        _refuse(func, _NO_FIT_MSG)


# The checks below run for every call, beside launches of 3 us: they test first and look for names only to refuse.


def _plain(func: str, dev: int, dtype, tensors, names: str):
    """Every tensor that is there: on that GPU, of that type, contiguous."""
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous()):
            bad = names.split()[[u is t for u in tensors].index(True)]
            _refuse(func, f"{bad} must be a contiguous {dtype} tensor on the same GPU")


def _at_least(func: str, n: int, tensors, names: str):
    for t in tensors:
        if t is not None and t.numel() < n:
            bad = names.split()[[u is t for u in tensors].index(True)]
            _refuse(func, f"{bad} must have at least {n} entries")


_PAGES_MSG = "k_pages must be [n_pages][kv_heads][page][head_dim], q and q_out [rows][heads][head_dim] or [rows][heads * head_dim]"


def _row_stride(func: str, name: str, t, dtype, dev: int, rows: int, heads: int, dim: int) -> int:
    """Row stride of a [rows][heads * dim] or [rows][heads][dim] tensor whose rows are whole; checks its shape."""
    sh, st = t.shape, t.stride()
    if len(sh) == 2:
        ok = sh[1] == heads * dim and st[1] == 1
    else:
        ok = len(sh) == 3 and sh[1] == heads and sh[2] == dim and st[2] == 1 and (heads == 1 or st[1] == dim)
    if not ok or sh[0] != rows or t.dtype is not dtype or t.get_device() != dev:
        _refuse(func, f"{name} must be [rows][{heads}][{dim}] with whole rows, of q's type and device")
    return st[0] if rows > 1 else heads * dim


def dllm_batch_plan(length, new, owned, owned_out, table, free, n_free, n_free_out, page: int, shared_pages: int, row0,
                    pos, slot, seq, lim, status, stream=None):
    """The row arrays' common length is the plan's max_rows; free has an entry per page of the pool."""
    f, B, ld, R, N = "dllm_batch_plan", length.numel(), table.shape[-1], pos.numel(), free.numel()
    dev = _gpu(f, length)
    _plain(f, dev, _Types.i32, (length, new, owned, owned_out, table, free, n_free, n_free_out, row0, pos, slot,
                                            seq, lim, status),
           "length new owned owned_out table free n_free n_free_out row0 pos slot seq lim status")
    if (new.numel() < B or owned.numel() < B or owned_out.numel() < B or slot.numel() < R or seq.numel() < R or
            lim.numel() < R or table.numel() < B * ld or row0.numel() <= B or status.numel() < 3 or not n_free.numel() or
            not n_free_out.numel()):
        _refuse(f, "new, owned and owned_out must have an entry and table a row per sequence (row0: one entry more), slot, seq "
                   "and lim as many as pos, status 3, n_free 1")
    _fits(f, page, shared_pages)
    rc = lib().dllm_batch_plan(length.data_ptr(), new.data_ptr(), owned.data_ptr(), owned_out.data_ptr(), B,
                               table.data_ptr(), ld, free.data_ptr(), n_free.data_ptr(), n_free_out.data_ptr(), N, page,
                               shared_pages, R, row0.data_ptr(), pos.data_ptr(), slot.data_ptr(), seq.data_ptr(),
                               lim.data_ptr(), status.data_ptr(), _stream(stream, dev))
    if rc:
        _check(rc, f)


def dllm_rope_table(table, head_dim: int, rope_base: float, stream=None):
    """table: float32 [max_pos][head_dim / 2][2]."""
    f = "dllm_rope_table"
    _plain(f, _gpu(f, table), _Types.f32, (table,), "table")
    _fits(f, head_dim, table.numel() // max(head_dim, 1))
    if head_dim < 1 or table.numel() % head_dim != 0:
        _refuse(f, "table must be [max_pos][head_dim / 2][2]")
    _check(lib().dllm_rope_table(table.data_ptr(), table.numel() // head_dim, head_dim, rope_base, _stream(stream)), f)


def dllm_qk_norm_rope(q, k, v, rope, pos, slot, q_out, k_pages, v_pages, q_gain=None, k_gain=None, eps: float = 1e-6,
                      stream=None):
    """q, k, v: [rows][heads][dim] or [rows][heads * dim], rows may be strided (slices of one projection's output);
    k_pages [n_pages][kv_heads][page][dim], v_pages [n_pages][kv_heads][dim][page]."""
    f, dt = "dllm_qk_norm_rope", q.dtype
    dev, qs = _gpu(f, q), q_out.shape
    try:
        T, (n_pages, kv, page, dim) = q.shape[0], k_pages.shape
        H = qs[1] if len(qs) == 3 else qs[1] // dim
    except _NO_SHAPE:
        _refuse(f, _PAGES_MSG)
    ld_q, ld_k = _row_stride(f, "q", q, dt, dev, T, H, dim), _row_stride(f, "k", k, dt, dev, T, kv, dim)
    ld_v = _row_stride(f, "v", v, dt, dev, T, kv, dim)
    _plain(f, dev, dt, (k_pages, v_pages, q_out), "k_pages v_pages q_out")
    _plain(f, dev, _Types.f32, (rope, q_gain, k_gain), "rope q_gain k_gain")
    _plain(f, dev, _Types.i32, (pos, slot), "pos slot")
    if (v_pages.shape != (n_pages, kv, dim, page) or pos.numel() < T or slot.numel() < T or qs[0] < T or
            q_out.numel() != qs[0] * H * dim or (q_gain is not None and q_gain.numel() < dim) or
            (k_gain is not None and k_gain.numel() < dim)):
        _refuse(f, "v_pages must be [n_pages][kv_heads][head_dim][page], q_out [rows][heads][dim], pos and slot have an entry "
                   "per row, gains head_dim")
    if T == 0:                      # (empty tensors have no address)
        return
    try:
        a = _pack_qk(_Types.elem.get(dt, -1), T, H, kv, dim, page, n_pages, rope.numel() // dim, eps, q.data_ptr(),
                     k.data_ptr(), v.data_ptr(), ld_q, ld_k, ld_v, 0 if q_gain is None else q_gain.data_ptr(),
                     0 if k_gain is None else k_gain.data_ptr(), rope.data_ptr(), pos.data_ptr(), slot.data_ptr(),
                     q_out.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr())
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    rc = lib().dllm_qk_norm_rope(a, _stream(stream, dev))
    if rc:
        _check(rc, f)


def _workspace(query, a, ws, stream, dev: int, f: str):
    """(args with their workspace, `ws` or memory of the call's own: on the current stream, freed once the call has been
    made)."""
    if ws is None:
        n = _sz()
        rc = query(a, n)
        if rc:
            _check(rc, f + "_ws")
        if not n.value:
            return a, None
        if stream is not None:
            _refuse(f, "a call on a given stream needs a workspace of the caller's")
        ws = _Types.torch.empty(n.value, dtype=_Types.torch.uint8, device=dev)
        return a[:-16] + _pack_ws(ws.data_ptr(), n.value), ws
    if ws.get_device() != dev or not ws.is_contiguous():
        _refuse(f, "ws must be a contiguous tensor on the same GPU")
    return a[:-16] + _pack_ws(ws.data_ptr(), ws.numel() * ws.element_size()), ws


def _attention(f, q, k_pages, v_pages, table, row0, length, out, max_rows, max_len, shared_len, lim, scale, ws, stream,
               mask=None):
    dt, sh = q.dtype, q.shape
    dev, B = _gpu(f, q), length.numel()
    try:
        T, ld, (n_pages, kv, page, dim) = sh[0], table.shape[-1], k_pages.shape
        H = sh[1] if len(sh) == 3 else sh[1] // dim
    except _NO_SHAPE:
        _refuse(f, _PAGES_MSG)
    ld_q, ld_out = _row_stride(f, "q", q, dt, dev, T, H, dim), _row_stride(f, "out", out, dt, dev, T, H, dim)
    _plain(f, dev, dt, (k_pages, v_pages), "k_pages v_pages")
    _plain(f, dev, _Types.i32, (table, row0, length, lim), "table row0 length lim")
    if (v_pages.shape != (n_pages, kv, dim, page) or table.numel() < B * ld or row0.numel() <= B or
            (lim is not None and lim.numel() < T)):
        _refuse(f, "v_pages must be [n_pages][kv_heads][head_dim][page], table must have a row and row0 an entry per sequence "
                   "(row0: one more), lim an entry per row")
    if mask is not None:
        _plain(f, dev, _Types.i32, (mask,), "mask")
        if mask.dim() != 2 or mask.shape[0] < T:
            _refuse(f, "mask must be [rows][words]")
    if T == 0:
        return
    try:
        a = _pack_attn(_Types.elem.get(dt, -1), T, B, H, kv, dim, page, n_pages, ld, shared_len, max_rows, max_len,
                       dim ** -0.5 if scale is None else scale, q.data_ptr(), ld_q, k_pages.data_ptr(),
                       v_pages.data_ptr(), table.data_ptr(), row0.data_ptr(), length.data_ptr(),
                       0 if lim is None else lim.data_ptr(), out.data_ptr(), ld_out, 0, 0)
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    L = lib()
    a, keep = _workspace(L.dllm_attention_paged_ws if mask is None else L.dllm_attention_tree_ws, a, ws, stream, dev, f)
    if mask is None:
        rc = L.dllm_attention_paged(a, _stream(stream, dev))
    else:
        rc = L.dllm_attention_tree(a, mask.data_ptr(), mask.shape[1], _stream(stream, dev))
    if rc:
        _check(rc, f)
    del keep


def dllm_attention_paged(q, k_pages, v_pages, table, row0, length, out, max_rows: int, max_len: int,
                         shared_len: int = 0, lim=None, scale: Optional[float] = None, ws=None, stream=None):
    """q, out: [rows][heads][dim] or [rows][heads * dim], rows may be strided; scale: 1 / sqrt(dim) if None;
    k_pages [n_pages][kv_heads][page][dim], v_pages [n_pages][kv_heads][dim][page]."""
    _attention("dllm_attention_paged", q, k_pages, v_pages, table, row0, length, out, max_rows, max_len, shared_len, lim,
               scale, ws, stream)


def _select_args(f, logits, out_id, out_conf, mask_id=-1, row0=None, hist=None, hist0=None, n_prompt=None, repetition=None,
                 presence=None, frequency=None, bias_id=None, bias=None, bias0=None, allow=None, allow_row=None,
                 out_logits=None, ws=None, stream=None):
    """(args, what keeps its workspace alive, the GPU) of a selection."""
    dev, dt = _gpu(f, logits), logits.dtype
    if (hist is not None and hist0 is None) or (bias is None) != (bias_id is None) or (bias is None) != (bias0 is None):
        _refuse(f, "hist needs hist0; bias, bias_id and bias0 go together")
    n_allow = allow_ld = 0
    try:
        T, V = logits.shape
        if allow is not None:
            n_allow, allow_ld = allow.shape
    except ValueError:
        _refuse(f, "logits must be [rows][vocab], allow [masks][words]")
    B = row0.numel() - 1 if row0 is not None else 1
    i32, f32 = [out_id], [out_conf]
    ok = out_id.numel() >= T and out_conf.numel() >= T and (V == 1 or logits.stride(1) == 1)
    p_row0 = p_hist = p_hist0 = p_prompt = p_rep = p_pres = p_freq = p_bias_id = p_bias = p_bias0 = p_allow = 0
    p_allow_row = p_out = ld_out = 0
    if row0 is not None:
        i32.append(row0)
        p_row0 = row0.data_ptr()
    if hist is not None:
        i32 += [hist, hist0]
        ok = ok and hist0.numel() > B
        p_hist0 = hist0.data_ptr()
        p_hist = hist.data_ptr() or p_hist0          # (an empty tensor has no address; nothing is read through this one)
    if n_prompt is not None:
        i32.append(n_prompt)
        ok = ok and n_prompt.numel() >= B
        p_prompt = n_prompt.data_ptr()
    if repetition is not None:
        f32.append(repetition)
        p_rep = repetition.data_ptr()
    if presence is not None:
        f32.append(presence)
        p_pres = presence.data_ptr()
    if frequency is not None:
        f32.append(frequency)
        p_freq = frequency.data_ptr()
    for t in f32[1:]:
        ok = ok and t.numel() >= B
    if bias is not None:
        i32 += [bias_id, bias0]
        f32.append(bias)
        ok = ok and bias0.numel() > B and bias.numel() >= bias_id.numel()
        p_bias0 = bias0.data_ptr()
        p_bias_id, p_bias = bias_id.data_ptr() or p_bias0, bias.data_ptr() or p_bias0
    if allow is not None:
        i32.append(allow)
        p_allow = allow.data_ptr()
    if allow_row is not None:
        i32.append(allow_row)
        ok = ok and allow_row.numel() >= T
        p_allow_row = allow_row.data_ptr()
    if out_logits is not None:
        ok = ok and (out_logits.shape == logits.shape and out_logits.dtype is dt and out_logits.get_device() == dev and
                     (V == 1 or out_logits.stride(1) == 1))
        p_out, ld_out = out_logits.data_ptr(), out_logits.stride(0) if T > 1 else V
    _plain(f, dev, _Types.i32, i32, "array " * len(i32))
    _plain(f, dev, _Types.f32, f32, "array " * len(f32))
    if not ok:
        _refuse(f, "out_id, out_conf and allow_row must have an entry per row, n_prompt and the penalties one per sequence "
                   "(hist0, bias0: one more), out_logits be of the logits' shape and type, rows be whole")
    try:
        a = _pack_select(_Types.elem.get(dt, -1), T, V, mask_id, B, logits.data_ptr(), logits.stride(0) if T > 1 else V,
                         p_row0, p_hist, p_hist0, p_prompt, p_rep, p_pres, p_freq, p_bias_id, p_bias, p_bias0, p_allow,
                         n_allow, allow_ld, p_allow_row, p_out, ld_out, out_id.data_ptr(), out_conf.data_ptr(), 0, 0)
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    return _workspace(lib().dllm_select_ws, a, ws, stream, dev, f) + (dev,)


def dllm_select(logits, out_id, out_conf, stream=None, **control):
    """logits (and out_logits): [rows][vocab], rows may be strided.  control: mask_id, row0, hist, hist0, n_prompt,
    repetition, presence, frequency, bias_id, bias, bias0, allow (int32 words [masks][words]), allow_row, out_logits, ws."""
    f = "dllm_select"
    sh = logits.shape
    if len(sh) == 2 and sh[0] == 0:
        return
    a, keep, dev = _select_args(f, logits, out_id, out_conf, stream=stream, **control)
    rc = lib().dllm_select(a, _stream(stream, dev))
    if rc:
        _check(rc, f)
    del keep


def dllm_model_set_qk_norm(model: int, q_gains, k_gains, stream=None):
    """q_gains, k_gains: one float32 [head_dim] tensor per layer."""
    f = "dllm_model_set_qk_norm"
    layers, dim = _gain_sizes.get(model, (len(q_gains), 1))
    if not len(q_gains) == len(k_gains) == layers or layers == 0:
        _refuse(f, f"q_gains and k_gains must have a tensor for each of the model's {layers} layers")
    if any(t.numel() != dim for t in (*q_gains, *k_gains)) and model in _gain_sizes:
        _refuse(f, f"a gain must have the model's head_dim of {dim} entries")
    _plain(f, _gpu(f, q_gains[0]), _Types.f32, tuple(q_gains) + tuple(k_gains), "gain " * (len(q_gains) + len(k_gains)))
    q, k = ((_vp * len(g))(*[t.data_ptr() for t in g]) for g in (q_gains, k_gains))
    _check(lib().dllm_model_set_qk_norm(model, q, k, _stream(stream)), f)


def dllm_batch_bytes(model: int, n_pages: int, page: int) -> int:
    n = _sz()
    _fits("dllm_batch_bytes", n_pages, page)
    _check(lib().dllm_batch_bytes(model, n_pages, page, ctypes.byref(n)), "dllm_batch_bytes")
    return n.value


def _batch_step(f, model, pages, n_pages, page, tok, mask, table, row0, pos, slot, length, max_rows, max_len, out_id, out_conf,
                shared_len, lim, logits, control, stream, tree=None):
    dev, R, B, ld = _gpu(f, tok), tok.numel(), length.numel(), table.shape[-1]
    _plain(f, dev, _Types.i32, (tok, table, row0, pos, slot, length, lim, out_id), "tok table row0 pos slot length lim out_id")
    _plain(f, dev, _Types.torch.uint8, (mask,), "mask")
    _plain(f, dev, _Types.f32, (out_conf, logits), "out_conf logits")
    _at_least(f, R, (pos, slot, lim, mask, out_id, out_conf), "pos slot lim mask out_id out_conf")
    if table.numel() < B * ld or row0.numel() < B + 1 or pages.get_device() != dev or not pages.is_contiguous():
        _refuse(f, "table must have a row and row0 an entry per sequence (row0: one more), pages be on the same GPU")
    if tree is not None:
        _plain(f, dev, _Types.i32, (tree,), "tree")
        if tree.dim() != 2 or tree.shape[0] < R:
            _refuse(f, "tree must be [rows][words]")
    try:
        rows = _pack_rows(R, B, page, n_pages, ld, shared_len, max_rows, max_len, table.data_ptr(), row0.data_ptr(),
                          pos.data_ptr(), slot.data_ptr(), length.data_ptr(), _ptr(lim) or 0)
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    sel = keep = None
    if (control and logits is None) or (logits is not None and (out_id is None or out_conf is None)):
        _refuse(f, "control needs logits, and logits need out_id and out_conf")
    if logits is not None:
        sel, keep, _ = _select_args(f, logits, out_id, out_conf, stream=stream, **(control or {}))
    head, tail = (model, pages.data_ptr(), pages.numel() * pages.element_size(), rows), (
        tok.data_ptr(), _ptr(mask), sel, _ptr(out_id), _ptr(out_conf), _stream(stream))
    if tree is None:
        _check(lib().dllm_batch_step(*head, *tail), f)
    else:
        _check(lib().dllm_batch_step_tree(*head, tree.data_ptr(), tree.shape[1], *tail), f)
    del keep


def dllm_batch_step(model: int, pages, n_pages: int, page: int, tok, mask, table, row0, pos, slot, length, max_rows: int,
                    max_len: int, out_id=None, out_conf=None, shared_len: int = 0, lim=None, logits=None, control=None,
                    stream=None):
    """tok's length is the number of rows.  logits (float32 [rows][vocab]) with control, a dict of dllm_select's options:
    the outputs come from the controlled logits."""
    _batch_step("dllm_batch_step", model, pages, n_pages, page, tok, mask, table, row0, pos, slot, length, max_rows, max_len,
                out_id, out_conf, shared_len, lim, logits, control, stream)


# ----------------------------------------------------------------------------
# Branches: trees of drafted rows, their log probabilities, accepted paths and forks
# ----------------------------------------------------------------------------


def dllm_tree_plan(parent, row0, length, pos, mask, stream=None):
    """parent and pos: an entry per row; mask: int32 words [rows][words]."""
    f, B = "dllm_tree_plan", length.numel()
    dev = _gpu(f, length)
    _plain(f, dev, _Types.i32, (parent, row0, length, pos, mask), "parent row0 length pos mask")
    if mask.dim() != 2:
        _refuse(f, "mask must be [rows][words]")
    T, ld = mask.shape
    if row0.numel() <= B or parent.numel() < T or pos.numel() < T:
        _refuse(f, "row0 must have an entry per sequence and one more, parent and pos an entry per row of mask")
    if T == 0:
        return
    _fits(f, T, ld)
    rc = lib().dllm_tree_plan(parent.data_ptr(), row0.data_ptr(), length.data_ptr(), T, B, pos.data_ptr(), mask.data_ptr(), ld,
                              _stream(stream, dev))
    if rc:
        _check(rc, f)


def dllm_attention_tree(q, k_pages, v_pages, table, row0, length, mask, out, max_rows: int, max_len: int,
                        shared_len: int = 0, lim=None, scale: Optional[float] = None, ws=None, stream=None):
    """As dllm_attention_paged, with mask: int32 words [rows][words]."""
    if mask is None:
        _refuse("dllm_attention_tree", "mask must be [rows][words]")
    _attention("dllm_attention_tree", q, k_pages, v_pages, table, row0, length, out, max_rows, max_len, shared_len, lim, scale,
               ws, stream, mask)


def dllm_batch_step_tree(model: int, pages, n_pages: int, page: int, tok, mask, tree, table, row0, pos, slot, length,
                         max_rows: int, max_len: int, out_id=None, out_conf=None, shared_len: int = 0, lim=None, logits=None,
                         control=None, stream=None):
    """As dllm_batch_step, with tree: int32 words [rows][words], and pos: dllm_tree_plan's."""
    if tree is None:
        _refuse("dllm_batch_step_tree", "tree must be [rows][words]")
    _batch_step("dllm_batch_step_tree", model, pages, n_pages, page, tok, mask, table, row0, pos, slot, length, max_rows, max_len,
                out_id, out_conf, shared_len, lim, logits, control, stream, tree)


def dllm_logprobs(logits, tok=None, tok_row=None, logp=None, entropy=None, top_id=None, top_logp=None, mask_id: int = -1,
                  ws=None, stream=None):
    """logits: [rows][vocab], rows may be strided; tok, tok_row and logp: an entry per token; entropy: one per row;
    top_id and top_logp: [rows][top]."""
    f = "dllm_logprobs"
    dev, dt = _gpu(f, logits), logits.dtype
    if logits.dim() != 2:
        _refuse(f, "logits must be [rows][vocab]")
    T, V = logits.shape
    if (tok is None) != (logp is None) or (tok is None and tok_row is not None) or (top_id is None) != (top_logp is None):
        _refuse(f, "tok and logp, top_id and top_logp go together; tok_row needs tok")
    _plain(f, dev, _Types.i32, (tok, tok_row, top_id), "tok tok_row top_id")
    _plain(f, dev, _Types.f32, (logp, entropy, top_logp), "logp entropy top_logp")
    n = 0 if tok is None else tok.numel()
    top = 0
    if top_id is not None:
        if top_id.dim() != 2 or top_id.shape[0] != T or top_logp.shape != top_id.shape:
            _refuse(f, "top_id and top_logp must be [rows][top]")
        top = top_id.shape[1]
    if ((V > 1 and logits.stride(1) != 1) or (n and logp.numel() < n) or (tok_row is not None and tok_row.numel() < n) or
            (entropy is not None and entropy.numel() < T)):
        _refuse(f, "rows must be whole, logp and tok_row have an entry per token, entropy one per row")
    if T == 0 and n == 0:
        return
    try:
        a = _pack_logprobs(_Types.elem.get(dt, -1), T, V, mask_id, n, top, logits.data_ptr(), logits.stride(0) if T > 1 else V,
                           tok.data_ptr() if n else 0, tok_row.data_ptr() if n and tok_row is not None else 0,
                           logp.data_ptr() if n else 0, 0 if entropy is None else entropy.data_ptr(),
                           top_id.data_ptr() if top else 0, top_logp.data_ptr() if top else 0, 0, 0)
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    L = lib()
    a, keep = _workspace(L.dllm_logprobs_ws, a, ws, stream, dev, f)
    rc = L.dllm_logprobs(a, _stream(stream, dev))
    if rc:
        _check(rc, f)
    del keep


def _cache(f, dev, pages, page) -> bytes:
    """The dllm_cache of pages [layers][2][n_pages][kv_heads][page * head_dim]."""
    sh = pages.shape
    if pages.get_device() != dev or not pages.is_contiguous():
        _refuse(f, "pages must be a contiguous tensor on the same GPU")
    if len(sh) != 5 or sh[1] != 2 or page < 1 or sh[4] % page != 0:
        _refuse(f, "pages must be [layers][2][n_pages][kv_heads][page * head_dim]")
    try:
        return _pack_cache(_Types.elem.get(pages.dtype, -1), sh[0], sh[3], sh[4] // page, page, sh[2], pages.data_ptr())
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)


def dllm_cache_compact(pages, page: int, table, base, path, n, stream=None):
    """pages: [layers][2][n_pages][kv_heads][page * head_dim], as dllm_batch_step's; base and n: an entry per
    sequence; path: [sequences][entries]."""
    f, B = "dllm_cache_compact", base.numel()
    dev = _gpu(f, base)
    c = _cache(f, dev, pages, page)
    _plain(f, dev, _Types.i32, (table, base, path, n), "table base path n")
    if path.dim() != 2 or path.shape[0] < B or n.numel() < B or table.numel() < B * table.shape[-1]:
        _refuse(f, "path must be [sequences][entries], n have an entry and table a row per sequence")
    _fits(f, table.shape[-1], path.shape[1])
    rc = lib().dllm_cache_compact(c, table.data_ptr(), table.shape[-1], base.data_ptr(), path.data_ptr(), path.shape[1],
                                  n.data_ptr(), B, _stream(stream, dev))
    if rc:
        _check(rc, f)


def dllm_batch_fork(src, keep, owned, owned_out, table, table_out, free, n_free, n_free_out, shared_pages: int, pages,
                    page: int, status, ws=None, stream=None):
    """src, keep, owned and owned_out: an entry, table and table_out: a row per sequence; free: an entry per page of
    pages, [layers][2][n_pages][kv_heads][page * head_dim]."""
    f, B, ld = "dllm_batch_fork", src.numel(), table.shape[-1]
    dev = _gpu(f, src)
    c = _cache(f, dev, pages, page)
    _plain(f, dev, _Types.i32, (src, keep, owned, owned_out, table, table_out, free, n_free, n_free_out, status),
           "src keep owned owned_out table table_out free n_free n_free_out status")
    if (keep.numel() < B or owned.numel() < B or owned_out.numel() < B or table.numel() < B * ld or
            table_out.shape != table.shape or free.numel() < pages.shape[2] or not n_free.numel() or not n_free_out.numel() or
            status.numel() < 3):
        _refuse(f, "keep, owned and owned_out must have an entry, table and table_out a row per sequence, free an entry per page, "
                   "status 3, n_free 1")
    try:
        a = _pack_fork(B, ld, shared_pages, src.data_ptr(), keep.data_ptr(), owned.data_ptr(), owned_out.data_ptr(),
                       table.data_ptr(), table_out.data_ptr(), free.data_ptr(), n_free.data_ptr(), n_free_out.data_ptr(),
                       status.data_ptr(), 0, 0)
    except _NO_FIT:
        _refuse(f, _NO_FIT_MSG)
    L, n_pages = lib(), pages.shape[2]
    a, hold = _workspace(lambda _, out: L.dllm_batch_fork_ws(B, n_pages, out), a, ws, stream, dev, f)
    rc = L.dllm_batch_fork(c, a, _stream(stream, dev))
    if rc:
        _check(rc, f)
    del hold


# ----------------------------------------------------------------------------
# Convenience holders: device weights and handles
# ----------------------------------------------------------------------------


DTYPES = {"f32": DLLM_F32, "bf16": DLLM_BF16, "w8": DLLM_W8, "q4": DLLM_Q4}


def make_config(shape, dtype: str, max_window: int = 64, max_pos: int = 8192) -> dllm_config:
    return dllm_config(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ff, shape.vocab,
                       shape.mask_id, shape.block, shape.eps, shape.rope_base, DTYPES[dtype], max_window, max_pos,
                       getattr(shape, "n_kv_heads", 0), int(getattr(shape, "qkv_bias", False)))


class Model:
    """A library model built from host weight arrays (float32 or bf16 bit patterns).

    `layer_source(l)` may stream one layer at a time (dict of arrays) so that the
    device copy of the caller-side weights never exceeds one layer.
    """

    def __init__(self, shape, dtype: str, globals_: dict, layer_source, max_window: int = 64,
                 max_pos: int = 8192, device: str = "cuda"):
        import numpy as np
        import torch

        self.shape, self.dtype = shape, dtype
        self.cfg = make_config(shape, dtype, max_window, max_pos)
        dev = torch.device(device)

        def up(a):
            a = np.ascontiguousarray(a)
            if a.dtype == np.uint16:
                return torch.from_numpy(a.view(np.int16)).to(dev).view(torch.bfloat16)
            return torch.from_numpy(a.astype(np.float32, copy=False)).to(dev)

        keep = []
        LW = dllm_layer_weights * shape.n_layers
        layers = LW()
        # Weights are uploaded in full before create; large models pass them layer by layer
        # through the same create call by uploading everything first (device memory is ample).
        for l in range(shape.n_layers):
            src = layer_source(l)
            t = {k: up(v) for k, v in src.items()}
            keep.append(t)
            layers[l] = dllm_layer_weights(*[t[k].data_ptr() if k in t else None
                                             for k in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "attn_norm",
                                                       "ffn_norm", "bq", "bk", "bv")])
        g = {k: up(v) for k, v in globals_.items()}
        keep.append(g)
        w = dllm_weights(g["embed"].data_ptr(), g["lm_head"].data_ptr(), g["final_norm"].data_ptr(), layers)
        stream = torch.cuda.current_stream()
        self.handle = dllm_model_create(self.cfg, w, stream)
        del keep
        torch.cuda.empty_cache()

    def close(self):
        if getattr(self, "handle", None):
            dllm_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVCache:
    """A torch-allocated KV cache buffer wrapped by the library."""

    def __init__(self, model: Model, capacity: int, device: str = "cuda"):
        import torch

        self.model = model
        self.capacity = capacity
        self.nbytes = dllm_kv_bytes(model.handle, capacity)
        self.buf = torch.zeros(self.nbytes // 2 + 8, dtype=torch.int16, device=device)
        self.handle = dllm_kv_create(model.handle, self.buf, self.nbytes, capacity)

    @property
    def row_stride(self) -> int:
        return (self.capacity + 31) // 32 * 32

    def views(self):
        """(K [L][Hkv][Cs][Dh], V^T [L][Hkv][Dh][Cs]) as float32 tensors (Hkv K/V heads).

        fp32 models: views of the buffer.  bf16 / int8 / Q4_0 models: the fp16 planes,
        widened (a new tensor, not a view)."""
        import torch

        sh = self.model.shape
        Cs = self.row_stride
        Hkv = getattr(sh, "kv_heads", sh.n_heads)
        plane = Hkv * Cs * sh.head_dim
        if self.model.dtype == "f32":
            flat = self.buf.view(torch.uint8)[: sh.n_layers * 2 * plane * 4].view(torch.float32)
            per = flat.view(sh.n_layers, 2, plane)
            K, Vt = per[:, 0], per[:, 1]
        else:
            flat = self.buf.view(torch.uint8)[: sh.n_layers * 2 * plane * 2].view(torch.float16)
            per = flat.view(sh.n_layers, 2, plane).float()
            K, Vt = per[:, 0], per[:, 1]
        return (K.reshape(sh.n_layers, Hkv, Cs, sh.head_dim),
                Vt.reshape(sh.n_layers, Hkv, sh.head_dim, Cs))

    @property
    def prefix_len(self) -> int:
        return dllm_kv_prefix_len(self.handle)[0]

    @property
    def prompt_len(self) -> int:
        return dllm_kv_prefix_len(self.handle)[1]

    def close(self):
        if getattr(self, "handle", None):
            dllm_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
