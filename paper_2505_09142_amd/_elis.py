"""ctypes binding of libelis (include/elis.h): argument marshalling only.

Every function below has the name of the C entry point it calls and passes
its arguments through unchanged (device pointers as Python ints, the stream
as a hipStream_t handle). All computation happens in the HIP kernels of
libelis.so; if the library is missing this module raises at import-use time,
and there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint32, c_void_p

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libelis.so")

ELIS_OK = 0
ELIS_EINVAL = -1
ELIS_ESHAPE = -2
ELIS_EWORKSPACE = -3
ELIS_EHIP = -4
ELIS_EDEVICE = -5
ELIS_EUNSUPPORTED = -6

ELIS_DEV_BAD_TOKEN = 1
ELIS_DEV_BAD_CU = 2
ELIS_DEV_LONG_SEQ = 4
ELIS_DEV_BAD_SLOT = 8
ELIS_DEV_PACK_SIZE = 16
ELIS_DEV_NO_PAGES = 32
ELIS_DEV_BAD_PAGE = 64

ELIS_POOL_CLS = 0
ELIS_POOL_MEAN = 1

ELIS_ACT_RELU = 0
ELIS_ACT_IDENTITY = 1
ELIS_EPI_BIAS_BF16 = 0
ELIS_EPI_BIAS_GELU_BF16 = 1
ELIS_EPI_BIAS_RES_F32 = 2
ELIS_DT_F32 = 0
ELIS_DT_BF16 = 1

KERNEL_CLASSES = ("seqmap", "embed_ln", "gemm_qkv", "attention", "gemm_o", "layernorm", "gemm_ffn1",
                  "gemm_ffn2", "pool_head", "select", "jobs", "pages", "kv", "kv_attention", "logits")
K = {name: i for i, name in enumerate(KERNEL_CLASSES)}


class ElisLibraryMissing(RuntimeError):
    pass


class ElisError(RuntimeError):
    def __init__(self, status: int, where: str = ""):
        self.status = status
        super().__init__(f"{where}: {elis_status_string(status)} ({status})")


class elis_config(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("d_model", c_int32), ("n_heads", c_int32), ("d_ff", c_int32),
                ("vocab", c_int32), ("max_pos", c_int32), ("pooling", c_int32), ("head_hidden", c_int32),
                ("head_layers", c_int32), ("head_act", c_int32),
                ("ln_eps", c_float), ("out_scale", c_float), ("out_shift", c_float)]


class elis_layer_weights(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_qkv", "w_o", "w_1", "w_2", "b_qkv", "b_o", "b_1", "b_2",
                                        "ln1_g", "ln1_b", "ln2_g", "ln2_b")]


class elis_weights(ctypes.Structure):
    _fields_ = [("cfg", elis_config), ("word", c_void_p), ("pos", c_void_p), ("type0", c_void_p),
                ("emb_ln_g", c_void_p), ("emb_ln_b", c_void_p), ("layers", POINTER(elis_layer_weights)),
                ("head_w1", c_void_p), ("head_b1", c_void_p), ("head_w2", c_void_p), ("head_b2", c_void_p),
                ("head_mid_w", POINTER(c_void_p)), ("head_mid_b", POINTER(c_void_p))]


class elis_job_table(ctypes.Structure):
    _fields_ = [("base", c_void_p), ("max_jobs", c_int32), ("max_pos", c_int32)]


class elis_page_pool(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("state", "free_pages", "held", "table", "scratch")] + \
               [(n, c_int32) for n in ("n_pages", "page_tokens", "max_jobs", "max_pages")]


class elis_kv_cache(ctypes.Structure):
    _fields_ = [("base", c_void_p)] + [(n, c_int32) for n in ("n_pages", "page_tokens", "n_kv_heads", "d_head")]


# name -> (restype, argtypes); mirrors include/elis.h
SIGNATURES = {
    "elis_abi_version": (c_int32, []),
    "elis_status_string": (ctypes.c_char_p, [c_int]),
    "elis_predict_workspace_bytes": (c_size_t, [POINTER(elis_config), c_int32, c_int32, c_int32]),
    "elis_predict_remaining": (c_int, [POINTER(elis_weights), c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                       c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "elis_select_max_n": (c_int32, []),
    "elis_select_max_batch_cap": (c_int32, [c_int32]),
    "elis_select_workspace_bytes": (c_size_t, [c_int32]),
    "elis_isrtf_select": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_size_t,
                                  c_void_p]),
    "elis_isrtf_select_noalloc": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "elis_read_status": (c_int, [c_void_p, c_void_p, POINTER(c_uint32)]),
    "elis_linear": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p,
                            c_void_p]),
    "elis_linear_plan": (c_int, [c_int32, c_int32, c_int32, c_int32, POINTER(c_int32)]),
    "elis_linear_with_plan": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32,
                                      POINTER(c_int32), c_void_p, c_void_p]),
    "elis_attention_workspace_bytes": (c_size_t, [c_int32, c_int32]),
    "elis_attention": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                               c_size_t, c_void_p]),
    "elis_layernorm": (c_int, [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_float, c_void_p, c_void_p,
                               c_void_p]),
    "elis_pool_head_workspace_bytes": (c_size_t, [POINTER(elis_config), c_int32, c_int32]),
    "elis_pool_head": (c_int, [POINTER(elis_weights), c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                               c_void_p, c_size_t, c_void_p]),
    "elis_jobs_table_bytes": (c_size_t, [c_int32, c_int32]),
    "elis_jobs_init": (c_int, [POINTER(elis_job_table), c_void_p]),
    "elis_jobs_start": (c_int, [POINTER(elis_job_table), c_void_p, c_void_p, c_int32, c_void_p]),
    "elis_jobs_append": (c_int, [POINTER(elis_job_table), c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                 c_void_p]),
    "elis_jobs_pack": (c_int, [POINTER(elis_job_table), c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                               c_void_p]),
    "elis_jobs_store_pred": (c_int, [POINTER(elis_job_table), c_void_p, c_void_p, c_int32, c_void_p]),
    "elis_jobs_select_workspace_bytes": (c_size_t, [c_int32]),
    "elis_jobs_select": (c_int, [POINTER(elis_job_table), c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                 c_void_p, c_size_t, c_void_p]),
    "elis_jobs_select_aged": (c_int, [POINTER(elis_job_table), c_void_p, c_void_p, c_float, c_int32, c_int32,
                                      c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "elis_pages_init": (c_int, [POINTER(elis_page_pool), c_void_p]),
    "elis_pages_grow": (c_int, [POINTER(elis_page_pool), c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                c_void_p, c_void_p, c_void_p]),
    "elis_pages_trim": (c_int, [POINTER(elis_page_pool), c_void_p, c_void_p, c_int32, c_void_p]),
    "elis_kv_cache_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32]),
    "elis_kv_init": (c_int, [POINTER(elis_kv_cache), c_void_p]),
    "elis_kv_append": (c_int, [POINTER(elis_kv_cache), c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_int32,
                               c_void_p]),
    "elis_kv_read": (c_int, [POINTER(elis_kv_cache), c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_int64,
                             c_void_p]),
    "elis_kv_attention_workspace_bytes": (c_size_t, [c_int32] * 7),
    "elis_kv_attention": (c_int, [POINTER(elis_kv_cache), c_void_p, c_int64, c_void_p, c_int32, c_int32, c_int32,
                                  c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_int32, c_int32, c_float, c_int32,
                                  c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "elis_logits_adjust": (c_int, [c_void_p, c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_int32, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                   c_int32, c_int64, c_void_p, c_void_p, c_int64, c_void_p]),
    "elis_timing_enable": (c_int, [c_uint32]),
    "elis_timing_stride": (c_int, [c_int32]),
    "elis_timing_reset": (c_int, []),
    "elis_timing_read": (c_int, [c_int32, POINTER(c_int32), POINTER(c_double)]),
}

_lib = None


def lib():
    """The loaded libelis.so (raises ElisLibraryMissing when it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ElisLibraryMissing(f"{LIB_PATH} not found: build it with `python -m paper_2505_09142_amd.build`")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        _lib = h
    return _lib


def elis_abi_version() -> int:
    return lib().elis_abi_version()


def elis_status_string(status: int) -> str:
    return lib().elis_status_string(status).decode()


def elis_predict_workspace_bytes(cfg: elis_config, total_tokens: int, n_seqs: int, max_seqlen: int) -> int:
    return lib().elis_predict_workspace_bytes(ctypes.byref(cfg), total_tokens, n_seqs, max_seqlen)


def elis_predict_remaining(w: elis_weights, token_ids: int, cu_seqlens: int, n_seqs: int, total_tokens: int,
                           max_seqlen: int, out_pred: int, out_hidden: int | None, workspace: int, ws_bytes: int,
                           stream: int | None) -> int:
    return lib().elis_predict_remaining(ctypes.byref(w) if w is not None else None, token_ids, cu_seqlens, n_seqs,
                                        total_tokens, max_seqlen, out_pred, out_hidden, workspace, ws_bytes, stream)


def elis_select_max_n() -> int:
    return lib().elis_select_max_n()


def elis_select_max_batch_cap(n: int) -> int:
    return lib().elis_select_max_batch_cap(n)


def elis_select_workspace_bytes(n: int) -> int:
    return lib().elis_select_workspace_bytes(n)


def elis_isrtf_select(pred: int, arrival_seq: int, n: int, batch_cap: int, out_idx: int, out_count: int,
                      workspace: int, ws_bytes: int, stream: int | None) -> int:
    return lib().elis_isrtf_select(pred, arrival_seq, n, batch_cap, out_idx, out_count, workspace, ws_bytes, stream)


ELIS_SELECT_NOALLOC_MAX_N = 1 << 18
ELIS_SELECT_NOALLOC_SCRATCH_BYTES = 3 << 20


def elis_isrtf_select_noalloc(pred: int, arrival_seq: int, n: int, batch_cap: int, out_idx: int, out_count: int,
                              stream: int | None) -> int:
    return lib().elis_isrtf_select_noalloc(pred, arrival_seq, n, batch_cap, out_idx, out_count, stream)


def elis_read_status(workspace: int, stream: int | None):
    """Returns (status, bits)."""
    bits = c_uint32(0)
    st = lib().elis_read_status(workspace, stream, ctypes.byref(bits))
    return st, bits.value


def elis_linear(x: int, w: int, bias: int, residual: int | None, m: int, n: int, k: int, epilogue: int, out: int,
                stream: int | None) -> int:
    return lib().elis_linear(x, w, bias, residual, m, n, k, epilogue, out, stream)


def elis_linear_with_plan(x: int, w: int, bias: int, residual: int | None, m: int, n: int, k: int, epilogue: int,
                          plan, out: int, stream: int | None) -> int:
    p = (c_int32 * 7)(*plan) if plan is not None else None
    return lib().elis_linear_with_plan(x, w, bias, residual, m, n, k, epilogue, p, out, stream)


def elis_linear_plan(m: int, n: int, k: int, epilogue: int):
    """Returns (status, (main_bm, main_bn, main_wgs, m1, rest_bm, rest_bn, rest_wgs))."""
    out = (c_int32 * 7)()
    st = lib().elis_linear_plan(m, n, k, epilogue, out)
    return st, tuple(out)


def elis_attention_workspace_bytes(n_seqs: int, total_tokens: int) -> int:
    return lib().elis_attention_workspace_bytes(n_seqs, total_tokens)


def elis_attention(qkv: int, cu_seqlens: int, n_seqs: int, total_tokens: int, max_seqlen: int, n_heads: int,
                   d_head: int, out: int, workspace: int, ws_bytes: int, stream: int | None) -> int:
    return lib().elis_attention(qkv, cu_seqlens, n_seqs, total_tokens, max_seqlen, n_heads, d_head, out, workspace,
                                ws_bytes, stream)


def elis_layernorm(x: int, g: int, b: int, rows: int, d: int, eps: float, out_f32: int | None,
                   out_bf16: int | None, stream: int | None) -> int:
    return lib().elis_layernorm(x, g, b, rows, d, eps, out_f32, out_bf16, stream)


def elis_pool_head_workspace_bytes(cfg: elis_config, n_seqs: int, max_seqlen: int) -> int:
    return lib().elis_pool_head_workspace_bytes(ctypes.byref(cfg), n_seqs, max_seqlen)


def elis_pool_head(w: elis_weights, hidden: int, cu_seqlens: int, n_seqs: int, total_tokens: int, max_seqlen: int,
                   out_pred: int, workspace: int, ws_bytes: int, stream: int | None) -> int:
    return lib().elis_pool_head(ctypes.byref(w) if w is not None else None, hidden, cu_seqlens, n_seqs,
                                total_tokens, max_seqlen, out_pred, workspace, ws_bytes, stream)


_byref = ctypes.byref


def _tab(t):
    return None if t is None else _byref(t)


def elis_jobs_table_bytes(max_jobs: int, max_pos: int) -> int:
    return lib().elis_jobs_table_bytes(max_jobs, max_pos)


def elis_jobs_init(t: elis_job_table, stream: int | None) -> int:
    return lib().elis_jobs_init(_tab(t), stream)


def elis_jobs_start(t: elis_job_table, slots: int, arrival_seq: int, m: int, stream: int | None) -> int:
    return lib().elis_jobs_start(_tab(t), slots, arrival_seq, m, stream)


def elis_jobs_append(t: elis_job_table, slots: int, tok_offsets: int, tokens: int | None, m: int, total_new: int,
                     stream: int | None) -> int:
    return lib().elis_jobs_append(_tab(t), slots, tok_offsets, tokens, m, total_new, stream)


def elis_jobs_pack(t: elis_job_table, slots: int, n: int, total_tokens: int, max_seqlen: int, out_token_ids: int,
                   out_cu_seqlens: int, stream: int | None) -> int:
    return lib().elis_jobs_pack(_tab(t), slots, n, total_tokens, max_seqlen, out_token_ids, out_cu_seqlens, stream)


def elis_jobs_store_pred(t: elis_job_table, slots: int, pred: int, n: int, stream: int | None) -> int:
    return lib().elis_jobs_store_pred(_tab(t), slots, pred, n, stream)


def elis_jobs_select_workspace_bytes(a: int) -> int:
    return lib().elis_jobs_select_workspace_bytes(a)


def elis_jobs_select(t: elis_job_table, slots: int, a: int, batch_cap: int, out_slots: int | None, out_count: int,
                     workspace: int, ws_bytes: int, stream: int | None) -> int:
    return lib().elis_jobs_select(_tab(t), slots, a, batch_cap, out_slots, out_count, workspace, ws_bytes, stream)


def elis_jobs_select_aged(t: elis_job_table, slots: int, wait: int, aging: float, a: int, batch_cap: int,
                          out_slots: int | None, out_count: int, workspace: int, ws_bytes: int,
                          stream: int | None) -> int:
    return lib().elis_jobs_select_aged(_tab(t), slots, wait, aging, a, batch_cap, out_slots, out_count, workspace,
                                       ws_bytes, stream)


def elis_pages_init(p: elis_page_pool, stream: int | None) -> int:
    return lib().elis_pages_init(_tab(p), stream)


def elis_pages_grow(p: elis_page_pool, slots: int, lens: int, cu_new: int | None, n: int, total_new: int, width: int,
                    out_blocks: int | None, out_slot_map: int | None, stream: int | None) -> int:
    return (_lib or lib()).elis_pages_grow(_tab(p), slots, lens, cu_new, n, total_new, width, out_blocks, out_slot_map, stream)


def elis_pages_trim(p: elis_page_pool, slots: int, lens: int, n: int, stream: int | None) -> int:
    return (_lib or lib()).elis_pages_trim(_tab(p), slots, lens, n, stream)


def elis_kv_cache_bytes(n_pages: int, page_tokens: int, n_kv_heads: int, d_head: int) -> int:
    return lib().elis_kv_cache_bytes(n_pages, page_tokens, n_kv_heads, d_head)


def elis_kv_init(c: elis_kv_cache, stream: int | None) -> int:
    return lib().elis_kv_init(_tab(c), stream)


def elis_kv_append(c: elis_kv_cache, k: int, v: int, k_stride: int, v_stride: int, slot_map: int, n_tokens: int,
                   stream: int | None) -> int:
    return (_lib or lib()).elis_kv_append(_tab(c), k, v, k_stride, v_stride, slot_map, n_tokens, stream)


def elis_kv_read(c: elis_kv_cache, slot_map: int, n_tokens: int, out_k: int, out_v: int, k_stride: int, v_stride: int,
                 stream: int | None) -> int:
    return (_lib or lib()).elis_kv_read(_tab(c), slot_map, n_tokens, out_k, out_v, k_stride, v_stride, stream)


def elis_kv_attention_workspace_bytes(n: int, total_q: int, max_q: int, max_kv: int, n_heads: int, n_kv_heads: int,
                                      d_head: int) -> int:
    return lib().elis_kv_attention_workspace_bytes(n, total_q, max_q, max_kv, n_heads, n_kv_heads, d_head)


def elis_kv_attention(c: elis_kv_cache, q: int, q_stride: int, cu_q: int, n: int, total_q: int, max_q: int, blocks: int,
                      block_rows: int, blocks_stride: int, rows: int | None, kv_lens: int, max_kv: int, n_heads: int,
                      scale: float, window: int, out: int, out_stride: int, workspace: int, ws_bytes: int,
                      stream: int | None) -> int:
    return (_lib or lib()).elis_kv_attention(_tab(c), q, q_stride, cu_q, n, total_q, max_q, blocks, block_rows, blocks_stride,
                                   rows, kv_lens, max_kv, n_heads, scale, window, out, out_stride, workspace, ws_bytes,
                                   stream)


def elis_logits_adjust(logits: int, dtype: int, in_stride: int, n: int, vocab: int, token_ids: int | None,
                       cu_seqlens: int | None, total_tokens: int, prompt_lens: int | None, repetition: int | None,
                       frequency: int | None, presence: int | None, bias_cu: int | None, bias_tokens: int | None,
                       bias_values: int | None, bias_total: int, mask: int | None, n_masks: int, mask_stride: int,
                       mask_rows: int | None, out: int, out_stride: int, stream: int | None) -> int:
    return (_lib or lib()).elis_logits_adjust(logits, dtype, in_stride, n, vocab, token_ids, cu_seqlens, total_tokens,
                                    prompt_lens, repetition, frequency, presence, bias_cu, bias_tokens, bias_values,
                                    bias_total, mask, n_masks, mask_stride, mask_rows, out, out_stride, stream)


def elis_timing_enable(class_mask: int) -> int:
    return lib().elis_timing_enable(class_mask)


def elis_timing_stride(every: int) -> int:
    return lib().elis_timing_stride(every)


def elis_timing_reset() -> int:
    return lib().elis_timing_reset()


def elis_timing_read(kernel_class: int):
    """Returns (status, launches, total_ms)."""
    n = c_int32(0)
    ms = c_double(0.0)
    st = lib().elis_timing_read(kernel_class, ctypes.byref(n), ctypes.byref(ms))
    return st, n.value, ms.value


def check(status: int, where: str = "") -> None:
    if status != ELIS_OK:
        raise ElisError(status, where)
