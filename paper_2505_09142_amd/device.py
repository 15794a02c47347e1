"""Device-side plumbing around libelis: weights resident in HBM, workspaces, streams.

PyTorch is used here only to own device memory and to name the current HIP
stream; every step of the predictor and of the selection runs in libelis'
kernels, reached through the same-named calls of ``_elis``.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import _elis as E

I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
BF16_KEYS = ("word", "pos", "w_qkv", "w_o", "w_1", "w_2")


def _stream(stream) -> int:
    if stream is None:  # the handle itself: making torch's stream object costs as much as a launch (2.8 us)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """An empty tensor that work on `stream` may write at once: memory that other streams' work may still use is not handed
    out again to this one."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream))):
        return torch.empty(shape, dtype=dtype, device=device)


def _to_dev(a: np.ndarray, device) -> torch.Tensor:
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device)  # bf16 bit patterns
    if a.dtype == np.float32:
        return torch.from_numpy(a).to(device)
    raise TypeError(a.dtype)


def config_of(shape) -> E.elis_config:
    """elis_config from any object with the encoder-shape attributes."""
    return E.elis_config(shape.n_layers, shape.d_model, shape.n_heads, shape.d_ff, shape.vocab, shape.max_pos,
                         shape.pooling, shape.head_hidden, shape.n_head_layers, shape.head_act, shape.ln_eps,
                         shape.out_scale, shape.out_shift)


class DeviceWeights:
    """Uploads one predictor's parameters and builds the elis_weights struct.

    ``tensors`` is a dict in the layout of include/elis.h: bf16 bit patterns
    (uint16) for the embedding tables and the four layer matrices, fp32 for the
    rest; per-layer entries are lists.
    """

    def __init__(self, shape, tensors: dict, device="cuda"):
        self.shape = shape
        self.cfg = config_of(shape)
        self.t = {}
        for k, v in tensors.items():
            self.t[k] = [_to_dev(x, device) for x in v] if isinstance(v, list) else _to_dev(v, device)
        L = shape.n_layers
        self._layers = (E.elis_layer_weights * max(1, L))()
        for l in range(L):
            y = self._layers[l]
            for name in ("w_qkv", "w_o", "w_1", "w_2", "b_qkv", "b_o", "b_1", "b_2", "ln1_g", "ln1_b", "ln2_g",
                         "ln2_b"):
                setattr(y, name, self.t[name][l].data_ptr())
        p = lambda k: self.t[k].data_ptr() if k in self.t else None
        nmid = len(self.t.get("head_mid_w", []))
        self._mid_w = (ctypes.c_void_p * max(1, nmid))(*[x.data_ptr() for x in self.t.get("head_mid_w", [])])
        self._mid_b = (ctypes.c_void_p * max(1, nmid))(*[x.data_ptr() for x in self.t.get("head_mid_b", [])])
        mid = lambda a: ctypes.cast(a, ctypes.POINTER(ctypes.c_void_p)) if nmid else None
        self.struct = E.elis_weights(self.cfg, p("word"), p("pos"), p("type0"), p("emb_ln_g"), p("emb_ln_b"),
                                     ctypes.cast(self._layers, ctypes.POINTER(E.elis_layer_weights)),
                                     p("head_w1"), p("head_b1"), p("head_w2"), p("head_b2"),
                                     mid(self._mid_w), mid(self._mid_b))


class Workspace:
    """A growable, 256-byte-aligned device scratch buffer owned by torch."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None

    def get(self, nbytes: int) -> tuple[int, int]:
        nbytes = max(256, int(nbytes))
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.buf.data_ptr()
        aligned = (base + 255) // 256 * 256
        return aligned, self.buf.numel() - (aligned - base)


class Predictor:
    """elis_predict_remaining + elis_isrtf_select on resident weights."""

    def __init__(self, weights: DeviceWeights, device="cuda"):
        self.w = weights
        self.device = device
        self.ws = Workspace(device)
        self.sel_ws = Workspace(device)

    def predict(self, token_ids: torch.Tensor, cu_seqlens: torch.Tensor, max_seqlen: int, out_pred=None,
                want_hidden=False, stream=None):
        n = cu_seqlens.numel() - 1
        T = token_ids.numel()
        need = E.elis_predict_workspace_bytes(self.w.cfg, T, n, max_seqlen)
        if need == 0:
            raise E.ElisError(E.ELIS_EINVAL, "elis_predict_workspace_bytes")
        ws, wsb = self.ws.get(need)
        if out_pred is None:
            out_pred = torch.empty(n, dtype=torch.float32, device=self.device)
        hid = torch.empty((T, self.w.shape.d_model), dtype=torch.float32, device=self.device) if want_hidden else None
        st = E.elis_predict_remaining(self.w.struct, token_ids.data_ptr(), cu_seqlens.data_ptr(), n, T, max_seqlen,
                                      out_pred.data_ptr(), hid.data_ptr() if hid is not None else None, ws, wsb,
                                      _stream(stream))
        E.check(st, "elis_predict_remaining")
        return out_pred, hid

    def status(self, stream=None):
        ws, _ = self.ws.get(0)
        return E.elis_read_status(ws, _stream(stream))

    def select(self, pred: torch.Tensor, arrival: torch.Tensor, batch_cap: int, out_idx=None, out_count=None,
               stream=None):
        n = pred.numel()
        if out_idx is None:
            out_idx = torch.full((max(1, batch_cap),), -1, dtype=torch.int32, device=self.device)
        if out_count is None:
            out_count = torch.zeros(1, dtype=torch.int32, device=self.device)
        ws, wsb = self.sel_ws.get(E.elis_select_workspace_bytes(n))
        st = E.elis_isrtf_select(pred.data_ptr(), arrival.data_ptr(), n, batch_cap, out_idx.data_ptr(),
                                 out_count.data_ptr(), ws, wsb, _stream(stream))
        E.check(st, "elis_isrtf_select")
        return out_idx, out_count


def upload_batch(batch, device="cuda"):
    """(token_ids, cu_seqlens, arrival_seq) of a packed batch as device tensors."""
    return (torch.from_numpy(batch.token_ids).to(device), torch.from_numpy(batch.cu_seqlens).to(device),
            torch.from_numpy(batch.arrival_seq).to(device))


class JobTable:
    """Device-resident job table (elis_jobs_*): per job slot the first token, a ring of the most
    recent max_pos - 1 tokens, the length, the cached prediction and the arrival number."""

    def __init__(self, max_jobs: int, max_pos: int, device="cuda", stream=None):
        nbytes = E.elis_jobs_table_bytes(max_jobs, max_pos)
        if nbytes == 0:
            raise E.ElisError(E.ELIS_EINVAL, "elis_jobs_table_bytes")
        self.device = device
        self.buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        base = (self.buf.data_ptr() + 255) // 256 * 256
        self.t = E.elis_job_table(base, max_jobs, max_pos)
        self.max_jobs, self.max_pos = max_jobs, max_pos
        self.sel_ws = Workspace(device)
        E.check(E.elis_jobs_init(self.t, _stream(stream)), "elis_jobs_init")

    def start(self, slots: torch.Tensor, arrival: torch.Tensor, stream=None):
        E.check(E.elis_jobs_start(self.t, slots.data_ptr(), arrival.data_ptr(), slots.numel(), _stream(stream)),
                "elis_jobs_start")

    def append(self, slots: torch.Tensor, offsets: torch.Tensor, tokens: torch.Tensor, total: int, stream=None):
        E.check(E.elis_jobs_append(self.t, slots.data_ptr(), offsets.data_ptr(),
                                   tokens.data_ptr() if total > 0 else None, slots.numel(), total, _stream(stream)),
                "elis_jobs_append")

    def pack(self, slots: torch.Tensor, total: int, max_seqlen: int, out_ids: torch.Tensor, out_cu: torch.Tensor,
             stream=None):
        E.check(E.elis_jobs_pack(self.t, slots.data_ptr(), slots.numel(), total, max_seqlen, out_ids.data_ptr(),
                                 out_cu.data_ptr(), _stream(stream)), "elis_jobs_pack")

    def store_pred(self, slots: torch.Tensor, pred: torch.Tensor, stream=None):
        E.check(E.elis_jobs_store_pred(self.t, slots.data_ptr(), pred.data_ptr(), slots.numel(), _stream(stream)),
                "elis_jobs_store_pred")

    def select(self, slots: torch.Tensor, batch_cap: int, out_slots: torch.Tensor, out_count: torch.Tensor,
               stream=None, wait: torch.Tensor | None = None, aging: float = 0.0):
        """Select over the cached keys; with `wait` (fp32 seconds per candidate) the keys are aged by
        `aging` tokens per second (elis_jobs_select_aged)."""
        a = slots.numel()
        ws, wsb = self.sel_ws.get(E.elis_jobs_select_workspace_bytes(a))
        if wait is None:
            E.check(E.elis_jobs_select(self.t, slots.data_ptr(), a, batch_cap, out_slots.data_ptr(),
                                       out_count.data_ptr(), ws, wsb, _stream(stream)), "elis_jobs_select")
        else:
            E.check(E.elis_jobs_select_aged(self.t, slots.data_ptr(), wait.data_ptr(), aging, a, batch_cap,
                                            out_slots.data_ptr(), out_count.data_ptr(), ws, wsb, _stream(stream)),
                    "elis_jobs_select_aged")

    def status(self, stream=None):
        return E.elis_read_status(self.t.base, _stream(stream))


def _dev() -> int:
    """The current device: kernels are launched there, so every argument has to be on it."""
    return torch._C._cuda_getDevice()


def _arg(t: torch.Tensor, dtype: torch.dtype, dev: int, where: str, at_least: int = 0) -> int:
    """Address of a contiguous argument of the given type, on device `dev`, of at least so many elements."""
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or (at_least and t.numel() < at_least):
        raise E.ElisError(E.ELIS_EINVAL, where)
    return t.data_ptr()


def _made_on(dev: int, where: str):
    """A state that a kernel of this call sets up has to lie on the current device."""
    if dev < 0 or dev != _dev():
        raise E.ElisError(E.ELIS_EINVAL, where)


def _opt(t: torch.Tensor | None, dtype: torch.dtype, dev: int, where: str, at_least: int = 0) -> int | None:
    """As _arg, None for None. (Its check once more: calling it for each of a call's arguments costs 0.6 us.)"""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or (at_least and t.numel() < at_least):
        raise E.ElisError(E.ELIS_EINVAL, where)
    return t.data_ptr()


def _heads(x: torch.Tensor, tokens: int, heads: int, d: int, dev: int, where: str) -> int:
    """Token stride of a [tokens, heads, d] or [tokens, heads * d] bf16 tensor whose rows are contiguous."""
    if x.dtype is not BF16 or x.get_device() != dev:
        raise E.ElisError(E.ELIS_EINVAL, where)
    shape, stride = x.shape, x.stride()
    if shape == (tokens, heads, d):
        if stride[2] == 1 and (heads == 1 or stride[1] == d):
            return stride[0] if tokens > 1 else heads * d
    elif shape == (tokens, heads * d):
        if stride[1] == 1:
            return stride[0] if tokens > 1 else heads * d
    else:
        raise E.ElisError(E.ELIS_ESHAPE, where)
    raise E.ElisError(E.ELIS_EINVAL, where)


class PagePool:
    """Pages of a KV cache handed out to job slots on the device (elis_pages_*): a stack of free pages and the
    pages each slot holds. ``tensors`` is (state, free_pages, held, table) of an existing pool; without it the
    pool starts with every page free."""

    def __init__(self, n_pages: int, page_tokens: int, max_jobs: int, max_pages: int, device="cuda", tensors=None,
                 stream=None):
        self.n_pages, self.page_tokens, self.max_jobs, self.max_pages = n_pages, page_tokens, max_jobs, max_pages
        sizes = ((2,), (n_pages,), (max_jobs,), (max_jobs, max_pages))
        if min(n_pages, page_tokens, max_jobs, max_pages) < 1:
            raise E.ElisError(E.ELIS_EINVAL, "PagePool")
        made = tensors is None
        if made:
            tensors = [_empty(s, I32, device, stream) for s in sizes]
        for t, s in zip(tensors, sizes, strict=True):
            if tuple(t.shape) != s:
                raise E.ElisError(E.ELIS_ESHAPE, "PagePool")
            _arg(t, torch.int32, tensors[0].get_device(), "PagePool")
        self.state, self.free_pages, self.held, self.table = tensors
        self.scratch = _empty(4 * max_jobs + 4, I32, self.state.device, stream)
        self.p = E.elis_page_pool(*(t.data_ptr() for t in (*tensors, self.scratch)), n_pages, page_tokens, max_jobs,
                                  max_pages)
        if made:
            _made_on(self.state.get_device(), "elis_pages_init")
            E.check(E.elis_pages_init(self.p, _stream(stream)), "elis_pages_init")

    def grow(self, slots: torch.Tensor, lens: torch.Tensor, cu_new: torch.Tensor | None, total_new: int,
             out_slot_map: torch.Tensor | None, out_blocks: torch.Tensor | None = None, stream=None):
        """Pages for lens[i] tokens of job slots[i]; the slots of the step's total_new new tokens into out_slot_map
        and, if given, the batch's block table into out_blocks [n, width]."""
        n, i32, dev, where = slots.numel(), I32, self.state.get_device(), "elis_pages_grow"
        if dev != _dev():
            raise E.ElisError(E.ELIS_EINVAL, where)
        if out_blocks is not None and (out_blocks.dim() != 2 or out_blocks.shape[0] != n):
            raise E.ElisError(E.ELIS_ESHAPE, where)
        E.check(E.elis_pages_grow(self.p, _arg(slots, i32, dev, where), _arg(lens, i32, dev, where, n),
                                  _opt(cu_new, i32, dev, where, n + 1), n, total_new,
                                  0 if out_blocks is None else out_blocks.shape[1], _opt(out_blocks, i32, dev, where),
                                  _opt(out_slot_map, i32, dev, where, total_new), _stream(stream)), where)

    def trim(self, slots: torch.Tensor, lens: torch.Tensor, stream=None):
        """Job slots[i] keeps the pages of its first lens[i] tokens; the others are free again."""
        n, dev, where = slots.numel(), self.state.get_device(), "elis_pages_trim"
        if dev != _dev():
            raise E.ElisError(E.ELIS_EINVAL, where)
        E.check(E.elis_pages_trim(self.p, _arg(slots, I32, dev, where), _arg(lens, I32, dev, where, n), n,
                                  _stream(stream)), where)

    def status(self, stream=None):
        return E.elis_read_status(self.p.state, _stream(stream))


class KVCache:
    """One layer's keys and values in 4 bits, in pages (elis_kv_*), and attention over them. ``buf`` is an existing
    cache's memory (uint8, 256-byte aligned); without it the cache is allocated and its status cleared."""

    def __init__(self, n_pages: int, page_tokens: int, n_kv_heads: int, d_head: int, device="cuda",
                 buf: torch.Tensor | None = None, stream=None):
        nbytes = E.elis_kv_cache_bytes(n_pages, page_tokens, n_kv_heads, d_head)
        if nbytes == 0:
            raise E.ElisError(E.ELIS_EINVAL, "elis_kv_cache_bytes")
        self.n_pages, self.page_tokens, self.n_kv_heads, self.d_head = n_pages, page_tokens, n_kv_heads, d_head
        made = buf is None
        if made:
            buf = _empty(nbytes + 256, torch.uint8, device, stream)
        base = (buf.data_ptr() + 255) // 256 * 256
        _arg(buf, torch.uint8, buf.get_device(), "KVCache", base - buf.data_ptr() + nbytes)
        self.buf, self.dev = buf, buf.get_device()
        self.c = E.elis_kv_cache(base, n_pages, page_tokens, n_kv_heads, d_head)
        self.ws = Workspace(buf.device)
        self._no_ws = self.ws.get(256)[0]
        self._last = None, 0  # sizes of an attention call and the workspace they take: one tuple, so that threads see a pair
        if made:
            _made_on(self.dev, "elis_kv_init")
            E.check(E.elis_kv_init(self.c, _stream(stream)), "elis_kv_init")

    def _here(self, where: str) -> int:
        if self.dev != _dev():
            raise E.ElisError(E.ELIS_EINVAL, where)
        return self.dev

    def append(self, k: torch.Tensor, v: torch.Tensor, slot_map: torch.Tensor, stream=None):
        """bf16 [tokens, n_kv_heads, d_head] (rows of a wider matrix are taken as they are) into their slots."""
        n, where = slot_map.numel(), "elis_kv_append"
        dev = self._here(where)
        ks = _heads(k, n, self.n_kv_heads, self.d_head, dev, where)
        vs = _heads(v, n, self.n_kv_heads, self.d_head, dev, where)
        E.check(E.elis_kv_append(self.c, k.data_ptr(), v.data_ptr(), ks, vs, _arg(slot_map, I32, dev, where), n,
                                 _stream(stream)), where)

    def read(self, slot_map: torch.Tensor, out_k: torch.Tensor, out_v: torch.Tensor, stream=None):
        """What the cache keeps of the tokens in slot_map, as bf16."""
        n, where = slot_map.numel(), "elis_kv_read"
        dev = self._here(where)
        ks = _heads(out_k, n, self.n_kv_heads, self.d_head, dev, where)
        vs = _heads(out_v, n, self.n_kv_heads, self.d_head, dev, where)
        E.check(E.elis_kv_read(self.c, _arg(slot_map, I32, dev, where), n, out_k.data_ptr(), out_v.data_ptr(), ks, vs,
                               _stream(stream)), where)

    def attention(self, q: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor, blocks: torch.Tensor, max_q: int,
                  max_kv: int, rows: torch.Tensor | None = None, scale: float | None = None, window: int = 0,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Causal attention of the new tokens q (bf16 [tokens, n_heads, d_head]) over the cache. ``blocks`` holds a
        row of page ids for every request, or, with ``rows``, for every job slot (a pool's table)."""
        n, i32, where = kv_lens.numel(), I32, "elis_kv_attention"
        dev = self._here(where)
        if q.dim() != 3 or blocks.dim() != 2:
            raise E.ElisError(E.ELIS_ESHAPE, where)
        total, heads, _ = q.shape
        d = self.d_head
        if out is None:
            out = _empty((total, heads, d), BF16, q.device, stream)
        qs, os_ = _heads(q, total, heads, d, dev, where), _heads(out, total, heads, d, dev, where)
        block_rows, block_cols = blocks.shape
        sizes = (n, total, max_q, max_kv, heads)
        last = self._last
        if sizes != last[0]:
            self._last = last = sizes, E.elis_kv_attention_workspace_bytes(*sizes, self.n_kv_heads, d)
        # A workspace of the call's own: calls on several streams, and captured graphs, share only the one that holds
        # nothing (256 bytes, not touched).
        ws, wsb = self._no_ws, last[1]
        if wsb > 256:
            scratch = _empty(wsb + 256, torch.uint8, q.device, stream)
            ws = (scratch.data_ptr() + 255) // 256 * 256
        E.check(E.elis_kv_attention(self.c, q.data_ptr(), qs, _arg(cu_q, i32, dev, where, n + 1), n, total, max_q,
                                    _arg(blocks, i32, dev, where), block_rows, block_cols,
                                    _opt(rows, i32, dev, where, n), _arg(kv_lens, i32, dev, where), max_kv, heads,
                                    self.d_head ** -0.5 if scale is None else scale, window, out.data_ptr(), os_, ws, wsb,
                                    _stream(stream)), where)
        return out

    def status(self, stream=None):
        return E.elis_read_status(self.c.base, _stream(stream))


def adjust_logits(logits: torch.Tensor, token_ids: torch.Tensor | None, cu_seqlens: torch.Tensor | None,
                  out: torch.Tensor | None = None, *, prompt_lens=None, repetition=None, frequency=None, presence=None,
                  bias=None, mask=None, mask_rows=None, stream=None) -> torch.Tensor:
    """elis_logits_adjust on [n, vocab] logits (bf16 or fp32, rows contiguous). token_ids / cu_seqlens: the histories
    as JobTable.pack writes them. bias: (cu [n + 1], tokens, values). mask: int32 or uint32 [n_masks, words]."""
    where, dev = "elis_logits_adjust", _dev()
    if logits.dim() != 2 or (logits.dtype is not F32 and logits.dtype is not BF16) or logits.stride(1) != 1 or \
            logits.get_device() != dev:
        raise E.ElisError(E.ELIS_EINVAL, where)
    n, vocab = logits.shape
    if out is None:
        out = _empty((n, vocab), F32, logits.device, stream)
    if out.shape != logits.shape or out.dtype is not F32 or out.stride(1) != 1 or out.get_device() != dev:
        raise E.ElisError(E.ELIS_EINVAL, where)
    f32, i32 = F32, I32
    b_cu, b_tok, b_val = bias if bias is not None else (None, None, None)
    total = 0 if token_ids is None else token_ids.numel()
    n_bias = 0 if b_tok is None else b_tok.numel()
    masks = words = 0
    if mask is not None:
        if mask.dim() != 2 or mask.dtype not in (torch.int32, torch.uint32):
            raise E.ElisError(E.ELIS_EINVAL, where)
        masks, words = mask.shape
    E.check(E.elis_logits_adjust(logits.data_ptr(), E.ELIS_DT_F32 if logits.dtype is f32 else E.ELIS_DT_BF16,
                                 logits.stride(0) if n > 1 else vocab, n, vocab, _opt(token_ids, i32, dev, where),
                                 _opt(cu_seqlens, i32, dev, where, n + 1), total, _opt(prompt_lens, i32, dev, where, n),
                                 _opt(repetition, f32, dev, where, n), _opt(frequency, f32, dev, where, n),
                                 _opt(presence, f32, dev, where, n), _opt(b_cu, i32, dev, where, n + 1),
                                 _opt(b_tok, i32, dev, where), _opt(b_val, f32, dev, where, n_bias), n_bias,
                                 None if mask is None else _arg(mask, mask.dtype, dev, where), masks, words,
                                 _opt(mask_rows, i32, dev, where, n), out.data_ptr(),
                                 out.stride(0) if n > 1 else vocab, _stream(stream)), where)
    return out
