"""The language model's side of a cache miss: a paged key/value cache that is quantised as it is written, the attention of new
tokens over it, and the verification of drafted tokens (a near hit's stored answer, or a drafting model's).  Argument
marshalling only; names and rules follow include/siso.h."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from .binding import SisoError, _ALLOC_FN, _FREE_FN, _Allocator, _ptr, load_library

ATTN_CAUSAL = 1
_CACHE_TYPES = {torch.bfloat16: 1, torch.float8_e4m3fn: 2, torch.int8: 3}
_ROW_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _stream(stream: Optional[torch.cuda.Stream], dev: torch.device) -> int:
    return (torch.cuda.current_stream(dev) if stream is None else stream).cuda_stream


class _KvConfig(ctypes.Structure):
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("d_k_exp", ctypes.c_void_p), ("d_v_exp", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("stride_layer", ctypes.c_int64), ("stride_page", ctypes.c_int64),
                ("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("n_layers", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("allocator", _Allocator)]


class _Attention(ctypes.Structure):
    _fields_ = [("d_q", ctypes.c_void_p), ("d_out", ctypes.c_void_p), ("d_lse", ctypes.c_void_p), ("d_cu_q", ctypes.c_void_p),
                ("d_kv_len", ctypes.c_void_p), ("d_pages", ctypes.c_void_p), ("q_stride_token", ctypes.c_int64),
                ("q_stride_head", ctypes.c_int64), ("out_stride_token", ctypes.c_int64), ("out_stride_head", ctypes.c_int64),
                ("pages_stride", ctypes.c_int64), ("n_tokens", ctypes.c_int64), ("n_seqs", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("layer", ctypes.c_int32), ("window", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("scale", ctypes.c_float)]


class PagedKV:
    """Handle over the pages of a key/value cache.  k, v: [layers, pages, tokens, kv heads, head dim], bfloat16, float8_e4m3fn or
    int8, any strides with the last one 1 and the same for both; 8-bit pages need k_exp, v_exp: contiguous uint8 [layers, pages,
    kv heads, tokens].  The tensors stay the caller's; the handle keeps them alive."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: Optional[torch.Tensor] = None, v_exp: Optional[torch.Tensor] = None):
        self._h = None
        if k.dtype not in _CACHE_TYPES:
            raise ValueError("pages must be bfloat16, float8_e4m3fn or int8")
        if k.dim() != 5 or k.stride(4) != 1:
            raise ValueError("pages must be [layers, pages, tokens, kv heads, head dim] with contiguous rows")
        if v.dtype != k.dtype or v.shape != k.shape or v.stride() != k.stride() or v.device != k.device:
            raise ValueError("k and v must have the same type, shape, strides and device")
        layers, pages, tokens, heads, dim = k.shape
        if (k_exp is None) != (k.dtype == torch.bfloat16) or (v_exp is None) != (k_exp is None):
            raise ValueError("8-bit pages need k_exp and v_exp, 16-bit pages have none")
        for e in (k_exp, v_exp):
            if e is not None and (e.dtype != torch.uint8 or tuple(e.shape) != (layers, pages, heads, tokens) or not e.is_contiguous()
                                  or e.device != k.device):
                raise ValueError("exponents must be contiguous uint8 [layers, pages, kv heads, tokens] beside the pages")
        if not k.is_cuda:
            raise RuntimeError("a CUDA device is required: this library has no CPU path")
        self._lib = load_library()
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.n_layers, self.n_pages, self.page_size, self.n_kv_heads, self.head_dim = layers, pages, tokens, heads, dim
        self._dev = k.device
        self._blocks = {}

        def _alloc(nbytes, stream, ctx):          # scratch from the pool of the stream it is first used on
            try:
                with torch.cuda.device(self._dev):
                    if stream:
                        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=self._dev)):
                            t = torch.empty(int(nbytes), dtype=torch.uint8, device=self._dev)
                    else:
                        t = torch.empty(int(nbytes), dtype=torch.uint8, device=self._dev)
            except Exception:                     # out of memory -> NULL -> SISO_ERR_OOM
                return None
            self._blocks[t.data_ptr()] = t
            return t.data_ptr()

        def _free(ptr, ctx):
            self._blocks.pop(ptr, None)

        self._alloc_cb, self._free_cb = _ALLOC_FN(_alloc), _FREE_FN(_free)
        cfg = _KvConfig(k.data_ptr(), v.data_ptr(), None if k_exp is None else k_exp.data_ptr(), None if v_exp is None else v_exp.data_ptr(),
                        pages, k.stride(0), k.stride(1), k.stride(2), k.stride(3), layers, tokens, heads, dim, _CACHE_TYPES[k.dtype],
                        k.device.index, _Allocator(self._alloc_cb, self._free_cb, None))
        h = ctypes.c_void_p()
        st = self._lib.siso_kv_create(ctypes.byref(h), ctypes.byref(cfg))
        self._h = h if st == 0 else None
        self._check(st, "siso_kv_create")
        self._args = _Attention()
        self._args_ref = ctypes.byref(self._args)

    @classmethod
    def allocate(cls, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16,
                 device: int = 0) -> "PagedKV":
        """A cache over new, token-major pages, every place zero."""
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: this library has no CPU path")
        dev = torch.device("cuda", device)
        k, v = (torch.zeros((n_layers, n_pages, page_size, n_kv_heads, head_dim), dtype=dtype, device=dev) for _ in range(2))
        exps = [None, None] if dtype == torch.bfloat16 else [torch.zeros((n_layers, n_pages, n_kv_heads, page_size), dtype=torch.uint8, device=dev)
                                                             for _ in range(2)]
        return cls(k, v, *exps)

    def _check(self, st: int, where: str) -> None:
        if st != 0:
            raise SisoError(st, where, self._lib.siso_last_cuda_error().decode() if st == 7 else "")

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            self._lib.siso_kv_destroy(self._h)
            self._h = None
            self._blocks.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t: torch.Tensor, n: int, name: str) -> torch.Tensor:
        if t.dtype not in _ROW_TYPES or t.device != self._dev or tuple(t.shape) != (n, self.n_kv_heads, self.head_dim):
            raise ValueError(f"{name} must be a [{n}, {self.n_kv_heads}, {self.head_dim}] float32 or bfloat16 tensor on {self._dev}")
        return t if t.stride(2) == 1 else t.contiguous()

    def _slots(self, slots: torch.Tensor) -> torch.Tensor:
        if slots.dtype != torch.int64 or slots.dim() != 1 or slots.device != self._dev:
            raise ValueError(f"slots must be a one-dimensional int64 tensor on {self._dev}")
        return slots.contiguous()

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, layer: int = 0, stream=None) -> None:
        """Rows k, v [n, kv heads, head dim] (fp32 or bf16) into `slots` [n] = page * page size + token (-1: skipped)."""
        slots = self._slots(slots)
        n = slots.shape[0]
        k, v = self._rows(k, n, "k"), self._rows(v, n, "v")
        if k.dtype != v.dtype:
            raise ValueError("k and v must have the same type")
        if k.stride() != v.stride():
            k, v = k.contiguous(), v.contiguous()
        self._check(self._lib.siso_kv_write(self._h, layer, k.data_ptr(), v.data_ptr(), _ROW_TYPES[k.dtype], n, k.stride(0), k.stride(1),
                                            slots.data_ptr(), _stream(stream, self._dev)), "siso_kv_write")

    def read(self, slots: torch.Tensor, layer: int = 0, dtype: torch.dtype = torch.bfloat16, stream=None, out=None
             ) -> Tuple[torch.Tensor, torch.Tensor]:
        """The rows of `slots` as (k, v) [n, kv heads, head dim] of `dtype` (float32 or bfloat16); zeros for slots outside the pool."""
        slots = self._slots(slots)
        n = slots.shape[0]
        if out is None:
            if dtype not in _ROW_TYPES:
                raise ValueError("dtype must be float32 or bfloat16")
            k, v = (torch.empty((n, self.n_kv_heads, self.head_dim), dtype=dtype, device=self._dev) for _ in range(2))
        else:
            k, v = out
            if self._rows(k, n, "out k") is not k or self._rows(v, n, "out v") is not v or k.stride() != v.stride() or k.dtype != v.dtype:
                raise ValueError("outputs must have contiguous rows, the same strides and the same type")
        self._check(self._lib.siso_kv_read(self._h, layer, k.data_ptr(), v.data_ptr(), _ROW_TYPES[k.dtype], n, k.stride(0), k.stride(1),
                                           slots.data_ptr(), _stream(stream, self._dev)), "siso_kv_read")
        return k, v

    def attention(self, q: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, max_q: int, layer: int = 0,
                  scale: Optional[float] = None, causal: bool = True, window: int = 0, want_lse: bool = False, stream=None,
                  out: Optional[torch.Tensor] = None):
        """q [n, heads, head dim] bf16: the queries of all sequences one after the other, sequence b's from cu_q[b] on (int32
        [seqs + 1]); kv_len int32 [seqs]: tokens in all, the new ones included (already written); pages int32 [seqs, max pages].
        Returns out [n, heads, head dim], or (out, lse [n, heads] fp32) with want_lse."""
        if q.dtype != torch.bfloat16 or q.dim() != 3 or q.shape[2] != self.head_dim or q.device != self._dev:
            raise ValueError(f"q must be a [n, heads, {self.head_dim}] bfloat16 tensor on {self._dev}")
        if not cu_q.dtype == kv_len.dtype == pages.dtype == torch.int32 or not cu_q.device == kv_len.device == pages.device == self._dev:
            raise ValueError(f"cu_q, kv_len and pages must be int32 tensors on {self._dev}")
        n, heads, _ = q.shape
        seqs = kv_len.shape[0]
        if cu_q.dim() != 1 or kv_len.dim() != 1 or cu_q.shape[0] != seqs + 1 or pages.dim() != 2 or pages.shape[0] != seqs:
            raise ValueError("cu_q must be [seqs + 1], kv_len [seqs], pages [seqs, max pages]")
        if q.stride(2) != 1:
            q = q.contiguous()
        if pages.stride(1) != 1:
            pages = pages.contiguous()
        cu_q, kv_len = cu_q.contiguous(), kv_len.contiguous()
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=torch.bfloat16, device=self._dev)
        elif out.dtype != torch.bfloat16 or out.shape != q.shape or out.device != self._dev or out.stride(2) != 1:
            raise ValueError("out must be a bfloat16 tensor like q with contiguous rows")
        lse = torch.empty((n, heads), dtype=torch.float32, device=self._dev) if want_lse else None
        a = self._args
        a.d_q, a.d_out, a.d_lse = q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else None
        a.d_cu_q, a.d_kv_len, a.d_pages = cu_q.data_ptr(), kv_len.data_ptr(), pages.data_ptr()
        a.q_stride_token, a.q_stride_head, _ = q.stride()
        a.out_stride_token, a.out_stride_head, _ = out.stride()
        a.pages_stride, a.n_tokens, a.n_seqs, a.max_q, a.max_pages = pages.stride(0), n, seqs, max_q, pages.shape[1]
        a.n_heads, a.layer, a.window, a.flags = heads, layer, window, ATTN_CAUSAL if causal else 0
        a.scale = self.head_dim ** -0.5 if scale is None else scale
        self._check(self._lib.siso_kv_attention(self._h, self._args_ref, _stream(stream, self._dev)), "siso_kv_attention")
        return (out, lse) if want_lse else out

    def sync_status(self, stream=None) -> int:
        """Synchronise and return the handle's device status word (0 = clear); it is cleared by the call."""
        return int(self._lib.siso_kv_sync_status(self._h, _stream(stream, self._dev)))

    def check_status(self, stream=None) -> None:
        st = self.sync_status(stream)
        if st != 0:
            raise SisoError(st, "device status")


def verify_drafts(target: torch.Tensor, draft: Optional[torch.Tensor], tokens: torch.Tensor, n_drafts: Optional[torch.Tensor],
                  u_accept: torch.Tensor, u_sample: torch.Tensor, stream=None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """target [seqs, drafts + 1, vocab] and draft [seqs, drafts, vocab] (or None: certain drafts) probabilities, fp32 or bf16;
    tokens int32 [seqs, drafts]; n_drafts int32 [seqs] or None (all); u_accept [seqs, drafts], u_sample [seqs] fp32 in [0, 1).
    Returns (tokens out int32 [seqs, drafts + 1]: those that stand, one drawn, then -1; accepted int32 [seqs])."""
    if target.dtype not in _ROW_TYPES or target.dim() != 3 or not target.is_cuda:
        raise ValueError("target must be a [seqs, drafts + 1, vocab] float32 or bfloat16 tensor on a GPU")
    seqs, n_max, vocab = target.shape[0], target.shape[1] - 1, target.shape[2]
    dev = target.device
    if n_max < 0:
        raise ValueError("target needs at least one row per sequence")
    if draft is not None and (draft.dtype != target.dtype or tuple(draft.shape) != (seqs, n_max, vocab) or draft.device != dev):
        raise ValueError("draft must be [seqs, drafts, vocab] of target's type and device")
    for t, dtype, shape, name in ((tokens, torch.int32, (seqs, n_max), "tokens"), (n_drafts, torch.int32, (seqs,), "n_drafts"),
                                  (u_accept, torch.float32, (seqs, n_max), "u_accept"), (u_sample, torch.float32, (seqs,), "u_sample")):
        if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or t.device != dev):
            raise ValueError(f"{name} must be a {list(shape)} {dtype} tensor on {dev}")
    target, tokens, u_accept, u_sample = target.contiguous(), tokens.contiguous(), u_accept.contiguous(), u_sample.contiguous()
    draft = None if draft is None else draft.contiguous()
    n_drafts = None if n_drafts is None else n_drafts.contiguous()
    new, accepted = out if out is not None else (torch.empty((seqs, n_max + 1), dtype=torch.int32, device=dev),
                                                 torch.empty((seqs,), dtype=torch.int32, device=dev))
    L = load_library()
    with torch.cuda.device(dev):
        st = L.siso_verify_drafts(_ptr(target), _ptr(draft), _ROW_TYPES[target.dtype], seqs, n_max, vocab, _ptr(tokens), _ptr(n_drafts),
                                  _ptr(u_accept), _ptr(u_sample), _ptr(new), _ptr(accepted), _stream(stream, dev))
    if st != 0:
        raise SisoError(st, "siso_verify_drafts", L.siso_last_cuda_error().decode() if st == 7 else "")
    return new, accepted
