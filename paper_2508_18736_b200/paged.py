"""The language model's side of a cache miss: a paged key/value cache that is quantised as it is written, the attention of new
tokens over it, the verification of drafted tokens (a near hit's stored answer, or a drafting model's), the same for trees of drafts (several near
hits), and eviction from the cache by the weight that attention gives.  Argument marshalling only; names and rules follow include/siso.h.

A call with `stream` runs on that stream as a whole, as under torch.cuda.stream: the copies of arguments that are not contiguous, the
kernels, and the outputs, whose memory is that stream's.  The arguments have to be ready there and to live until it is done with them."""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from .binding import SisoError, _ALLOC_FN, _FREE_FN, _Allocator, load_library

ATTN_CAUSAL = 1
_CACHE_TYPES = {torch.bfloat16: 1, torch.float8_e4m3fn: 2, torch.int8: 3}
_ROW_TYPES = {torch.float32: 0, torch.bfloat16: 1}


_raw_stream = torch._C._cuda_getCurrentRawStream        # the current stream's handle, without building a Stream object


def _on(stream, index: int):
    """The context of `stream`, which has to be one of device `index`."""
    if stream.device_index != index:
        raise ValueError(f"stream must be one of cuda:{index}")
    return torch.cuda.stream(stream)


class _KvConfig(ctypes.Structure):
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("d_k_exp", ctypes.c_void_p), ("d_v_exp", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("stride_layer", ctypes.c_int64), ("stride_page", ctypes.c_int64),
                ("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("n_layers", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("allocator", _Allocator)]


# siso_attention_t: 6 pointers, 6 int64, 6 int32, uint32, float.  Packed by hand: a call costs the host a few microseconds in all
_ATTENTION = struct.Struct("@6P6q6iIf")
_WEIGHTS = struct.Struct("@6P4q5iIff")          # siso_weights_t: 6 pointers, 4 int64, 5 int32, uint32, 2 floats


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
        self._dev, self._index = k.device, k.get_device()
        blocks, dev = {}, k.device
        self._blocks = blocks

        # scratch from the pool of the stream it is first used on.  (The callbacks hold no reference to the handle: it has to go, and
        # give its pages back, with the last reference to it)
        def _alloc(nbytes, stream, ctx):
            try:
                with torch.cuda.device(dev):
                    if stream:
                        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=dev)):
                            t = torch.empty(int(nbytes), dtype=torch.uint8, device=dev)
                    else:
                        t = torch.empty(int(nbytes), dtype=torch.uint8, device=dev)
            except Exception:                     # out of memory -> NULL -> SISO_ERR_OOM
                return None
            blocks[t.data_ptr()] = t
            return t.data_ptr()

        def _free(ptr, ctx):
            blocks.pop(ptr, None)

        self._alloc_cb, self._free_cb = _ALLOC_FN(_alloc), _FREE_FN(_free)
        cfg = _KvConfig(k.data_ptr(), v.data_ptr(), None if k_exp is None else k_exp.data_ptr(), None if v_exp is None else v_exp.data_ptr(),
                        pages, k.stride(0), k.stride(1), k.stride(2), k.stride(3), layers, tokens, heads, dim, _CACHE_TYPES[k.dtype],
                        k.device.index, _Allocator(self._alloc_cb, self._free_cb, None))
        h = ctypes.c_void_p()
        st = self._lib.siso_kv_create(ctypes.byref(h), ctypes.byref(cfg))
        self._h = h if st == 0 else None
        self._check(st, "siso_kv_create")
        self._args = ctypes.create_string_buffer(_ATTENTION.size)
        self._default_scale = dim ** -0.5
        self._none = {t: torch.empty(0, dtype=t, device=self._dev) for t in _ROW_TYPES}

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
        if t.dtype not in _ROW_TYPES or t.get_device() != self._index or t.shape != (n, self.n_kv_heads, self.head_dim):
            raise ValueError(f"{name} must be a [{n}, {self.n_kv_heads}, {self.head_dim}] float32 or bfloat16 tensor on {self._dev}")
        return t if t.stride(2) == 1 else t.contiguous()

    def _slots(self, slots: torch.Tensor) -> torch.Tensor:
        if slots.dtype is not torch.int64 or slots.dim() != 1 or slots.get_device() != self._index:
            raise ValueError(f"slots must be a one-dimensional int64 tensor on {self._dev}")
        return slots if slots.is_contiguous() else slots.contiguous()

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, layer: int = 0, stream=None) -> None:
        """Rows k, v [n, kv heads, head dim] (fp32 or bf16) into `slots` [n] = page * page size + token (-1: skipped)."""
        if stream is not None:
            with _on(stream, self._index):
                return self.write(k, v, slots, layer)
        slots = self._slots(slots)
        n = slots.shape[0]
        k, v = self._rows(k, n, "k"), self._rows(v, n, "v")
        if k.dtype is not v.dtype:
            raise ValueError("k and v must have the same type")
        strides = k.stride()
        if strides != v.stride():
            k, v = k.contiguous(), v.contiguous()
            strides = k.stride()
        st = self._lib.siso_kv_write(self._h, layer, k.data_ptr(), v.data_ptr(), _ROW_TYPES[k.dtype], n, strides[0], strides[1],
                                     slots.data_ptr(), _raw_stream(self._index))
        if st:
            self._check(st, "siso_kv_write")

    def read(self, slots: torch.Tensor, layer: int = 0, dtype: torch.dtype = torch.bfloat16, stream=None, out=None
             ) -> Tuple[torch.Tensor, torch.Tensor]:
        """The rows of `slots` as (k, v) [n, kv heads, head dim] of `dtype` (float32 or bfloat16); zeros for slots outside the pool."""
        if stream is not None:
            with _on(stream, self._index):
                return self.read(slots, layer, dtype, out=out)
        slots = self._slots(slots)
        n = slots.shape[0]
        if out is None:
            if dtype not in _ROW_TYPES:
                raise ValueError("dtype must be float32 or bfloat16")
            k = self._none[dtype].new_empty((n, self.n_kv_heads, self.head_dim))
            v = torch.empty_like(k)
        else:
            k, v = out
            if self._rows(k, n, "out k") is not k or self._rows(v, n, "out v") is not v or k.stride() != v.stride() or k.dtype is not v.dtype:
                raise ValueError("outputs must have contiguous rows, the same strides and the same type")
        strides = k.stride()
        st = self._lib.siso_kv_read(self._h, layer, k.data_ptr(), v.data_ptr(), _ROW_TYPES[k.dtype], n, strides[0], strides[1],
                                    slots.data_ptr(), _raw_stream(self._index))
        if st:
            self._check(st, "siso_kv_read")
        return k, v

    def attention(self, q: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, max_q: int, layer: int = 0,
                  scale: Optional[float] = None, causal: bool = True, window: int = 0, want_lse: bool = False, stream=None,
                  out: Optional[torch.Tensor] = None):
        """q [n, heads, head dim] bf16: the queries of all sequences one after the other, sequence b's from cu_q[b] on (int32
        [seqs + 1]); kv_len int32 [seqs]: tokens in all, the new ones included (already written); pages int32 [seqs, max pages].
        Rows of q that no sequence covers leave theirs of the outputs as they were (of new outputs: anything).  Returns out [n, heads, head dim], or (out, lse [n, heads] fp32) with want_lse."""
        if stream is not None:
            with _on(stream, self._index):
                return self.attention(q, cu_q, kv_len, pages, max_q, layer, scale, causal, window, want_lse, out=out)
        return self._attend(None, q, cu_q, kv_len, pages, max_q, layer, scale, causal, window, want_lse, out)

    def tree_attention(self, q: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, mask: torch.Tensor, max_q: int,
                       layer: int = 0, scale: Optional[float] = None, window: int = 0, want_lse: bool = False, stream=None,
                       out: Optional[torch.Tensor] = None):
        """attention() of new tokens that are nodes of trees: each sees the tokens before the new ones and, of the new ones, those of its row of
        mask int32 [n, words] (bit j % 32 of word j // 32: node j of its sequence; tree_mask() gives the ancestors).  A window counts from
        a node's place below the tokens before the new ones, and limits only those; of the new ones the mask alone decides."""
        if stream is not None:
            with _on(stream, self._index):
                return self.tree_attention(q, cu_q, kv_len, pages, mask, max_q, layer, scale, window, want_lse, out=out)
        if mask.dtype is not torch.int32 or mask.dim() != 2 or mask.shape[0] != q.shape[0] or mask.shape[1] < 1 or mask.get_device() != self._index:
            raise ValueError(f"mask must be an int32 [n, words] tensor on {self._dev}")
        return self._attend(mask if mask.stride(1) == 1 else mask.contiguous(), q, cu_q, kv_len, pages, max_q, layer, scale, True, window, want_lse, out)

    def _attend(self, mask, q, cu_q, kv_len, pages, max_q, layer, scale, causal, window, want_lse, out):
        index, i32 = self._index, torch.int32
        shape = q.shape
        if q.dtype is not torch.bfloat16 or len(shape) != 3 or shape[2] != self.head_dim or q.get_device() != index:
            raise ValueError(f"q must be a [n, heads, {self.head_dim}] bfloat16 tensor on {self._dev}")
        if cu_q.dtype is not i32 or kv_len.dtype is not i32 or pages.dtype is not i32 or cu_q.get_device() != index or kv_len.get_device() != index \
                or pages.get_device() != index:
            raise ValueError(f"cu_q, kv_len and pages must be int32 tensors on {self._dev}")
        n, heads, dim = shape
        table = pages.shape
        seqs = kv_len.numel()
        if cu_q.dim() != 1 or kv_len.dim() != 1 or cu_q.numel() != seqs + 1 or len(table) != 2 or table[0] != seqs:
            raise ValueError("cu_q must be [seqs + 1], kv_len [seqs], pages [seqs, max pages]")
        sq = q.stride()
        if sq[2] != 1:
            q = q.contiguous()
            sq = q.stride()
        if pages.stride(1) != 1:
            pages = pages.contiguous()
        if not cu_q.is_contiguous():
            cu_q = cu_q.contiguous()
        if not kv_len.is_contiguous():
            kv_len = kv_len.contiguous()
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.dtype is not torch.bfloat16 or out.shape != shape or out.get_device() != index or out.stride(2) != 1:
            raise ValueError("out must be a bfloat16 tensor like q with contiguous rows")
        so = out.stride()
        lse = torch.empty((n, heads), dtype=torch.float32, device=self._dev) if want_lse else None
        _ATTENTION.pack_into(self._args, 0, q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else 0, cu_q.data_ptr(), kv_len.data_ptr(),
                             pages.data_ptr(), sq[0], sq[1], so[0], so[1], pages.stride(0), n, seqs, max_q, table[1], heads, layer, window,
                             ATTN_CAUSAL if causal else 0, self._default_scale if scale is None else scale)
        if mask is None:
            st = self._lib.siso_kv_attention(self._h, self._args, _raw_stream(index))
            if st:
                self._check(st, "siso_kv_attention")
        else:
            st = self._lib.siso_kv_tree_attention(self._h, self._args, mask.data_ptr(), mask.shape[1], mask.stride(0), _raw_stream(index))
            if st:
                self._check(st, "siso_kv_tree_attention")
        return (out, lse) if want_lse else out

    def _sequences(self, kv_len, pages, cu_q=None):
        """(kv_len, pages, cu_q) as the library takes them: contiguous, rows of pages at any stride."""
        i32, index = torch.int32, self._index
        if kv_len.dtype is not i32 or pages.dtype is not i32 or kv_len.get_device() != index or pages.get_device() != index or \
                (cu_q is not None and (cu_q.dtype is not i32 or cu_q.get_device() != index)):
            raise ValueError(f"cu_q, kv_len and pages must be int32 tensors on {self._dev}")
        if kv_len.dim() != 1 or pages.dim() != 2 or pages.shape[0] != kv_len.numel() or \
                (cu_q is not None and (cu_q.dim() != 1 or cu_q.numel() != kv_len.numel() + 1)):
            raise ValueError("cu_q must be [seqs + 1], kv_len [seqs], pages [seqs, max pages]")
        if pages.stride(1) != 1:
            pages = pages.contiguous()
        if not kv_len.is_contiguous():
            kv_len = kv_len.contiguous()
        if cu_q is not None and not cu_q.is_contiguous():
            cu_q = cu_q.contiguous()
        return kv_len, pages, cu_q

    def _weights(self, weights):
        if weights.dtype is not torch.float32 or weights.get_device() != self._index or not weights.is_contiguous() or \
                weights.shape != (self.n_layers, self.n_pages, self.n_kv_heads, self.page_size):
            raise ValueError(f"weights must be a contiguous float32 [{self.n_layers}, {self.n_pages}, {self.n_kv_heads}, {self.page_size}] tensor "
                             f"on {self._dev}")

    def new_weights(self) -> torch.Tensor:
        """A number for each cached row, zero: what add_weights() adds to (it wants them to begin on a 16-byte boundary, as these do) and evict() goes by."""
        return torch.zeros((self.n_layers, self.n_pages, self.n_kv_heads, self.page_size), dtype=torch.float32, device=self._dev)

    def keep_path(self, path: torch.Tensor, accepted: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, stream=None
                  ) -> torch.Tensor:
        """Moves the rows (all layers) of the nodes path [seqs, longest], the first accepted [seqs] of each, behind node 0 of their sequence (rows, not weights:
        node 0 and the path's are new tokens to add_weights(); their queries and lse, gathered in the path's order, are those of a causal chunk).
        cu_q, kv_len, pages as tree_attention() had them.  Returns the tokens that the sequences have now, int32 [seqs]."""
        if stream is not None:
            with _on(stream, self._index):
                return self.keep_path(path, accepted, cu_q, kv_len, pages)
        kv_len, pages, cu_q = self._sequences(kv_len, pages, cu_q)
        seqs, i32, index = kv_len.numel(), torch.int32, self._index
        if path.dtype is not i32 or path.dim() != 2 or path.shape[0] != seqs or path.get_device() != index or accepted.dtype is not i32 or \
                accepted.shape != (seqs,) or accepted.get_device() != index:
            raise ValueError(f"path must be [seqs, longest] and accepted [seqs], int32 on {self._dev}")
        if not path.is_contiguous():
            path = path.contiguous()
        if not accepted.is_contiguous():
            accepted = accepted.contiguous()
        new_len = torch.empty_like(kv_len)
        st = self._lib.siso_kv_keep_path(self._h, path.data_ptr(), accepted.data_ptr(), path.shape[1], cu_q.data_ptr(), kv_len.data_ptr(), pages.data_ptr(),
                                         pages.stride(0), pages.shape[1], seqs, new_len.data_ptr(), _raw_stream(index))
        if st:
            self._check(st, "siso_kv_keep_path")
        return new_len

    def add_weights(self, weights: torch.Tensor, q: torch.Tensor, lse: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor,
                    max_q: int, layer: int = 0, scale: Optional[float] = None, causal: bool = True, decay: float = 1.0, stream=None,
                    n_new: Optional[torch.Tensor] = None) -> None:
        """Adds to weights (see new_weights()) what the queries q [n, heads, head dim] bf16 give each token that they see, summed over the
        queries and the heads of a kv head: their probabilities, from lse [n, heads] as attention(want_lse=True) returned it for the same queries and
        `causal`, without a window (tokens before it would be weighed too, by numbers that may be above 1); a tree's queries are weighed once their path is kept (see
        keep_path()), as before that each would weigh its sisters.  What was there counts
        `decay` times (0: not at all, whatever it is); the new tokens start from zero: a sequence's last ones, as many as it has queries, or n_new int32 [seqs] of
        them.  For the last queries of a longer chunk alone pass them with their own cu_q and the chunk's length as n_new, for the first query behind a
        path that keep_path() kept the path's tokens and the query's: until a call has counted a token as new, its place may hold an evicted token's weight, a
        draft's, or that of a page's last owner.  Sequences of one call that have queries must not share pages, though attention() lets them: each would write the
        shared tokens' weights without the other's."""
        if stream is not None:
            with _on(stream, self._index):
                return self.add_weights(weights, q, lse, cu_q, kv_len, pages, max_q, layer, scale, causal, decay, n_new=n_new)
        index = self._index
        shape = q.shape
        if q.dtype is not torch.bfloat16 or len(shape) != 3 or shape[2] != self.head_dim or q.get_device() != index:
            raise ValueError(f"q must be a [n, heads, {self.head_dim}] bfloat16 tensor on {self._dev}")
        if lse.dtype is not torch.float32 or lse.shape != shape[:2] or lse.get_device() != index:
            raise ValueError(f"lse must be a [n, heads] float32 tensor on {self._dev}")
        self._weights(weights)
        kv_len, pages, cu_q = self._sequences(kv_len, pages, cu_q)
        if q.stride(2) != 1 or 0 in q.stride():
            q = q.contiguous()
        if not lse.is_contiguous():
            lse = lse.contiguous()
        if n_new is not None:
            if n_new.dtype is not torch.int32 or n_new.shape != kv_len.shape or n_new.get_device() != index:
                raise ValueError(f"n_new must be an int32 [{kv_len.numel()}] tensor on {self._dev}")
            if not n_new.is_contiguous():
                n_new = n_new.contiguous()
        sq = q.stride()
        _WEIGHTS.pack_into(self._args, 0, q.data_ptr(), lse.data_ptr(), weights.data_ptr(), cu_q.data_ptr(), kv_len.data_ptr(), pages.data_ptr(), sq[0], sq[1],
                           pages.stride(0), shape[0], kv_len.numel(), max_q, pages.shape[1], shape[1], layer, ATTN_CAUSAL if causal else 0,
                           self._default_scale if scale is None else scale, decay)
        if n_new is None:
            st = self._lib.siso_kv_add_weights(self._h, self._args, _raw_stream(index))
        else:
            st = self._lib.siso_kv_add_weights_new(self._h, self._args, n_new.data_ptr(), _raw_stream(index))
        if st:
            self._check(st, "siso_kv_add_weights")

    def evict(self, weights: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, budget: int, recent: int, out_pages: Optional[torch.Tensor] = None,
              stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Cuts every sequence down to `budget` tokens, for each layer and kv head by itself: the last `recent` stay and the heaviest others (ties: the
        earlier one), moved in order to the front of their pages, or of out_pages [seqs, max pages] (each the same as in pages at that index, or not otherwise in
        use).  Places that nothing is moved to keep what they held, weights among it: tokens written there are new ones to add_weights().  Returns (tokens now int32 [seqs], which places stayed int32 [layers, seqs, kv heads, budget], then -1)."""
        if stream is not None:
            with _on(stream, self._index):
                return self.evict(weights, kv_len, pages, budget, recent, out_pages)
        self._weights(weights)
        kv_len, pages, _ = self._sequences(kv_len, pages)
        out_pages = pages if out_pages is None else self._sequences(kv_len, out_pages)[1]
        seqs = kv_len.numel()
        if budget < 1 or not 0 <= recent <= budget:
            raise ValueError("budget must be at least 1 and recent from 0 to budget")
        new_len = torch.empty_like(kv_len)
        kept = torch.empty((self.n_layers, seqs, self.n_kv_heads, budget), dtype=torch.int32, device=self._dev)
        st = self._lib.siso_kv_evict(self._h, weights.data_ptr(), kv_len.data_ptr(), pages.data_ptr(), pages.stride(0), pages.shape[1], out_pages.data_ptr(),
                                     out_pages.stride(0), out_pages.shape[1], seqs, budget, recent, new_len.data_ptr(), kept.data_ptr(),
                                     _raw_stream(self._index))
        if st:
            self._check(st, "siso_kv_evict")
        return new_len, kept

    def sync_status(self, stream=None) -> int:
        """Synchronise and return the handle's device status word (0 = clear); it is cleared by the call."""
        return int(self._lib.siso_kv_sync_status(self._h, _raw_stream(self._index) if stream is None else stream.cuda_stream))

    def selftest_wait_timeout(self, stream=None) -> None:
        """Lets one bounded wait of the attention kernels run out (see siso_kv_selftest_wait_timeout)."""
        self._check(self._lib.siso_kv_selftest_wait_timeout(self._h, _raw_stream(self._index) if stream is None else stream.cuda_stream),
                    "siso_kv_selftest_wait_timeout")

    def check_status(self, stream=None) -> None:
        st = self.sync_status(stream)
        if st != 0:
            raise SisoError(st, "device status")


def verify_drafts(target: torch.Tensor, draft: Optional[torch.Tensor], tokens: torch.Tensor, n_drafts: Optional[torch.Tensor],
                  u_accept: torch.Tensor, u_sample: torch.Tensor, stream=None, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """target [seqs, drafts + 1, vocab] and draft [seqs, drafts, vocab] (or None: certain drafts) probabilities, fp32 or bf16;
    tokens int32 [seqs, drafts]; n_drafts int32 [seqs] or None (all); u_accept [seqs, drafts], u_sample [seqs] fp32 in [0, 1).
    Returns (tokens out int32 [seqs, drafts + 1]: those that stand, one drawn, then -1; accepted int32 [seqs])."""
    if stream is not None:
        with _on(stream, target.get_device()):
            return verify_drafts(target, draft, tokens, n_drafts, u_accept, u_sample, out=out)
    shape, i32, f32 = target.shape, torch.int32, torch.float32
    if target.dtype not in _ROW_TYPES or len(shape) != 3 or not target.is_cuda:
        raise ValueError("target must be a [seqs, drafts + 1, vocab] float32 or bfloat16 tensor on a GPU")
    seqs, rows, vocab = shape
    n_max, index = rows - 1, target.get_device()
    if n_max < 0:
        raise ValueError("target needs at least one row per sequence")
    if draft is not None:
        if draft.dtype is not target.dtype or draft.shape != (seqs, n_max, vocab) or draft.get_device() != index:
            raise ValueError("draft must be [seqs, drafts, vocab] of target's type and device")
        if not draft.is_contiguous():
            draft = draft.contiguous()
    if tokens.dtype is not i32 or tokens.shape != (seqs, n_max) or tokens.get_device() != index:
        raise ValueError(f"tokens must be an int32 [{seqs}, {n_max}] tensor on {target.device}")
    if n_drafts is not None and (n_drafts.dtype is not i32 or n_drafts.shape != (seqs,) or n_drafts.get_device() != index):
        raise ValueError(f"n_drafts must be an int32 [{seqs}] tensor on {target.device}")
    if u_accept.dtype is not f32 or u_accept.shape != (seqs, n_max) or u_accept.get_device() != index:
        raise ValueError(f"u_accept must be a float32 [{seqs}, {n_max}] tensor on {target.device}")
    if u_sample.dtype is not f32 or u_sample.shape != (seqs,) or u_sample.get_device() != index:
        raise ValueError(f"u_sample must be a float32 [{seqs}] tensor on {target.device}")
    if not target.is_contiguous():
        target = target.contiguous()
    if not tokens.is_contiguous():
        tokens = tokens.contiguous()
    if not u_accept.is_contiguous():
        u_accept = u_accept.contiguous()
    if not u_sample.is_contiguous():
        u_sample = u_sample.contiguous()
    if n_drafts is not None and not n_drafts.is_contiguous():
        n_drafts = n_drafts.contiguous()
    if out is None:
        new = tokens.new_empty((seqs, rows))
        accepted = tokens.new_empty((seqs,)) if n_drafts is None else torch.empty_like(n_drafts)
    else:
        new, accepted = out
        if new.dtype is not i32 or new.shape != (seqs, rows) or not new.is_contiguous() or accepted.dtype is not i32 or accepted.shape != (seqs,) \
                or not accepted.is_contiguous() or new.get_device() != index or accepted.get_device() != index:
            raise ValueError("out must be contiguous int32 tensors [seqs, drafts + 1] and [seqs] beside target")
    here = torch._C._cuda_getDevice()
    if here != index:
        torch.cuda.set_device(index)
    try:
        st = load_library().siso_verify_drafts(target.data_ptr(), 0 if draft is None else draft.data_ptr(), _ROW_TYPES[target.dtype], seqs, n_max, vocab,
                                               tokens.data_ptr(), 0 if n_drafts is None else n_drafts.data_ptr(), u_accept.data_ptr(),
                                               u_sample.data_ptr(), new.data_ptr(), accepted.data_ptr(),
                                               _raw_stream(index))
    finally:
        if here != index:
            torch.cuda.set_device(here)
    if st:
        raise SisoError(st, "siso_verify_drafts", load_library().siso_last_cuda_error().decode() if st == 7 else "")
    return new, accepted


def _call(index: int, where: str, *args) -> None:
    """An entry point without a handle, on device `index` and its current stream."""
    lib = load_library()
    here = torch._C._cuda_getDevice()
    if here != index:
        torch.cuda.set_device(index)
    try:
        st = getattr(lib, where)(*args, _raw_stream(index))
    finally:
        if here != index:
            torch.cuda.set_device(here)
    if st:
        raise SisoError(st, where, lib.siso_last_cuda_error().decode() if st == 7 else "")


def tree_mask(parents: torch.Tensor, cu_q: torch.Tensor, max_nodes: int, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """parents int32 [n]: for each node of each sequence (from cu_q[b] on, int32 [seqs + 1]) the number of an earlier node of the sequence, anything
    else: none.  Returns (mask int32 [n, words], depth int32 [n]): bit j of a row says that node j is the row's own or above it (max_nodes, the most of one
    sequence, says how many words that takes), and how many are above.  Rows that no sequence covers hold anything."""
    if stream is not None:
        with _on(stream, parents.get_device()):
            return tree_mask(parents, cu_q, max_nodes)
    i32 = torch.int32
    if parents.dtype is not i32 or parents.dim() != 1 or not parents.is_cuda:
        raise ValueError("parents must be a one-dimensional int32 tensor on a GPU")
    if cu_q.dtype is not i32 or cu_q.dim() != 1 or cu_q.numel() < 1 or cu_q.get_device() != parents.get_device():
        raise ValueError(f"cu_q must be an int32 [seqs + 1] tensor on {parents.device}")
    if not parents.is_contiguous():
        parents = parents.contiguous()
    if not cu_q.is_contiguous():
        cu_q = cu_q.contiguous()
    n, words = parents.numel(), max(1, -(-max_nodes // 32))
    mask, depth = parents.new_empty((n, words)), torch.empty_like(parents)
    _call(parents.get_device(), "siso_tree_mask", parents.data_ptr(), cu_q.data_ptr(), n, cu_q.numel() - 1, words, mask.data_ptr(), depth.data_ptr())
    return mask, depth


def verify_tree(target: torch.Tensor, draft: Optional[torch.Tensor], tokens: torch.Tensor, parents: torch.Tensor, cu_q: torch.Tensor, max_path: int,
                u_accept: torch.Tensor, u_sample: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Verification of trees of drafts, nodes of all sequences one after the other (cu_q int32 [seqs + 1]), node 0 of each the last token that stands
    already: target [n, vocab] probabilities of the token after each node, draft [n, vocab] those that a node's children were drawn from, each by itself (None:
    the drafts were certain), fp32 or bf16; tokens, parents int32 [n]; u_accept [n], u_sample [seqs] fp32 in [0, 1).  Children are tried in order.
    Returns (tokens out int32 [seqs, max_path + 1]: those that stand, one drawn, then -1; accepted int32 [seqs]; their nodes int32 [seqs, max_path], then -1)."""
    if stream is not None:
        with _on(stream, target.get_device()):
            return verify_tree(target, draft, tokens, parents, cu_q, max_path, u_accept, u_sample)
    shape, i32, f32 = target.shape, torch.int32, torch.float32
    if target.dtype not in _ROW_TYPES or len(shape) != 2 or not target.is_cuda:
        raise ValueError("target must be a [n, vocab] float32 or bfloat16 tensor on a GPU")
    n, vocab = shape
    index = target.get_device()
    if draft is not None:
        if draft.dtype is not target.dtype or draft.shape != shape or draft.get_device() != index:
            raise ValueError("draft must be [n, vocab] of target's type and device")
        if not draft.is_contiguous():
            draft = draft.contiguous()
    if tokens.dtype is not i32 or parents.dtype is not i32 or tokens.dim() != 1 or parents.dim() != 1 or tokens.numel() != n or parents.numel() != n or \
            tokens.get_device() != index or parents.get_device() != index:
        raise ValueError(f"tokens and parents must be int32 [{n}] tensors on {target.device}")
    if u_accept.dtype is not f32 or u_accept.dim() != 1 or u_accept.numel() != n or u_accept.get_device() != index:
        raise ValueError(f"u_accept must be a float32 [{n}] tensor on {target.device}")
    if u_sample.dtype is not f32 or u_sample.dim() != 1 or u_sample.get_device() != index:
        raise ValueError(f"u_sample must be a float32 [seqs] tensor on {target.device}")
    seqs = u_sample.numel()
    if cu_q.dtype is not i32 or cu_q.dim() != 1 or cu_q.numel() != seqs + 1 or cu_q.get_device() != index:
        raise ValueError(f"cu_q must be an int32 [{seqs + 1}] tensor on {target.device}")
    if max_path < 0:
        raise ValueError("max_path must not be negative")
    if not target.is_contiguous():
        target = target.contiguous()
    if not (tokens.is_contiguous() and parents.is_contiguous() and cu_q.is_contiguous() and u_accept.is_contiguous() and u_sample.is_contiguous()):
        tokens, parents, cu_q, u_accept, u_sample = (t.contiguous() for t in (tokens, parents, cu_q, u_accept, u_sample))
    out, accepted, path = tokens.new_empty((seqs, max_path + 1)), tokens.new_empty((seqs,)), tokens.new_empty((seqs, max_path))
    _call(index, "siso_verify_tree", target.data_ptr(), 0 if draft is None else draft.data_ptr(), _ROW_TYPES[target.dtype], n, seqs, vocab, tokens.data_ptr(),
          parents.data_ptr(), cu_q.data_ptr(), max_path, u_accept.data_ptr(), u_sample.data_ptr(), out.data_ptr(), accepted.data_ptr(), path.data_ptr())
    return out, accepted, path
