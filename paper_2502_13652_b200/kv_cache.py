"""The paged key/value cache and the rules on logits: ctypes layer over the calls of include/c2t.h that need no context.

As in `binding`, arguments are only marshalled; tensors are the caller's, work goes to the current stream of the tensors'
device unless a stream is given, and nothing synchronises.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from .binding import BF16, EINVAL, F32, _check, _stream, lib

F16 = 2
ST_NO_PAGE, ST_BAD_PAGE = 32, 64


class c2t_cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "batch", "layers", "kv_heads", "head_dim", "page_size", "n_pages", "max_pages")] + \
               [("k_dev", C.c_void_p), ("v_dev", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("layer_stride", "page_stride", "token_stride", "head_stride")] + \
               [(n, C.c_void_p) for n in ("table_dev", "held_dev", "refs_dev", "status_dev")]


class c2t_attention(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("layer", "q_heads", "max_queries")] + [("q_dev", C.c_void_p), ("out_dev", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("q_seq_stride", "q_token_stride", "q_head_stride", "out_seq_stride", "out_token_stride",
                                         "out_head_stride")] + \
               [(n, C.c_void_p) for n in ("lse_dev", "n_queries_dev", "prefix_len_dev", "mask_bits_dev")] + \
               [("mask_words", C.c_int32), ("position_ids_dev", C.c_void_p), ("window", C.c_int32), ("sinks", C.c_int32),
                ("scale", C.c_float)]


class c2t_logit_rules(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "batch", "rows", "vocab")] + [("in_dev", C.c_void_p), ("out_dev", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("in_seq_stride", "in_row_stride", "out_seq_stride", "out_row_stride")] + \
               [("n_rows_dev", C.c_void_p), ("counts_dev", C.c_void_p), ("counts_stride", C.c_int64)] + \
               [(n, C.c_void_p) for n in ("repetition_dev", "frequency_dev", "presence_dev", "bias_dev")] + \
               [("bias_stride", C.c_int64), ("allowed_dev", C.c_void_p), ("allowed_seq_stride", C.c_int64),
                ("allowed_row_stride", C.c_int64), ("nodes", C.c_int32)] + \
               [(n, C.c_void_p) for n in ("node_token_dev", "node_parent_dev", "row_node_dev")]


_ready = False


def _calls() -> C.CDLL:
    """The library, with the argument types of the calls below."""
    global _ready
    L = lib()
    if not _ready:
        cache, ptr, i32, i64 = C.POINTER(c2t_cache), C.c_void_p, C.c_int32, C.c_int64
        for name, args in (("c2t_cache_reserve", [cache, ptr, ptr]), ("c2t_cache_release", [cache, ptr, ptr]),
                           ("c2t_cache_fork", [cache, ptr, ptr, ptr, ptr]),
                           ("c2t_cache_append", [cache, i32, ptr, ptr, i32, i64, i64, i64, ptr, ptr, ptr]),
                           ("c2t_cache_compact", [cache, ptr, ptr, ptr, i32, ptr, ptr]),
                           ("c2t_verify_attention", [cache, C.POINTER(c2t_attention), ptr, C.c_size_t, ptr]),
                           ("c2t_penalize_logits", [C.POINTER(c2t_logit_rules), ptr]),
                           ("c2t_count_tokens", [ptr, i64, i32, i32, ptr, i32, ptr, i32, ptr, i32, i32, i32, ptr])):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = args
        L.c2t_verify_attention_workspace_bytes.restype = C.c_size_t
        L.c2t_verify_attention_workspace_bytes.argtypes = [cache, i32, i32]
        _ready = True
    return L


# The calls are short on the device, so their arguments are marshalled with as few steps as the checks allow: the structures of a call are
# packed in one step (native alignment gives C's layout, "0P" the padding at its end, which the library copies too; a test compares it with
# the ctypes structures above).
_ATTENTION = struct.Struct("@iiiPPqqqqqqPPPPiPiif0P")
_RULES = struct.Struct("@iiiiPPqqqqPPqPPPPqPqqiPPP0P")
_int32, _float32, _int64 = torch.int32, torch.float32, torch.int64


def _ints(t: Optional[torch.Tensor], n: int, device: int) -> int:
    """Pointer of a contiguous int32 tensor of n elements on CUDA device `device`; 0 for None."""
    if t is None:
        return 0
    assert t.dtype is _int32 and t.get_device() == device and t.numel() == n and t.is_contiguous()
    return t.data_ptr()


def _device_call(device: int, call, *args) -> int:
    """call(*args) with `device` current."""
    if torch._C._cuda_getDevice() == device:
        return call(*args)
    with torch.cuda.device(device):
        return call(*args)


def _stream_on(device: int, stream) -> int:
    """Handle of a stream, of the device's current one by default."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


class KVCache:
    """A `c2t_cache` over the caller's tensors, and the workspace of its attention calls.

    k, v: [layers, n_pages, page_size, kv_heads, head_dim], bfloat16 or float16, equal strides, last dimension contiguous (any
    order of the others: `permute` a pool that is laid out head by head).  table: [batch, max_pages] int32, held: [batch] int32, refs:
    [n_pages] int32; `new_state` makes them for an empty cache.  q_heads, max_queries: the largest attention call that will
    be made; without them the cache has no workspace and its other calls work.  One thread at a time makes calls, as on a context.
    status and workspace are made on the stream that is current here: a call on another one waits for it first, as for the caller's own tensors, and the
    object outlives the work and the graphs that use it.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, held: torch.Tensor, refs: torch.Tensor,
                 q_heads: int = 0, max_queries: int = 0):
        assert k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.device == v.device
        assert k.is_cuda and k.dtype in (torch.bfloat16, torch.float16) and k.stride(4) == 1
        self.layers, self.n_pages, self.page_size, self.kv_heads, self.head_dim = k.shape
        assert table.dim() == 2
        self.B, self.max_pages = table.shape
        self.device = k.device
        self._dev = k.get_device()
        self.k, self.v, self.table, self.held, self.refs = k, v, table, held, refs
        self.status = torch.zeros(self.B, dtype=torch.int32, device=self.device)
        self._c = c2t_cache(BF16 if k.dtype == torch.bfloat16 else F16, self.B, self.layers, self.kv_heads, self.head_dim,
                            self.page_size, self.n_pages, self.max_pages, k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                            k.stride(2), k.stride(3), _ints(table, self.B * self.max_pages, self._dev), _ints(held, self.B, self._dev),
                            _ints(refs, self.n_pages, self._dev), self.status.data_ptr())
        self._ref = C.byref(self._c)
        self._calls = _calls()
        self._attention = C.create_string_buffer(_ATTENTION.size)
        self._attention_at = C.cast(self._attention, C.POINTER(c2t_attention))
        self.q_heads, self.max_queries, self.workspace, self._workspace = q_heads, max_queries, None, (None, 0)
        if q_heads:
            nbytes = self._calls.c2t_verify_attention_workspace_bytes(self._ref, q_heads, max_queries)
            if nbytes == 0:
                _check(EINVAL, "c2t_verify_attention_workspace_bytes")
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            self._workspace = ((self.workspace.data_ptr() + 255) & ~255, nbytes)

    @staticmethod
    def new_state(batch: int, max_pages: int, n_pages: int, device="cuda"):
        """table, held and refs of an empty cache."""
        i32 = dict(dtype=torch.int32, device=device)
        return torch.full((batch, max_pages), -1, **i32), torch.zeros(batch, **i32), torch.zeros(n_pages, **i32)

    def _call(self, name: str, *args, stream=None) -> None:
        rc = _device_call(self._dev, getattr(self._calls, name), self._ref, *args, _stream_on(self._dev, stream))
        if rc:
            _check(rc, name)

    def c2t_cache_reserve(self, length: torch.Tensor, stream=None) -> None:
        self._call("c2t_cache_reserve", _ints(length, self.B, self._dev), stream=stream)

    def c2t_cache_release(self, keep: torch.Tensor, stream=None) -> None:
        self._call("c2t_cache_release", _ints(keep, self.B, self._dev), stream=stream)

    def c2t_cache_fork(self, src: torch.Tensor, length: torch.Tensor, forked: torch.Tensor, stream=None) -> None:
        B, dev = self.B, self._dev
        self._call("c2t_cache_fork", _ints(src, B, dev), _ints(length, B, dev), _ints(forked, B, dev), stream=stream)

    def c2t_cache_append(self, layer: int, k_new: torch.Tensor, v_new: torch.Tensor, start: torch.Tensor, count: torch.Tensor,
                         stream=None) -> None:
        """k_new, v_new: [B, max_new, kv_heads, head_dim] of the cache's dtype, equal strides, last dimension contiguous."""
        B, dev = self.B, self._dev
        shape, strides = k_new.shape, k_new.stride()
        assert shape == v_new.shape and strides == v_new.stride() and k_new.dtype is v_new.dtype is self.k.dtype
        assert len(shape) == 4 and k_new.get_device() == v_new.get_device() == dev and strides[3] == 1
        assert shape[0] == B and shape[2] == self.kv_heads and shape[3] == self.head_dim
        self._call("c2t_cache_append", layer, k_new.data_ptr(), v_new.data_ptr(), shape[1], strides[0], strides[1], strides[2],
                   _ints(start, B, dev), _ints(count, B, dev), stream=stream)

    def c2t_cache_compact(self, prefix_len: torch.Tensor, accept_len: torch.Tensor, path: torch.Tensor,
                          new_len: Optional[torch.Tensor] = None, stream=None) -> None:
        """path: [B, D + 1] as c2t_accept writes it."""
        B, dev = self.B, self._dev
        assert path.dim() == 2
        width = path.shape[1]
        self._call("c2t_cache_compact", _ints(prefix_len, B, dev), _ints(accept_len, B, dev), _ints(path, B * width, dev), width,
                   _ints(new_len, B, dev), stream=stream)

    def c2t_verify_attention(self, layer: int, q: torch.Tensor, out: torch.Tensor, n_queries: torch.Tensor, prefix_len: torch.Tensor,
                             mask_bits: Optional[torch.Tensor] = None, position_ids: Optional[torch.Tensor] = None, window: int = 0,
                             sinks: int = 0, scale: Optional[float] = None, lse: Optional[torch.Tensor] = None, stream=None) -> None:
        """q, out: [B, Nq, q_heads, head_dim] of the cache's dtype, last dimension contiguous; mask_bits: [B, Nq, W] int64 (the raw
        bits), None: causal; position_ids: [B, Nq] int32; lse: [B, Nq, q_heads] float32.  scale defaults to head_dim ** -0.5."""
        B, dev = self.B, self._dev
        shape, qs, os = q.shape, q.stride(), out.stride()
        assert len(shape) == 4 and shape == out.shape and q.dtype is out.dtype is self.k.dtype and q.get_device() == out.get_device() == dev
        assert shape[0] == B and shape[3] == self.head_dim and qs[3] == os[3] == 1
        Nq, heads = shape[1], shape[2]
        words = bits = 0
        if mask_bits is not None:
            assert mask_bits.dtype is _int64 and mask_bits.get_device() == dev and mask_bits.is_contiguous()
            assert mask_bits.dim() == 3 and mask_bits.shape[0] == B and mask_bits.shape[1] == Nq
            bits, words = mask_bits.data_ptr(), mask_bits.shape[2]
        lse_at = 0
        if lse is not None:
            assert lse.dtype is _float32 and lse.get_device() == dev and lse.is_contiguous() and lse.shape == (B, Nq, heads)
            lse_at = lse.data_ptr()
        _ATTENTION.pack_into(self._attention, 0, layer, heads, Nq, q.data_ptr(), out.data_ptr(), qs[0], qs[1], qs[2], os[0], os[1], os[2],
                             lse_at, _ints(n_queries, B, dev), _ints(prefix_len, B, dev), bits, words, _ints(position_ids, B * Nq, dev),
                             window, sinks, self.head_dim ** -0.5 if scale is None else scale)
        self._call("c2t_verify_attention", self._attention_at, *self._workspace, stream=stream)


def _floats(t: Optional[torch.Tensor], n: int, device: int) -> int:
    if t is None:
        return 0
    assert t.dtype is _float32 and t.get_device() == device and t.numel() == n and t.is_contiguous()
    return t.data_ptr()


def c2t_penalize_logits(logits: torch.Tensor, out: torch.Tensor, n_rows: Optional[torch.Tensor] = None,
                        counts: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                        frequency: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None,
                        bias: Optional[torch.Tensor] = None, allowed: Optional[torch.Tensor] = None,
                        node_token: Optional[torch.Tensor] = None, node_parent: Optional[torch.Tensor] = None,
                        row_node: Optional[torch.Tensor] = None, stream=None) -> None:
    """logits, out: [B, rows, V] CUDA tensors, float32 or bfloat16, last dimension contiguous (the same one for in place); counts: [B, V]
    int32; repetition, frequency, presence: [B] float32; bias: [V] or [B, V] float32; allowed: [B, rows, words] or [B, words] int32 (raw
    bits, the latter for all rows of a sequence); node_token, node_parent: [B, N] int32; row_node: [B, rows] int32."""
    dev = logits.get_device()
    shape, ins, outs, dtype = logits.shape, logits.stride(), out.stride(), logits.dtype
    assert logits.is_cuda and len(shape) == 3 and shape == out.shape and dtype is out.dtype and out.get_device() == dev
    assert (dtype is torch.bfloat16 or dtype is _float32) and ins[2] == 1 and outs[2] == 1
    B, R, V = shape
    counts_at = counts_stride = bias_at = bias_stride = allowed_at = allowed_seq = allowed_row = nodes = 0
    if counts is not None:
        assert counts.dtype is _int32 and counts.get_device() == dev and counts.shape == (B, V) and counts.stride(1) == 1
        counts_at, counts_stride = counts.data_ptr(), counts.stride(0)
    if bias is not None:
        assert bias.dtype is _float32 and bias.get_device() == dev and bias.stride(-1) == 1 and bias.shape in ((V,), (B, V))
        bias_at, bias_stride = bias.data_ptr(), bias.stride(0) if bias.dim() == 2 else 0
    if allowed is not None:
        assert allowed.dtype is _int32 and allowed.get_device() == dev and allowed.stride(-1) == 1
        assert allowed.shape[0] == B and allowed.shape[-1] >= (V + 31) // 32
        assert allowed.dim() == 2 or (allowed.dim() == 3 and allowed.shape[1] == R)
        allowed_at, allowed_seq, allowed_row = allowed.data_ptr(), allowed.stride(0), allowed.stride(1) if allowed.dim() == 3 else 0
    if node_token is not None:
        assert node_token.dim() == 2 and node_parent is not None
        nodes = node_token.shape[1]
    rules = C.create_string_buffer(_RULES.size)
    _RULES.pack_into(rules, 0, BF16 if dtype is torch.bfloat16 else F32, B, R, V, logits.data_ptr(), out.data_ptr(), ins[0], ins[1], outs[0],
                     outs[1], _ints(n_rows, B, dev), counts_at, counts_stride, _floats(repetition, B, dev), _floats(frequency, B, dev),
                     _floats(presence, B, dev), bias_at, bias_stride, allowed_at, allowed_seq, allowed_row, nodes,
                     _ints(node_token, B * nodes, dev), _ints(node_parent, B * nodes, dev), _ints(row_node, B * R, dev))
    rc = _device_call(dev, _calls().c2t_penalize_logits, C.cast(rules, C.POINTER(c2t_logit_rules)), _stream_on(dev, stream))
    if rc:
        _check(rc, "c2t_penalize_logits")


def c2t_count_tokens(counts: torch.Tensor, tokens: torch.Tensor, n: torch.Tensor, index: Optional[torch.Tensor] = None,
                     plus_one: bool = False, delta: int = 1, stream=None) -> None:
    """counts: [B, V] int32; tokens: [B, N] int32; n: [B] int32; index: [B, width] int32.  With c2t_build_verify's tokens and
    c2t_accept's accept_len (plus_one: the root counts too) and path, the accepted tokens enter the history."""
    dev = counts.get_device()
    assert counts.is_cuda and counts.dtype is _int32 and counts.dim() == 2 and counts.stride(1) == 1
    B, V = counts.shape
    assert tokens.dim() == 2 and (index is None or index.dim() == 2)
    N = tokens.shape[1]
    width = N if index is None else index.shape[1]
    rc = _device_call(dev, _calls().c2t_count_tokens, counts.data_ptr(), counts.stride(0), B, V, _ints(tokens, B * N, dev), N,
                      _ints(index, B * width, dev), width, _ints(n, B, dev), int(plus_one), width, delta, _stream_on(dev, stream))
    if rc:
        _check(rc, "c2t_count_tokens")
