"""Python binding of the key/value cache operators (argument marshalling only).

    kv_write(cache, batch, k, v)   -> status         new tokens quantised into their blocks
    kv_read(cache, batch)          -> k, v, status   tokens read back
    kv_attend(cache, batch, q)     -> out, lse, status   attention over the cache

A KvCache is a pool of blocks in 8 bits (its memory may be given, e.g. views of a planned slab); a KvBatch says which
blocks the sequences of a call have, how many tokens they hold and which rows of the call's tensors are theirs.  Its
tensors stay on the device and may be changed there between calls.  All calls are asynchronous on the current (or given)
CUDA stream; what they allocate belongs to that stream.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from .api import Workspace, _check, _ptr

_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}  # mp_dtype


def _tensor(name, t, dtype, shape, device=None):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} is needed, "
                         f"got {t.dtype} {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t


class KvCache:
    """A pool of n_blocks blocks of block_tokens tokens: e4m3 keys and values of n_heads heads of head_dim values, one
    scale for each block and head.  k, v (uint8[n_blocks, n_heads, block_tokens * head_dim], 16-byte aligned) and
    k_scale, v_scale (float32[n_blocks, n_heads]) are allocated unless given; nothing needs to be initialised."""

    def __init__(self, n_blocks: int, block_tokens: int, n_heads: int, head_dim: int, device="cuda", k=None, v=None,
                 k_scale=None, v_scale=None):
        self.n_blocks, self.block_tokens, self.n_heads, self.head_dim = n_blocks, block_tokens, n_heads, head_dim
        if block_tokens % 32 or not 32 <= block_tokens <= 256 or head_dim not in (64, 128) or n_heads < 1:
            raise ValueError("block_tokens is a multiple of 32 up to 256, head_dim 64 or 128, n_heads at least 1")
        shape = (n_blocks, n_heads, block_tokens * head_dim)
        given = [t for t in (k, v, k_scale, v_scale) if t is not None]
        device = given[0].device if given else torch.device(device)

        def make(name, t, dtype, shape):
            if t is None:
                return torch.empty(shape, dtype=dtype, device=device)
            return _tensor(name, t, dtype, shape, device)

        self.k, self.v = make("k", k, torch.uint8, shape), make("v", v, torch.uint8, shape)
        self.k_scale = make("k_scale", k_scale, torch.float32, shape[:2])
        self.v_scale = make("v_scale", v_scale, torch.float32, shape[:2])
        self.device = self.k.device
        self._struct = _lib.MpKvCache(n_blocks, block_tokens, n_heads, head_dim, _ptr(self.k), _ptr(self.v),
                                      _ptr(self.k_scale), _ptr(self.v_scale))
        self._ref = ctypes.byref(self._struct)

    @staticmethod
    def block_bytes(block_tokens: int, n_heads: int, head_dim: int) -> int:
        """Bytes of one block: keys, values and their scales (what a plan counts a request's blocks at)."""
        return 2 * n_heads * (block_tokens * head_dim + 4)


class KvBatch:
    """The sequences of a call.  table int32[B, columns]: pool block of each run of block_tokens positions; lens
    int32[B]: tokens held, the call's included; token_ptr int64[B + 1]: rows of the call's tensors, the last ones that
    each sequence holds.  Host bounds: n_tokens = token_ptr[B]; max_tokens of a sequence in the call (default n_tokens);
    max_len >= lens (default what the table has room for)."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, token_ptr: torch.Tensor, n_tokens: int,
                 max_tokens: int | None = None, max_len: int | None = None):
        B = lens.numel()
        if table.dim() != 2:
            raise ValueError("table has two axes: sequences, columns")
        self.table = _tensor("table", table, torch.int32, (B, table.shape[1]))
        self.lens = _tensor("lens", lens, torch.int32, (B,), table.device)
        self.token_ptr = _tensor("token_ptr", token_ptr, torch.int64, (B + 1,), table.device)
        self.n_tokens = int(n_tokens)
        self.max_tokens = self.n_tokens if max_tokens is None else int(max_tokens)
        self.max_len = max_len
        self.n_seqs, self.device = B, table.device
        self._structs, self._needs = {}, {}

    def _ref(self, cache: KvCache):
        ref = self._structs.get(cache.block_tokens)
        if ref is None:
            room = self.table.shape[1] * cache.block_tokens
            s = _lib.MpKvBatch(self.n_seqs, self.table.shape[1], self.max_tokens,
                               room if self.max_len is None else int(self.max_len), self.n_tokens, _ptr(self.table),
                               _ptr(self.lens), _ptr(self.token_ptr))
            ref = self._structs[cache.block_tokens] = ctypes.byref(s)
        return ref


def _tokens(name, t, cache, batch, n_heads=None):
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != batch.n_tokens or shape[2] != cache.head_dim or \
            (n_heads is not None and shape[1] != n_heads):
        raise ValueError(f"{name}: shape [{batch.n_tokens}, {n_heads or 'heads'}, {cache.head_dim}] is needed, "
                         f"got {list(shape)}")
    if strides[2] != 1 and shape[0] > 0:
        raise ValueError(f"{name}: the values of a head have to be dense")
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: float16, bfloat16 or float32 is needed, got {t.dtype}")
    if t.device != cache.device:
        raise ValueError(f"{name} is on {t.device}, the cache on {cache.device}")
    return _lib.MpTokens(t.data_ptr() or None, strides[0], strides[1], shape[1], dtype)


def _fresh(t, heads, dim):  # a dense tensor that this module has made
    return _lib.MpTokens(t.data_ptr() or None, heads * dim, dim, heads, _DTYPES[t.dtype])


def _status(status, batch):
    if status is None:
        return torch.empty_like(batch.lens)
    return _tensor("status", status, torch.int32, (batch.n_seqs,), batch.device)


def _stream(device):
    # torch.cuda.current_stream() builds a Stream object: 5 us of a call's 22
    return torch._C._cuda_getCurrentRawStream(device.index)


_workspaces = {}


def _workspace_of(stream_ptr, device):
    # calls on different streams may overlap: each stream has its own
    key = (device.index, stream_ptr)
    ws = _workspaces.get(key)
    if ws is None:
        ws = _workspaces[key] = Workspace(device)
    return ws


def kv_write(cache: KvCache, batch: KvBatch, k: torch.Tensor, v: torch.Tensor, status=None, stream=None):
    """Quantises the call's keys and values ([n_tokens, n_heads, head_dim], any strides with dense values) into the
    blocks of their positions.  Returns the status of each sequence."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_write(cache, batch, k, v, status)
    kt = _tokens("k", k, cache, batch, cache.n_heads)
    vt = _tokens("v", v, cache, batch, cache.n_heads)
    status = _status(status, batch)
    _check("mp_kv_write", _lib.load().mp_kv_write(cache._ref, batch._ref(cache), kt, vt, status.data_ptr() or None,
                                                  _stream(cache.device)))
    return status


def kv_read(cache: KvCache, batch: KvBatch, dtype=torch.bfloat16, k=None, v=None, status=None, stream=None):
    """Reads the last n_b of the tokens that each sequence holds back.  Returns (k, v, status)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_read(cache, batch, dtype, k, v, status)
    heads, dim = cache.n_heads, cache.head_dim
    outs = []
    for name, t in (("k", k), ("v", v)):
        if t is None:
            if dtype not in _DTYPES:
                raise ValueError(f"float16, bfloat16 or float32 can be read, not {dtype}")
            t = torch.empty((batch.n_tokens, heads, dim), dtype=dtype, device=cache.device)
            outs += [t, _fresh(t, heads, dim)]
        else:
            outs += [t, _tokens(name, t, cache, batch, heads)]
    k, kt, v, vt = outs
    status = _status(status, batch)
    _check("mp_kv_read", _lib.load().mp_kv_read(cache._ref, batch._ref(cache), kt, vt, status.data_ptr() or None,
                                                _stream(cache.device)))
    return k, v, status


def kv_attend_workspace_bytes(cache: KvCache, batch: KvBatch, n_q_heads: int) -> int:
    key = (n_q_heads, cache.n_heads, cache.head_dim, cache.block_tokens)
    need = batch._needs.get(key)
    if need is None:
        need = batch._needs[key] = int(_lib.load().mp_kv_attend_workspace_bytes(cache._ref, batch._ref(cache), n_q_heads))
    return need


def kv_attend(cache: KvCache, batch: KvBatch, q: torch.Tensor, scale: float | None = None, causal: bool = True,
              window: int = 0, out=None, lse=None, want_lse: bool = False, status=None,
              workspace: Workspace | None = None, stream=None):
    """Attention of the call's queries ([n_tokens, query heads, head_dim], float16 or bfloat16) over what their
    sequences hold: causal unless told otherwise, over the last `window` positions if that is not 0, scale 1 /
    sqrt(head_dim) unless given.  Returns (out, lse or None, status); a query that sees nothing gets 0 and -inf."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return kv_attend(cache, batch, q, scale, causal, window, out, lse, want_lse, status, workspace)
    lib = _lib.load()
    qt = _tokens("q", q, cache, batch)
    heads = q.shape[1]
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        ot = _fresh(out, heads, cache.head_dim)
    else:
        ot = _tokens("out", out, cache, batch, heads)
    if lse is not None:
        _tensor("lse", lse, torch.float32, (batch.n_tokens, heads), cache.device)
    elif want_lse:
        lse = torch.empty((batch.n_tokens, heads), dtype=torch.float32, device=q.device)
    status = _status(status, batch)
    stream_ptr = _stream(cache.device)
    ref = batch._ref(cache)
    need = kv_attend_workspace_bytes(cache, batch, heads)
    wptr, wbytes = (workspace or _workspace_of(stream_ptr, cache.device)).get(need) if need else (None, 0)
    _check("mp_kv_attend",
           lib.mp_kv_attend(cache._ref, ref, qt, cache.head_dim ** -0.5 if scale is None else scale, 1 if causal else 0,
                            window, ot, None if lse is None else lse.data_ptr() or None, status.data_ptr() or None, wptr,
                            wbytes, stream_ptr))
    return out, lse, status
