"""Python binding of the key/value cache operators (argument marshalling only).

    kv_write(cache, batch, k, v)   -> status         new tokens quantised into their blocks
    kv_read(cache, batch)          -> k, v, status   tokens read back
    kv_attend(cache, batch, q)     -> out, lse, status   attention over the cache

A KvCache is a pool of blocks in 8 bits (its memory may be given, e.g. views of a planned slab); a KvBatch says which
blocks the sequences of a call have, how many tokens they hold and which rows of the call's tensors are theirs.  Its
tensors stay on the device and may be changed there between calls, not replaced by others.  All calls are asynchronous on the
current (or given) CUDA stream; what they allocate belongs to that stream.  No gradient passes through them: outputs are
detached from their inputs, whatever these require.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from .api import Workspace, _check, _ptr

_MOST = 1 << 28  # positions, tokens and query rows a head of a sequence
_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}  # mp_dtype


def _tensor(name, t, dtype, shape, device=None):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} is needed, "
                         f"got {t.dtype} {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t


class _Fixed:
    """Attributes whose addresses and values the C structs hold: what they point to may change, they may not."""

    _fixed = frozenset()

    def __setattr__(self, name, value):
        if name in self._fixed and name in self.__dict__ and self.__dict__[name] is not value:
            raise AttributeError(f"{name} cannot be replaced: change its contents, or make another {type(self).__name__}")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{name} cannot be deleted")
        object.__delattr__(self, name)


class KvCache(_Fixed):
    """A pool of n_blocks blocks of block_tokens tokens: e4m3 keys and values of n_heads heads of head_dim values, one
    scale for each block and head.  k, v (uint8[n_blocks, n_heads, block_tokens * head_dim], 16-byte aligned) and
    k_scale, v_scale (float32[n_blocks, n_heads]) are allocated unless given; nothing needs to be initialised."""

    _fixed = frozenset(("n_blocks", "block_tokens", "n_heads", "head_dim", "k", "v", "k_scale", "v_scale", "device"))

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
        for name, t in (("k", self.k), ("v", self.v)):
            if t.data_ptr() % 16:
                raise ValueError(f"{name} has to start on a 16-byte boundary")
        self.device = self.k.device
        self._struct = _lib.MpKvCache(n_blocks, block_tokens, n_heads, head_dim, _ptr(self.k), _ptr(self.v),
                                      _ptr(self.k_scale), _ptr(self.v_scale))
        self._ref = ctypes.byref(self._struct)
        # what a batch's struct and scratch depend on
        self._key, self._index = (n_blocks > 0, block_tokens, n_heads, head_dim, self.device), self.k.get_device()

    @staticmethod
    def block_bytes(block_tokens: int, n_heads: int, head_dim: int) -> int:
        """Bytes of one block: keys, values and their scales (what a plan counts a request's blocks at)."""
        return 2 * n_heads * (block_tokens * head_dim + 4)


class KvBatch(_Fixed):
    """The sequences of a call.  table int32[B, columns]: pool block of each run of block_tokens positions; lens
    int32[B]: tokens held, the call's included; token_ptr int64[B + 1]: rows of the call's tensors, the last ones that
    each sequence holds.  Host bounds: n_tokens = token_ptr[B]; max_tokens of a sequence in the call (default n_tokens);
    max_len >= lens (default what the table has room for).  Either is at most 2^28."""

    _fixed = frozenset(("table", "lens", "token_ptr", "n_tokens", "max_tokens", "max_len", "n_seqs", "device"))

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
        for name, bound in (("max_tokens", self.max_tokens), ("max_len", max_len or 0)):
            if not 0 <= bound <= _MOST:
                raise ValueError(f"{name} is {bound}: 0 to 2^28 is possible")
        self.n_seqs, self.device = B, table.device
        self._made = {}

    def _for(self, cache: KvCache):
        """What calls with this batch and a cache of that shape and device share: the C struct, the shape of the call's keys and
        values, and the scratch by number of query heads."""
        made = self._made.get(cache._key)
        if made is None:
            if cache.device != self.device:
                raise ValueError(f"the batch is on {self.device}, the cache on {cache.device}")
            room = min(self.table.shape[1] * cache.block_tokens, _MOST)
            s = _lib.MpKvBatch(self.n_seqs, self.table.shape[1], self.max_tokens,
                               room if self.max_len is None else int(self.max_len), self.n_tokens, _ptr(self.table),
                               _ptr(self.lens), _ptr(self.token_ptr))
            made = self._made[cache._key] = (ctypes.byref(s), (self.n_tokens, cache.n_heads, cache.head_dim), {})
        return made


def _tokens(name, t, cache, shape):
    """The C struct of a tensor, after the checks; shape: what it has to be, heads None if any number will do."""
    have = t.shape
    if have != shape and (shape[1] is not None or len(have) != 3 or have[0] != shape[0] or have[2] != shape[2]):
        raise ValueError(f"{name}: shape [{shape[0]}, {shape[1] or 'heads'}, {shape[2]}] is needed, got {list(have)}")
    token, head, last = t.stride()
    if last != 1 and have[0] > 0:
        raise ValueError(f"{name}: the values of a head have to be dense")
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: float16, bfloat16 or float32 is needed, got {t.dtype}")
    if t.get_device() != cache._index:
        raise ValueError(f"{name} is on {t.device}, the cache on {cache.device}")
    return _lib.MpTokens(t.data_ptr() or None, token, head, have[1], dtype)


def _fresh(t, heads, dim):  # a dense tensor that this module has made
    return _lib.MpTokens(t.data_ptr() or None, heads * dim, dim, heads, _DTYPES[t.dtype])


def _status(status, batch):
    if status is None:
        return torch.empty_like(batch.lens)
    return _tensor("status", status, torch.int32, (batch.n_seqs,), batch.device)


def _away(cache, stream):
    """Whether a call has to change the current stream or device first: kernels are launched on the current device."""
    return stream is not None or (cache._index >= 0 and torch._C._cuda_getDevice() != cache._index)


def _at(cache, stream):
    """... the context in which it is made."""
    if stream is None:
        return torch.cuda.device(cache._index)
    if stream.device_index != cache._index:
        raise ValueError(f"the stream is on device {stream.device_index}, the cache on {cache.device}")
    return torch.cuda.stream(stream)


def _stream(cache):
    if cache._index < 0:
        raise ValueError(f"the cache is on {cache.device}: these calls run on a GPU")
    # torch.cuda.current_stream() builds a Stream object: 5 us of a call's 22
    return torch._C._cuda_getCurrentRawStream(cache._index)


_workspaces = {}


def _workspace_of(stream_ptr, device):
    # A captured call's scratch belongs to its graph's memory: replays may overlap whatever runs on the stream of the
    # capture, other graphs captured there among it, and go on when that stream's own scratch has been replaced.
    if torch._C._cuda_isCurrentStreamCapturing():
        return Workspace(device)
    # calls on different streams may overlap: each stream has its own
    key = (device.index, stream_ptr)
    ws = _workspaces.get(key)
    if ws is None:
        ws = _workspaces[key] = Workspace(device)
    return ws


def kv_write(cache: KvCache, batch: KvBatch, k: torch.Tensor, v: torch.Tensor, status=None, stream=None):
    """Quantises the call's keys and values ([n_tokens, n_heads, head_dim], any strides with dense values) into the
    blocks of their positions.  Returns the status of each sequence."""
    if _away(cache, stream):
        with _at(cache, stream):
            return kv_write(cache, batch, k, v, status)
    ref, shape, _ = batch._for(cache)
    kt, vt = _tokens("k", k, cache, shape), _tokens("v", v, cache, shape)
    status, stream_ptr = _status(status, batch), _stream(cache)
    _check("mp_kv_write", _lib.load().mp_kv_write(cache._ref, ref, kt, vt, status.data_ptr() or None, stream_ptr))
    return status


def kv_read(cache: KvCache, batch: KvBatch, dtype=torch.bfloat16, k=None, v=None, status=None, stream=None):
    """Reads the last n_b of the tokens that each sequence holds back, as `dtype` or as a k or v that is given.  Returns
    (k, v, status)."""
    if _away(cache, stream):
        with _at(cache, stream):
            return kv_read(cache, batch, dtype, k, v, status)
    ref, shape, _ = batch._for(cache)
    if k is not None:
        kt = _tokens("k", k, cache, shape)
    if v is not None:
        vt = _tokens("v", v, cache, shape)
    if k is None or v is None:
        if k is not None or v is not None:
            dtype = (v if k is None else k).dtype
        if dtype not in _DTYPES:
            raise ValueError(f"float16, bfloat16 or float32 can be read, not {dtype}")
        if k is None:
            k = torch.empty(shape, dtype=dtype, device=cache.device)
            kt = _fresh(k, shape[1], shape[2])
        if v is None:
            v = torch.empty_like(k) if k.is_contiguous() else torch.empty(shape, dtype=dtype, device=cache.device)
            vt = _fresh(v, shape[1], shape[2])
    status, stream_ptr = _status(status, batch), _stream(cache)
    _check("mp_kv_read", _lib.load().mp_kv_read(cache._ref, ref, kt, vt, status.data_ptr() or None, stream_ptr))
    return k, v, status


def kv_attend_workspace_bytes(cache: KvCache, batch: KvBatch, n_q_heads: int) -> int:
    ref, _, needs = batch._for(cache)
    need = needs.get(n_q_heads)
    if need is None:
        need = needs[n_q_heads] = int(_lib.load().mp_kv_attend_workspace_bytes(cache._ref, ref, n_q_heads))
    return need


def kv_attend(cache: KvCache, batch: KvBatch, q: torch.Tensor, scale: float | None = None, causal: bool = True,
              window: int = 0, out=None, lse=None, want_lse: bool = False, status=None,
              workspace: Workspace | None = None, stream=None):
    """Attention of the call's queries ([n_tokens, query heads, head_dim], float16 or bfloat16) over what their
    sequences hold: causal unless told otherwise, over the last `window` positions if that is not 0, scale 1 /
    sqrt(head_dim) unless given.  Returns (out, lse or None, status); a query that sees nothing gets 0 and -inf.  Scratch
    is the stream's unless given, and the graph's own in a capture."""
    if _away(cache, stream):
        with _at(cache, stream):
            return kv_attend(cache, batch, q, scale, causal, window, out, lse, want_lse, status, workspace)
    ref, shape, needs = batch._for(cache)
    if not 0 <= window <= 0x7fffffff:
        window = -1 if window < 0 else 0x7fffffff
    qt = _tokens("q", q, cache, (shape[0], None, shape[2]))
    heads = qt.n_heads
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        ot = _fresh(out, heads, shape[2])
    else:
        ot = _tokens("out", out, cache, (shape[0], heads, shape[2]))
    if lse is not None:
        _tensor("lse", lse, torch.float32, (shape[0], heads), cache.device)
    elif want_lse:
        lse = torch.empty((shape[0], heads), dtype=torch.float32, device=q.device)
    status, stream_ptr = _status(status, batch), _stream(cache)
    need = needs.get(heads)
    if need is None:
        need = kv_attend_workspace_bytes(cache, batch, heads)
    if need:
        scratch = workspace or _workspace_of(stream_ptr, cache.device)
        wptr, wbytes = scratch.get(need)
    else:
        wptr, wbytes = None, 0
    _check("mp_kv_attend",
           _lib.load().mp_kv_attend(cache._ref, ref, qt, shape[2] ** -0.5 if scale is None else scale, 1 if causal else 0,
                                    window, ot, None if lse is None else lse.data_ptr() or None,
                                    status.data_ptr() or None, wptr, wbytes, stream_ptr))
    return out, lse, status
