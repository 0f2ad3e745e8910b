"""Python binding of rotary positions (argument marshalling only).

    rotary(rotation, positions, q, k)  -> q, k   queries and keys turned to their positions, or gradients turned back

A Rotary holds the frequencies of one kind of model on the device.  Calls are asynchronous on the current (or given) CUDA
stream.  No gradient passes through them: the gradient of a call is the call with inverse=True on the gradients of its outputs.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _lib
from .api import _check
from .kv import _DTYPES, _at, _away, _Fixed, _stream, _tensor

LAYOUTS = ("half", "interleaved")
_KINDS = {"linear": ("factor",), "base": ("factor",), "parts": ("factor", "original", "fast", "slow"),
          "bands": ("factor", "original", "low", "high")}


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: dict | None = None):
    """Radians a position of each of dim / 2 pairs (float64) and the amplitude: base ** (-2 i / dim), for longer contexts scaled
    by {"kind": ..}:

    linear  factor                          all divided by factor
    base    factor                          base times factor ** (dim / (dim - 2)): the slowest pair is divided by factor
    parts   factor, original, fast, slow    pairs that turn `fast` times over the original length stay, those that turn `slow`
                                            times are divided by factor, a ramp over the pairs' indexes between; amplitude 0.1
                                            ln(factor) + 1, 1 for factors below 1
    bands   factor, original, low, high     the same with a ramp over the number of turns, from low (divided) to high (as they
                                            are); amplitude 1
    """
    if dim < 2 or dim % 2 or not base > 0:
        raise ValueError(f"dim is even and at least 2, base positive; got {dim}, {base}")
    index = torch.arange(dim // 2, dtype=torch.float64)
    f = base ** (-2 * index / dim)
    if scaling is None:
        return f, 1.0
    kind = scaling.get("kind")
    if kind not in _KINDS or set(scaling) != {"kind", *_KINDS[kind]}:
        raise ValueError(f"scaling is a kind of {sorted(_KINDS)} with its numbers, got {scaling}")
    factor = float(scaling["factor"])
    if not 0 < factor < math.inf:
        raise ValueError("factor is positive")
    if kind == "linear":
        return f / factor, 1.0
    if kind == "base":
        if dim < 4:
            raise ValueError("kind 'base' needs dim of 4 or more")
        return (base * factor ** (dim / (dim - 2))) ** (-2 * index / dim), 1.0
    original = float(scaling["original"])
    lo, hi = (("slow", "fast") if kind == "parts" else ("low", "high"))
    lo, hi = float(scaling[lo]), float(scaling[hi])
    if not (0 < lo < hi < math.inf and 0 < original < math.inf):
        raise ValueError("original is positive, and the numbers of turns are in order")
    if kind == "bands":
        stay = ((original * f / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1)
        return f * stay + f / factor * (1 - stay), 1.0
    if base == 1:
        raise ValueError("kind 'parts' needs a base other than 1")
    place = [dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (hi, lo)]
    first, last = max(0, math.floor(place[0])), min(dim - 1, math.ceil(place[1]))
    scaled = ((index - first) / max(last - first, 1e-3)).clamp(0, 1)
    return f * (1 - scaled) + f / factor * scaled, 0.1 * math.log(max(factor, 1.0)) + 1


def _turns(frequencies):
    """Turns a position, times 2^64, whole turns left out: int64 with the bits of the unsigned number; as exact as doubles,
    2^-52 of a frequency's turns."""
    out = []
    for f in frequencies.tolist():
        if not math.isfinite(f):
            raise ValueError("frequencies have to be finite")
        t = round(math.fmod(f / (2 * math.pi), 1.0) * 2.0 ** 64) % (1 << 64)
        out.append(t - (1 << 64) if t >= 1 << 63 else t)
    return torch.tensor(out, dtype=torch.int64)


class Rotary(_Fixed):
    """Frequencies and layout of a model's rotary positions: the first dim elements of a head turn, in pairs (i, i + dim / 2)
    ("half") or (2 i, 2 i + 1) ("interleaved").  frequencies (radians a position, dim / 2 of them) and amplitude take the
    place of those that base and scaling give."""

    _fixed = frozenset(("dim", "layout", "frequencies", "amplitude", "turns", "device"))

    def __init__(self, dim: int, base: float = 10000.0, layout: str = "half", scaling: dict | None = None, frequencies=None,
                 amplitude: float | None = None, device="cuda"):
        if layout not in LAYOUTS:
            raise ValueError(f"layout is one of {LAYOUTS}, got {layout!r}")
        if frequencies is None:
            frequencies, own = rotary_frequencies(dim, base, scaling)
        else:
            if scaling is not None:
                raise ValueError("frequencies that are given are not scaled")
            frequencies, own = torch.as_tensor(frequencies, dtype=torch.float64).cpu(), 1.0
            if dim < 2 or dim % 2 or tuple(frequencies.shape) != (dim // 2,):
                raise ValueError(f"dim is even and at least 2, and frequencies are dim / 2, got {dim} and {tuple(frequencies.shape)}")
        amplitude = own if amplitude is None else float(amplitude)
        if not math.isfinite(amplitude):
            raise ValueError("amplitude has to be finite")
        self.dim, self.layout, self.frequencies, self.amplitude = dim, layout, frequencies, amplitude
        self.turns = _turns(frequencies).to(device)
        self.device, self._index = self.turns.device, self.turns.get_device()
        self._struct = _lib.MpRotation(dim, LAYOUTS.index(layout), self.turns.data_ptr(), amplitude)
        self._ref = ctypes.byref(self._struct)


def _rows(name, t, like, index):
    """The C struct of [tokens, heads, head_dim] rows, after the checks; like: shape and dtype it has to have."""
    if t.dim() != 3 or (like is not None and (t.shape != like.shape or t.dtype != like.dtype)):
        raise ValueError(f"{name}: a tensor [tokens, heads, head_dim]" + ("" if like is None else f" like {list(like.shape)} {like.dtype}")
                         + f" is needed, got {list(t.shape)} {t.dtype}")
    token, head, last = t.stride()
    if last != 1 and t.numel() > 0:
        raise ValueError(f"{name}: the values of a head have to be dense")
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: float16, bfloat16 or float32 is needed, got {t.dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on the frequencies' device")
    return _lib.MpTokens(t.data_ptr() or None, token, head, t.shape[1], dtype)


def rotary(rotation: Rotary, positions: torch.Tensor, q: torch.Tensor | None, k: torch.Tensor | None = None, q_out=None, k_out=None,
           inverse: bool = False, stream=None):
    """Turns q and k ([n_tokens, heads, head_dim], any strides with dense values, either may be None) to positions
    int32[n_tokens], back with inverse.  Returns (q, k): new tensors, or q_out and k_out, which may be q and k themselves."""
    if _away(rotation, stream):
        with _at(rotation, stream):
            return rotary(rotation, positions, q, k, q_out, k_out, inverse)
    stream_ptr, index = _stream(rotation), rotation._index
    some = q if q is not None else k
    if some is None or (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("q or k is needed, and an output only for what is there")
    _tensor("positions", positions, torch.int32, some.shape[:1], rotation.device)
    structs, outs = [], []
    for name, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            structs += (None, None)
            outs.append(None)
            continue
        a = _rows(name, x, None, index)
        tokens, heads, dim = x.shape
        if x is not some and (tokens != some.shape[0] or dim != some.shape[2] or x.dtype != some.dtype):
            raise ValueError("q and k have as many tokens, heads of one size and one type")
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            b = _lib.MpTokens(out.data_ptr() or None, heads * dim, dim, heads, a.dtype)
        else:
            b = _rows(name + "_out", out, x, index)
        structs += (a, b) if heads else (None, None)  # nothing of a tensor without heads turns
        outs.append(out)
    if rotation.dim > some.shape[2]:
        raise ValueError(f"dim is {rotation.dim}, heads have {some.shape[2]} values")
    qi, qo, ki, ko = structs
    if some.shape[0] > 0 and (qi is not None or ki is not None):
        _check("mp_rotary", _lib.load().mp_rotary(rotation._ref, positions.data_ptr(), some.shape[0], some.shape[2], qi, ki, qo, ko,
                                                  1 if inverse else 0, stream_ptr))
    return tuple(outs)
