"""Plain 64-bit implementations of the key/value cache operators, on the CPU, for the tests."""
import math

import numpy as np
import torch


def e4m3_values():
    """What the 256 bytes stand for (NaN for the two that stand for none)."""
    x = np.zeros(256)
    for b in range(256):
        e, f = b >> 3 & 15, b & 7
        m = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        x[b] = math.nan if b & 127 == 127 else -m if b & 128 else m
    return x


VALUES = e4m3_values()
_FINITE = np.array([b for b in range(127)])


def to_byte(x):
    """The byte of the nearest e4m3 value (ties to the even byte, saturating); x: float64 array without NaN."""
    grid = VALUES[_FINITE]
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


class Pool:
    """A pool in plain order: bytes [blocks, heads, tokens, d] and scales, and the stored layout of it."""

    def __init__(self, n_blocks, block, heads, d, rng, fill="random"):
        self.n, self.block, self.heads, self.d = n_blocks, block, heads, d
        shape = (n_blocks, heads, block, d)
        if fill == "nan":
            self.k, self.v = (np.full(shape, 0x7F, np.uint8) for _ in range(2))
        else:
            self.k, self.v = (to_byte(rng.standard_normal(shape) * 60) for _ in range(2))
        self.ks, self.vs = (np.exp2(rng.integers(-7, -4, (n_blocks, heads))).astype(np.float32) for _ in range(2))

    def layout(self):
        """Place in a block and head of key and value (t, d)."""
        t, d = np.meshgrid(np.arange(self.block), np.arange(self.d), indexing="ij")
        k = (t // 8 * (self.d // 16) + d // 16) * 128 + t % 8 * 16 + d % 16
        v = t // 32 * 32 * self.d + d // 8 * 256 + t // 16 % 2 * 128 + d % 8 * 16 + t % 16
        return k, v

    def stored(self):
        out = []
        for x, at in zip((self.k, self.v), self.layout()):
            y = np.zeros((self.n, self.heads, self.block * self.d), np.uint8)
            y[:, :, at.reshape(-1)] = x.reshape(self.n, self.heads, -1)
            out.append(y)
        return out

    def from_stored(self, k, v):
        return [y[:, :, at.reshape(-1)].reshape(self.n, self.heads, self.block, self.d)
                for y, at in zip((k, v), self.layout())]

    def cache(self, device="cuda"):
        import paper_2203_00448_gb300 as mp

        k, v = (torch.from_numpy(x).to(device) for x in self.stored())
        return mp.KvCache(self.n, self.block, self.heads, self.d, k=k, v=v,
                          k_scale=torch.from_numpy(self.ks).to(device), v_scale=torch.from_numpy(self.vs).to(device))


def make_table(lens, block, rng, spare=2):
    """A table over shuffled blocks, -1 past each sequence's end; returns it and the pool's size."""
    cols = [-(-n // block) for n in lens]
    ids = rng.permutation(sum(cols) + spare)
    table = np.full((len(lens), max([1] + cols)), -1, np.int32)
    at = 0
    for b, c in enumerate(cols):
        table[b, :c] = ids[at:at + c]
        at += c
    return table, len(ids)


def scale_of(a):
    """The least power of two 2^e, -60 <= e <= 120, with a <= 448 * 2^e."""
    e = -60
    while e < 120 and a > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def write(pool, table, lens, new, k, v):
    """In place; k, v: float64 [tokens, heads, d]; new: tokens of each sequence.  Returns the status."""
    status, row = [], 0
    for b, (length, n) in enumerate(zip(lens, new)):
        status.append(0)
        for x, data, scales in ((k, pool.k, pool.ks), (v, pool.v, pool.vs)):
            mine = x[row:row + n]
            if not np.isfinite(mine).all():
                status[b] = 1
            for col in range((length - n) // pool.block, -(-length // pool.block) if n else 0):
                first = max(length - n, col * pool.block)
                past = min(length, (col + 1) * pool.block)
                page, s0, s1 = table[b, col], first - col * pool.block, past - col * pool.block
                for h in range(pool.heads):
                    y = mine[first - (length - n):past - (length - n), h]
                    fine = np.abs(y[np.isfinite(y)])
                    scale = scale_of(fine.max() if fine.size else 0.0)
                    old = float(scales[page, h])
                    if s0 > 0 and old >= scale:
                        scale = old
                    elif s0 > 0:
                        data[page, h, :s0] = to_byte(VALUES[data[page, h, :s0]] * (old / scale))
                    scales[page, h] = scale
                    data[page, h, s0:s1] = to_byte(np.where(np.isnan(y), 0.0, y) / scale)
        row += n
    return np.array(status, np.int32)


def held(pool, table, b, first, past):
    """Keys and values of positions [first, past) of sequence b: float64 [tokens, heads, d]."""
    j = np.arange(first, past)
    page, slot = table[b, j // pool.block], j % pool.block
    k = VALUES[pool.k[page, :, slot]] * pool.ks[page].astype(np.float64)[:, :, None]
    v = VALUES[pool.v[page, :, slot]] * pool.vs[page].astype(np.float64)[:, :, None]
    return k, v


def attend(pool, table, lens, new, q, scale, causal=True, window=0):
    """q float64 [tokens, query heads, d].  Returns out, lse, and for error bounds the softmax-weighted mean of |v| and the
    largest sum |q| |k| * scale of each query."""
    T, hq, d = q.shape
    group = hq // pool.heads
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, size = np.full((T, hq), -np.inf), np.zeros((T, hq))
    row = 0
    for b, (length, n) in enumerate(zip(lens, new)):
        k, v = held(pool, table, b, 0, length)
        for i in range(n):
            p = length - n + i
            hi = min(length, p + 1) if causal else length
            lo = max(0, p - window + 1) if window else 0
            if hi <= lo:
                continue
            for h in range(hq):
                kk, vv = k[lo:hi, h // group], v[lo:hi, h // group]
                x = kk @ q[row + i, h] * scale
                top = x.max()
                w = np.exp(x - top)
                out[row + i, h] = w @ vv / w.sum()
                mag[row + i, h] = w @ np.abs(vv) / w.sum()
                lse[row + i, h] = top + np.log(w.sum())
                size[row + i, h] = (np.abs(kk) @ np.abs(q[row + i, h])).max() * scale
        row += n
    return out, lse, mag, size


def attend_bounds(dtype, out, lse, mag, size):
    """How far an output may be off, from the formats: products of 16-bit values summed in 32 bits (d + 1 roundings of
    2^-23, truncation included, and two of the scaling), exponentials good to 2^-21, weights rounded to 11 bits, sums of
    up to 2^13 terms in no order (their error grows with the terms' count's root: 2^-17 is taken), and one rounding to the
    output's type."""
    d = out.shape[-1]
    x = size * (d + 4) * 2.0 ** -23 + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))
    w = 2 * x + 2.0 ** -17
    last = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    tiny = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -25
    return (w[..., None] + 2.0 ** -11) * mag + last * np.abs(out) + tiny, w
