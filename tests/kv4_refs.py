"""Plain implementations of the 4-bit cache, of block tables from request lengths and of rotary positions, on the CPU, for
the tests.  The cache's is a kv_refs.Pool in which a value is a code and a scale of its own."""
import math
from fractions import Fraction

import numpy as np
import torch

from tests import kv_refs as R

SCALES = np.array([(b & 7) / 8 * 2.0 ** -14 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 15) for b in range(184)])


def scale_byte(a):
    """Of the least scale with a <= 7.5 of it, in whole numbers."""
    for b, s in enumerate(SCALES):
        if Fraction(float(a)) <= Fraction(15, 2) * Fraction(float(s)):
            return b
    return 183


def quantise(x):
    """Codes and scale bytes of [..., 32] float64 values without NaN, of magnitudes up to 1,800."""
    a = np.abs(x).max(-1)
    byte = np.searchsorted(7.5 * SCALES, a)  # 7.5 * s has 8 significant bits
    s = SCALES[byte]
    n = np.clip(np.rint(np.divide(x, s[..., None], out=np.zeros_like(x), where=s[..., None] > 0)), -7, 7)
    return (n + 8).astype(np.uint8), byte.astype(np.uint8)


class Pool:
    """A pool in plain order: codes [blocks, heads, tokens, d], scale bytes [blocks, heads, tokens, d / 32]."""

    def __init__(self, n_blocks, block, heads, d, rng):
        self.n, self.block, self.heads, self.d = n_blocks, block, heads, d
        shape = (n_blocks, heads, block, d)
        self.k, self.v = (np.clip(np.rint(rng.standard_normal(shape) * 3) + 8, 0, 15).astype(np.uint8) for _ in range(2))
        self.ks, self.vs = (rng.integers(80, 104, (*shape[:3], d // 32)).astype(np.uint8) for _ in range(2))

    def places(self, keys):
        """Byte and half of each code (t, d) of a granule, and byte of each scale (t, group)."""
        D = self.d
        t, d = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
        u, g = np.meshgrid(np.arange(32), np.arange(D // 32), indexing="ij")
        if keys:
            return t * D // 2 + d // 2, d % 2, 16 * D + u % 8 * D // 8 + g * 4 + u // 8
        e = D // 8
        code = ((t // 8 * 8 + d // e) * 4 + t % 8 // 2) * e + d % e // 4 * 4 + t % 2 * 2 + d % 4 // 2
        return code, d % 2, 16 * D + (g * 4 + u // 2 % 4) * 8 + u // 8 * 2 + u % 2

    def stored(self):
        out = []
        for code, scale, keys in ((self.k, self.ks, True), (self.v, self.vs, False)):
            at, half, scale_at = self.places(keys)
            y = np.zeros((self.n, self.heads, self.block // 32, 17 * self.d), np.uint8)
            code = code.reshape(*y.shape[:3], 32, self.d)
            for h in (0, 1):
                y[..., at[half == h]] |= code[..., half == h] << (4 * h)
            y[..., scale_at] = scale.reshape(*y.shape[:3], 32, -1)
            out.append(y.reshape(self.n, self.heads, -1))
        return out

    def from_stored(self, k, v):
        """Codes and scales of stored bytes, keys' then values'."""
        out = []
        for y, keys in ((k, True), (v, False)):
            at, half, scale_at = self.places(keys)
            y = y.reshape(self.n, self.heads, self.block // 32, 17 * self.d)
            code = y[..., at] >> (4 * half) & 15
            out += [code.reshape(self.k.shape).astype(np.uint8), y[..., scale_at].reshape(self.ks.shape)]
        return out

    def cache(self, device="cuda"):
        import paper_2203_00448_gb300 as mp

        k, v = (torch.from_numpy(x).to(device) for x in self.stored())
        return mp.KvCache4(self.n, self.block, self.heads, self.d, k=k, v=v)


def write(pool, table, lens, new, k, v):
    """In place; k, v: float64 [tokens, heads, d].  Returns the status."""
    status, row = [], 0
    for b, (length, n) in enumerate(zip(lens, new)):
        status.append(0)
        for x, codes, scales in ((k, pool.k, pool.ks), (v, pool.v, pool.vs)):
            y = x[row:row + n]
            if not (np.abs(y) <= 1800).all():
                status[b] = 1
            y = np.clip(np.where(np.isnan(y), 0, y), -1800, 1800).reshape(n, pool.heads, pool.d // 32, 32)
            at = np.arange(length - n, length)
            page, slot = table[b, at // pool.block], at % pool.block
            code, byte = quantise(y)
            codes[page, :, slot], scales[page, :, slot] = code.reshape(n, pool.heads, pool.d), byte
        row += n
    return np.array(status, np.int32)


def held(pool, table, b, first, past):
    j = np.arange(first, past)
    page, slot = table[b, j // pool.block], j % pool.block
    out = []
    for code, scale in ((pool.k, pool.ks), (pool.v, pool.vs)):
        s = SCALES[np.minimum(scale[page, :, slot], 183)].repeat(32, -1)
        out.append((code[page, :, slot].astype(np.float64) - 8) * s)
    return out


def attend(pool, table, lens, new, q, scale, causal=True, window=0):
    """kv_refs.attend over this pool."""
    was, R.held = R.held, held
    try:
        return R.attend(pool, table, lens, new, q, scale, causal, window)
    finally:
        R.held = was


def extend(table, lens, new, block, n_tokens, max_tokens, max_len, free=None, n_free=0, n_blocks=0, first=None, room=None):
    """One step, a request at a time; table and free (lists or arrays) in place.  Returns what kv_extend makes."""
    B = len(lens)
    blocks = lambda n: -(-n // block)  # noqa: E731
    status, out, step = [1] * B, list(lens), [-1] * B
    ptr = np.concatenate([[0], np.cumsum([max(n, 0) for n in new])]).astype(np.int64)
    positions, slots = np.full(n_tokens, -77, np.int32), np.full(n_tokens, -77, np.int64)
    room_for = len(table[0]) * block if B else 0
    sound = [0 <= a and max(n, 0) <= max_tokens and a + max(n, 0) <= (room_for if n < 0 else max_len) for a, n in zip(lens, new)]
    stack = first is not None or 0 <= n_free <= n_blocks
    top = back = n_free
    if first is None and stack:
        for b in range(B):
            if new[b] < 0 and sound[b]:
                back += blocks(lens[b])
                if back <= n_blocks:
                    for j in range(blocks(lens[b])):
                        free[top + j] = table[b][j]
                    top, status[b], out[b] = back, 0, 0
    want = given = 0
    for b in range(B):
        if new[b] < 0 and first is not None and sound[b]:
            status[b], out[b] = 0, 0
        if new[b] < 0 or not sound[b] or ptr[b + 1] > n_tokens:
            continue
        need = blocks(lens[b] + new[b]) - blocks(lens[b])
        if not stack:
            want += need
            continue
        if first is None:
            want += need
            status[b] = 5 if need and want > top else 0
        else:
            last = blocks(lens[b] + new[b])
            status[b] = 1 if first[b] < 0 or first[b] + last > n_blocks else 5 if last > room[b] else 0
        if status[b]:
            continue
        for j in range(need):
            col = blocks(lens[b]) + j
            table[b][col] = free[top - 1 - (want - need) - j] if first is None else first[b] + col
        if first is None and need:
            given = want
        out[b] = step[b] = lens[b] + new[b]
    for b in range(B):
        for i in range(min(max(new[b], 0), max(0, n_tokens - int(ptr[b])))):
            row, p = ptr[b] + i, lens[b] + i
            positions[row] = slots[row] = -1
            if step[b] >= 0:
                positions[row] = p
                slots[row] = (int(table[b][p // block]) if first is None else first[b] + p // block) * block + p % block
    return {"status": status, "lens": out, "step_lens": step, "token_ptr": ptr, "positions": positions, "slots": slots,
            "n_free": top - given if stack else n_free}


def rotary(x, positions, frequencies, amplitude, layout, inverse):
    """x float64 [tokens, heads, d]; angles reduced with whole numbers."""
    y = x.copy()
    pairs = len(frequencies)
    two_pi = Fraction(math.pi) + Fraction(1.2246467991473532e-16)  # sin(pi) in doubles is what pi's double lacks
    for t, p in enumerate(positions):
        for i, f in enumerate(frequencies):
            turns = Fraction(int(p)) * Fraction(float(f)) / (2 * two_pi)
            turns -= round(turns)
            angle = float(turns * 2 * two_pi) * (-1 if inverse else 1)
            a, b = (i, i + pairs) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = amplitude * math.cos(angle), amplitude * math.sin(angle)
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, a] * s + x[t, :, b] * c
    return y
