"""The key/value cache operators of a serving step, as cases that can be timed.

The cache is held in 8 bits (e4m3 bytes, one power-of-two scale for each block of tokens and head) in a pool of blocks;
``table[b, j]`` is the pool block that holds positions [j * block, (j + 1) * block) of sequence b. A case is one operator:

op       write    new tokens quantised into their blocks (kv_write)
         read     tokens read back, scales applied (kv_read)
         attend   attention of new tokens over what their sequences hold (kv_attend)

and its sizes: ``seqs`` sequences that hold ``len_lo`` .. ``len_hi`` tokens, of which the last ``n_lo`` .. ``n_hi`` are the
call's; ``hq`` query heads over ``hkv`` cached heads of ``d`` values; blocks of ``block`` tokens. ``packed``: queries, keys and
values are column ranges of one projection's output, as they leave it, not tensors of their own.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    base = {"dtype": "bf16", "block": 64, "hq": 32, "hkv": 8, "d": 128, "packed": False, "causal": True, "window": 0, "lse": False}
    return [
        # one generated token for each of 8 requests of a small model (hidden 1,024): latency counts
        {"name": "write-step", **base, "op": "write", "seqs": 8, "n_lo": 1, "n_hi": 1, "len_lo": 1, "len_hi": 512, "block": 32,
         "hq": 8, "packed": True},
        # a step of a large serving batch
        {"name": "write-batch", **base, "op": "write", "seqs": 253, "n_lo": 1, "n_hi": 1, "len_lo": 1, "len_hi": 1024},
        # prompts of different lengths enter the cache in one call, some onto a prefix that ends inside a block
        {"name": "write-prompts", **base, "op": "write", "seqs": 9, "n_lo": 511, "n_hi": 4093, "len_lo": 4093, "len_hi": 4500,
         "dtype": "f16", "packed": True},
        # a request's state read back to be moved or inspected, 32 bits
        {"name": "read-ragged", **base, "op": "read", "seqs": 8, "n_lo": 1, "n_hi": 512, "len_lo": 512, "len_hi": 512, "block": 32,
         "hkv": 16, "d": 64, "dtype": "f32"},
        # a long context read back whole
        {"name": "read-long", **base, "op": "read", "seqs": 1, "n_lo": 131071, "n_hi": 131071, "len_lo": 131071, "len_hi": 131071},
        # one request generates a token: the smallest call
        {"name": "step-single", **base, "op": "attend", "seqs": 1, "n_lo": 1, "n_hi": 1, "len_lo": 512, "len_hi": 512, "block": 32,
         "hq": 8, "packed": True},
        # a step of a serving batch of ragged lengths, one of them still empty
        {"name": "step-batch", **base, "op": "attend", "seqs": 64, "n_lo": 1, "n_hi": 1, "len_lo": 0, "len_hi": 8191},
        # two very long contexts
        {"name": "step-long", **base, "op": "attend", "seqs": 2, "n_lo": 1, "n_hi": 1, "len_lo": 250001, "len_hi": 262144,
         "lse": True},
        # a few proposed tokens checked at once, over a window of the context
        {"name": "verify-window", **base, "op": "attend", "seqs": 31, "n_lo": 3, "n_hi": 5, "len_lo": 100, "len_hi": 6000,
         "hq": 12, "hkv": 4, "d": 64, "dtype": "f16", "window": 1000, "block": 32},
        # pieces of prompts over the context before them
        {"name": "chunk", **base, "op": "attend", "seqs": 3, "n_lo": 300, "n_hi": 512, "len_lo": 4000, "len_hi": 16384,
         "packed": True},
        # a whole prompt
        {"name": "prompt", **base, "op": "attend", "seqs": 1, "n_lo": 8000, "n_hi": 8000, "len_lo": 8000, "len_hi": 8000, "lse": True},
        # decoder tokens over an encoder's output (sequence to sequence, hidden 1,024): no causal order
        {"name": "cross", **base, "op": "attend", "seqs": 8, "n_lo": 100, "n_hi": 512, "len_lo": 37, "len_hi": 512, "hq": 16,
         "hkv": 16, "d": 64, "causal": False, "dtype": "f16", "block": 32},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A case within the listed ones' ranges: lengths over their logarithm, any ragged spread, heads and blocks from small sets."""
    hkv, group = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 1, 2, 3, 4, 4, 6, 8])
    c = {"op": rng.choice(["write", "read", "attend", "attend", "attend"]), "dtype": rng.choice(["bf16", "f16"]),
         "block": rng.choice([32, 64, 96, 128]), "hq": hkv * group, "hkv": hkv, "d": rng.choice([64, 128]),
         "packed": rng.random() < 0.5, "causal": True, "window": 0, "lse": rng.random() < 0.3}
    if c["op"] != "attend":
        c["dtype"] = rng.choice(["bf16", "f16", "f32"])
        n = _log(rng, 1, 16384)
        seqs = _log(rng, 1, max(1, min(256, 40_000_000 // (n * hkv * c["d"]))))
        before = rng.choice([0, _log(rng, 1, 1000)])
        c |= {"seqs": seqs, "n_lo": max(1, int(n * rng.uniform(0.2, 1))), "n_hi": n, "len_lo": n, "len_hi": n + before}
        return c
    kind = rng.choice(["step", "step", "few", "chunk", "cross"])
    n = {"step": 1, "few": rng.randint(2, 16), "chunk": _log(rng, 17, 4096), "cross": _log(rng, 17, 512)}[kind]
    length = _log(rng, 16, 512) if kind == "cross" else max(n, _log(rng, 16, 131072 if n <= 16 else 8192))
    most = min(134_000_000 // (length * hkv * c["d"]), 1_000_000_000 // (n * c["hq"] * length))
    c |= {"seqs": _log(rng, 1, max(1, min(128, most))), "n_lo": max(1, int(n * rng.uniform(0.3, 1))), "n_hi": n,
          "len_lo": int(length * rng.uniform(0, 1)), "len_hi": length, "causal": kind != "cross"}
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log(rng, 16, length)
    return c


def _lengths(case):
    """Tokens held and new tokens of every sequence: spread over their ranges, the last sequence at the low end of both."""
    held, new = [], []
    for b in range(case["seqs"]):
        last = b == case["seqs"] - 1 and b > 1
        f, g = (0.0, 0.0) if last else ((b + 1) * 0.6180339887 % 1, (b + 1) * 0.7548776662 % 1)
        n = case["n_lo"] + int((case["n_hi"] - case["n_lo"] + 1) * g)
        length = case["len_lo"] + int((case["len_hi"] - case["len_lo"] + 1) * f)
        held.append(length)
        new.append(n if case["op"] == "attend" else min(n, length))
    return held, new


def _seen(case, length, n):
    """[first, past the last) position seen by each of the n last tokens of a sequence."""
    for i in range(n):
        past = length - n + i + 1 if case["causal"] else length
        yield max(0, past - case["window"]) if case["window"] else 0, max(0, past)


def work(case):
    held, new = _lengths(case)
    row = case["hkv"] * case["d"]
    size = 4 if case["dtype"] == "f32" else 2
    tokens = sum(new)
    if case["op"] in ("write", "read"):
        blocks = sum(-(-length // case["block"]) - (length - n) // case["block"] for length, n in zip(held, new))
        return {"bytes": 2 * tokens * row * (size + 1) + 8 * blocks * case["hkv"], "flops": 0}
    pairs = cached = 0
    for length, n in zip(held, new):
        spans = [s for s in _seen(case, length, n) if s[1] > s[0]]
        pairs += sum(b - a for a, b in spans)
        cached += max(b for _, b in spans) - min(a for a, _ in spans) if spans else 0
    scales = 8 * case["hkv"] * cached // case["block"]
    return {"bytes": 2 * cached * row + scales + 2 * tokens * case["hq"] * case["d"] * 2 + (4 * tokens * case["hq"] if case["lse"] else 0),
            "flops": 4 * pairs * case["hq"] * case["d"]}


def prepare(case, seed):
    """The pool with what the sequences hold, their tables (blocks in no order, -1 past the end), and the new tokens."""
    dev = "cuda"
    gen = torch.Generator(dev).manual_seed(seed)
    held, new = _lengths(case)
    block, hkv, hq, d = case["block"], case["hkv"], case["hq"], case["d"]
    dt = TYPES[case["dtype"]]
    cols = [-(-length // block) for length in held]
    n_blocks, width = max(1, sum(cols)), max(1, max(cols))
    s = SimpleNamespace(case=case, held=held, new=new, width=width)
    shuffled = torch.randperm(n_blocks, generator=gen, device=dev).to(torch.int32)
    ends = torch.tensor([0] + cols, device=dev).cumsum(0)
    j = torch.arange(width, device=dev)
    there = j < (ends[1:] - ends[:-1])[:, None]
    s.table = torch.where(there, shuffled[(ends[:-1, None] + j).clamp(max=n_blocks - 1)], -1).to(torch.int32)
    s.lens = torch.tensor(held, dtype=torch.int32, device=dev)
    s.token_ptr = torch.tensor([0] + new, device=dev).cumsum(0)
    s.tokens, s.most = sum(new), max(new)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    # bytes of the sizes that a block's scale leaves, a few channels of the keys much larger than the others
    loud = torch.where(torch.rand(d, generator=gen, device=dev) < 0.05, 6.0, 1.0)
    s.k, s.v = (torch.empty(n_blocks, hkv, block * d, dtype=torch.uint8, device=dev) for _ in range(2))
    for pool in (s.k, s.v):
        step = max(1, (1 << 26) // (hkv * block * d))
        for at in range(0, n_blocks, step):
            x = normal(min(step, n_blocks - at), hkv, block * d) * 60
            if pool is s.k:
                x = (x.view(-1, hkv, block // 8, d // 16, 8, 16) * loud.view(d // 16, 1, 16)).view_as(x) / 3
            pool[at:at + step] = x.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    s.k_scale, s.v_scale = (torch.exp2(torch.randint(-7, -4, (n_blocks, hkv), generator=gen, device=dev).float()) for _ in range(2))
    # slots past a sequence's end hold anything, here the byte that stands for no number
    b = torch.tensor([b for b, length in enumerate(held) for _ in range(cols[b] * block - length)], dtype=torch.int64, device=dev)
    at = torch.tensor([p for b, length in enumerate(held) for p in range(length, cols[b] * block)], dtype=torch.int64, device=dev)
    if at.numel():
        page, slot = s.table[b, at // block].long(), at % block
        s.k.view(n_blocks, hkv, block // 8, d // 16, 8, 16)[page, :, slot // 8, :, slot % 8] = 0x7F
        s.v.view(n_blocks, hkv, block // 32, d // 8, 2, 8, 16)[page, :, slot // 32, :, slot // 16 % 2, :, slot % 16] = 0x7F

    size = {"write": 2 * hkv, "read": 0, "attend": hq}[case["op"]]
    if case["packed"]:
        proj = normal(s.tokens, (hq + 2 * hkv) * d).to(dt)
        parts = proj.split([hq * d, hkv * d, hkv * d], dim=1)
    else:
        parts = [normal(s.tokens, h * d).to(dt) for h in ((hq, 0, 0) if case["op"] == "attend" else (0, hkv, hkv))]
    if size:
        s.q, s.new_k, s.new_v = (p.view(s.tokens, -1, d) for p in parts)
    s.scale = 1 / math.sqrt(d)
    if own:
        import paper_2203_00448_gb300 as mp

        s.cache = mp.KvCache(n_blocks, block, hkv, d, k=s.k, v=s.v, k_scale=s.k_scale, v_scale=s.v_scale)
        s.batch = mp.KvBatch(s.table, s.lens, s.token_ptr, n_tokens=s.tokens, max_tokens=s.most, max_len=max(held))
    return s


def run(s):
    c = s.case
    if own:
        import paper_2203_00448_gb300 as mp

        if c["op"] == "write":
            mp.kv_write(s.cache, s.batch, s.new_k, s.new_v)
            return _state(s)
        if c["op"] == "read":
            return mp.kv_read(s.cache, s.batch, dtype=TYPES[c["dtype"]])[:2]
        return mp.kv_attend(s.cache, s.batch, s.q, scale=s.scale, causal=c["causal"], window=c["window"], want_lse=c["lse"])[:2]
    return {"write": _write, "read": _read, "attend": _attend}[c["op"]](s)


def _state(s):
    e4m3 = torch.float8_e4m3fn
    return {"k": s.k.view(e4m3), "v": s.v.view(e4m3), "k_scale": s.k_scale, "v_scale": s.v_scale}


# The plain forms.


def _k_tokens(pool, block, d):
    """The pool's key bytes as [blocks, heads, tokens, d]: 8 tokens by 16 values lie together."""
    n, h = pool.shape[:2]
    return pool.view(n, h, block // 8, d // 16, 8, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, h, block, d)


def _v_tokens(pool, block, d):
    """The pool's value bytes as [blocks, heads, tokens, d]: 16 tokens of one value lie together, 8 values by 32 tokens after that."""
    n, h = pool.shape[:2]
    return pool.view(n, h, block // 32, d // 8, 2, 8, 16).permute(0, 1, 2, 4, 6, 3, 5).reshape(n, h, block, d)


def _k_bytes(tokens, block, d):
    n, h = tokens.shape[:2]
    return tokens.view(n, h, block // 8, 8, d // 16, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, h, block * d)


def _v_bytes(tokens, block, d):
    n, h = tokens.shape[:2]
    return tokens.view(n, h, block // 32, 2, 16, d // 8, 8).permute(0, 1, 2, 5, 3, 6, 4).reshape(n, h, block * d)


def _places(s):
    """Every new token's sequence and position."""
    new = s.token_ptr[1:] - s.token_ptr[:-1]
    seq = torch.repeat_interleave(torch.arange(len(s.new), device=s.lens.device), new, output_size=s.tokens)
    at = torch.arange(s.tokens, device=s.lens.device) - s.token_ptr[seq] + (s.lens - new)[seq]
    return seq, at


def _write(s):
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    seq, at = _places(s)
    page, slot = s.table[seq, at // block].long(), at % block
    new = s.token_ptr[1:] - s.token_ptr[:-1]
    # each touched block once: a call's columns of a table are consecutive
    wide = -(-(s.most + block - 1) // block)
    first = (s.lens - new) // block
    col = first[:, None] + torch.arange(wide, device=first.device)
    seq_of, j = ((new[:, None] > 0) & (col * block < s.lens[:, None])).nonzero(as_tuple=True)
    col = col[seq_of, j]
    pages = s.table[seq_of, col].long()
    older = ((s.lens - new)[seq_of] - col * block).clamp(0, block)
    slots = torch.arange(block, device=pages.device)
    is_old = (slots < older[:, None])[:, None, :, None]
    row_of = torch.empty(s.k.shape[0], dtype=torch.int64, device=pages.device)
    row_of[pages] = torch.arange(len(pages), device=pages.device)
    for pool, scales, x, tokens_of, bytes_of in ((s.k, s.k_scale, s.new_k, _k_tokens, _k_bytes), (s.v, s.v_scale, s.new_v, _v_tokens, _v_bytes)):
        x = x.float()
        most = torch.zeros(len(pages), hkv, device=x.device).index_reduce_(0, row_of[page], x.abs().amax(-1), "amax")
        part, power = torch.frexp(most)
        power = torch.where(most > 0, power - 8 - (part <= 0.875).int(), -60).clamp(-60, 120)
        old_scale = scales[pages]
        scale = torch.ldexp(torch.ones_like(most), power)
        scale = torch.where((older > 0)[:, None], torch.maximum(scale, old_scale), scale)
        held = tokens_of(pool[pages], block, d)
        again = (held.view(torch.float8_e4m3fn).float() * (old_scale / scale)[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        held = torch.where(is_old, again, held)
        held[row_of[page], :, slot] = (x / scale[row_of[page], :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[pages] = bytes_of(held, block, d)
        scales[pages] = scale
    return _state(s)


def _read(s):
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    seq, at = _places(s)
    page, slot = s.table[seq, at // block].long(), at % block
    k = s.k.view(-1, hkv, block // 8, d // 16, 8, 16)[page, :, slot // 8, :, slot % 8]
    v = s.v.view(-1, hkv, block // 32, d // 8, 2, 8, 16)[page, :, slot // 32, :, slot // 16 % 2, :, slot % 16]
    out = []
    for x, scales in ((k, s.k_scale), (v, s.v_scale)):
        x = x.reshape(s.tokens, hkv, d).view(torch.float8_e4m3fn).float() * scales[page][:, :, None]
        out.append(x.to(TYPES[c["dtype"]]))
    return tuple(out)


def _attend(s):
    c = s.case
    block, d, hkv, hq, n = c["block"], c["d"], c["hkv"], c["hq"], s.most
    group, seqs = hq // hkv, c["seqs"]
    pages = s.table.clamp(min=0).long()
    full = s.width * block
    k = _k_tokens(s.k, block, d)[pages].view(torch.float8_e4m3fn).float() * s.k_scale[pages][..., None, None]
    v = _v_tokens(s.v, block, d)[pages].view(torch.float8_e4m3fn).float() * s.v_scale[pages][..., None, None]
    k, v = (x.transpose(1, 2).reshape(seqs, hkv, full, d) for x in (k, v))
    seq, at = _places(s)
    i = torch.arange(s.tokens, device=seq.device) - s.token_ptr[seq]
    q = torch.zeros(seqs, n, hq, d, device=seq.device)
    q[seq, i] = s.q.float()
    q = q.view(seqs, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, group * n, d)
    j = torch.arange(full, device=seq.device)
    sees = (j < s.lens[:, None])[:, None, :].expand(seqs, n, full)
    v = torch.where(sees[:, :1, :, None], v, 0)
    if c["causal"]:
        place = (s.lens - (s.token_ptr[1:] - s.token_ptr[:-1]))[:, None] + torch.arange(n, device=seq.device)
        sees = sees & (j <= place[..., None])
        if c["window"]:
            sees = sees & (j > place[..., None] - c["window"])
    x = (q * s.scale) @ k.transpose(2, 3)
    x = x.view(seqs, hkv, group, n, full)
    x = torch.where(sees[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top > -math.inf, top, 0))
    total = x.sum(-1, keepdim=True)
    o = x.view(seqs, hkv, group * n, full) @ v
    o = o.view(seqs, hkv, group, n, d) / torch.where(total > 0, total, 1)
    o = o.permute(0, 3, 1, 2, 4).reshape(seqs, n, hq, d)[seq, i].to(TYPES[c["dtype"]])
    if not c["lse"]:
        return o, None
    lse = (top + torch.log(total)).squeeze(-1)
    return o, lse.permute(0, 3, 1, 2).reshape(seqs, n, hq)[seq, i]


# The definitions in 64 bits, one sequence and head at a time.


def _value(byte):
    """What e4m3 bytes stand for: sign, 4 bits of exponent (bias 7), 3 of fraction."""
    byte = byte.long()
    e, f = byte >> 3 & 15, (byte & 7).double()
    x = torch.where(e > 0, (1 + f / 8) * torch.exp2((e - 7).double()), f / 8 * 2.0 ** -6)
    return torch.where(byte > 127, -x, x)


def _nearest(x):
    """The nearest value that an e4m3 byte holds, ties to the even one."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def _held(s, b, first, past, which):
    """Positions [first, past) of sequence b as stored, in 64 bits: [tokens, heads, d], and the scale of each token and head."""
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    at = torch.arange(first, past, device=s.lens.device)
    page, t = s.table[b, at // block].long()[:, None, None], (at % block)[:, None, None]
    h, i = torch.arange(hkv, device=at.device)[:, None], torch.arange(d, device=at.device)
    if which == "k":
        flat, pool, scales = (t // 8 * (d // 16) + i // 16) * 128 + t % 8 * 16 + i % 16, s.k, s.k_scale
    else:
        flat, pool, scales = t // 32 * (32 * d) + i // 8 * 256 + t // 16 % 2 * 128 + i % 8 * 16 + t % 16, s.v, s.v_scale
    return (page, h, flat), pool[page, h, flat], scales[page[:, 0], h[:, 0]].double()


def exact(case, seed):
    s = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["op"]](s)


def _exact_write(s):
    block = s.case["block"]
    out = {"k_scale": s.k_scale.double(), "v_scale": s.v_scale.double()}
    for which, x in (("k", s.new_k), ("v", s.new_v)):
        pool = _value(getattr(s, which))
        for b, (length, n) in enumerate(zip(s.held, s.new)):
            new = x[int(s.token_ptr[b]):int(s.token_ptr[b + 1])].double()
            for first in range((length - n) // block * block, length if n else 0, block):
                start, past = max(first, length - n), min(first + block, length)
                mine = new[start - (length - n):past - (length - n)]
                most = mine.abs().amax((0, 2)) / 448
                _, e = torch.frexp(most)
                e = torch.where(torch.exp2((e - 1).double()) == most, e - 1, e)
                scale = torch.exp2(torch.where(most > 0, e, -60).clamp(-60, 120).double())
                page = int(s.table[b, first // block])
                if start > first:
                    old = getattr(s, which + "_scale")[page].double()
                    scale = torch.maximum(scale, old)
                    at, byte, _ = _held(s, b, first, start, which)
                    pool[at] = _nearest(_value(byte) * (old / scale)[None, :, None])
                at, _, _ = _held(s, b, start, past, which)
                pool[at] = _nearest(mine / scale[None, :, None])
                out[which + "_scale"][page] = scale
        # the byte that stands for no number, in slots that no token has
        out[which] = torch.where(getattr(s, which) & 127 == 127, math.nan, pool) if s.tokens else pool
        for b, (length, n) in enumerate(zip(s.held, s.new)):
            at, _, _ = _held(s, b, length - n, length, which)
            out[which][at] = pool[at]
    return out


def _exact_read(s):
    out = []
    for which in "kv":
        parts = []
        for b, (length, n) in enumerate(zip(s.held, s.new)):
            _, byte, scale = _held(s, b, length - n, length, which)
            parts.append(_value(byte) * scale[..., None])
        out.append(torch.cat(parts))
    return tuple(out)


def _exact_attend(s):
    c = s.case
    group = c["hq"] // c["hkv"]
    o = torch.zeros(s.q.shape, dtype=torch.float64, device=s.q.device)
    lse = torch.full(s.q.shape[:2], -math.inf, dtype=torch.float64, device=s.q.device)
    for b, (length, n) in enumerate(zip(s.held, s.new)):
        if not length or not n:
            continue
        spans = list(_seen(c, length, n))
        lo = torch.tensor([a for a, _ in spans], device=s.q.device)
        hi = torch.tensor([z for _, z in spans], device=s.q.device)
        k, v = (_value(byte) * scale[..., None] for _, byte, scale in (_held(s, b, 0, length, w) for w in "kv"))
        first = int(s.token_ptr[b])
        for h in range(c["hq"]):
            kh, vh = k[:, h // group], v[:, h // group]
            for i in range(0, n, 1024):
                at = slice(first + i, first + min(n, i + 1024))
                lo_i, hi_i = lo[i:i + 1024, None], hi[i:i + 1024, None]
                x = s.q[at, h].double() @ kh.T * s.scale
                j = torch.arange(length, device=x.device)
                x = x.masked_fill((j < lo_i) | (j >= hi_i), -math.inf)
                total = torch.logsumexp(x, -1)
                w = torch.exp(x - total.clamp(min=-1e300)[:, None])
                o[at, h] = w @ vh
                lse[at, h] = total
    return o, lse if c["lse"] else None
