"""The operators around a serving step's attention, as cases that can be timed.

A request's tokens get their blocks, their queries and keys are turned to their positions, keys and values go into a cache
held in 4 bits, and attention reads it.  A case is one operator:

op       extend   a step's block table, lengths, positions and slots from the requests' new tokens (kv_extend)
         rotary   queries and keys turned by their positions, or gradients turned back (rotary)
         store    a call's tokens quantised into their blocks of 4 bits, and what is held of them (kv_write, kv_read)
         read     tokens read back (kv_read)
         attend   attention of new tokens over what their sequences hold (kv_attend)

The cache: 32 values of a token and head share a scale of 8 bits, which are the 8 bits behind the sign of an f16; a value
is a code of 4 bits (8 more than a whole number) times the scale.  32 tokens of a head lie together, codes first, then scales.

extend: ``seqs`` requests that hold up to ``len_hi`` tokens and get ``n_lo`` .. ``n_hi`` more, a share ``ends`` of them is done
and gives its blocks back; the pool has ``spare`` of the blocks that the step needs.  rotary: ``tokens`` of ``hq`` + ``hkv`` heads of
``d`` values, of which the first ``dim`` turn, positions up to ``far``.  store, read, attend: ``seqs`` sequences that hold ``len_lo`` ..
``len_hi`` tokens, of which the last ``n_lo`` .. ``n_hi`` are the call's.  ``packed``: queries, keys and values are column ranges of
one projection's output.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32  # values that share a scale, and tokens that lie together


def listed():
    base = {"dtype": "bf16", "block": 64, "hq": 32, "hkv": 8, "d": 128, "packed": False, "causal": True, "window": 0, "lse": False}
    return [
        # a generated token for each of 64 requests, a few of them done, all blocks to be had: latency counts
        {"name": "extend-step", "op": "extend", "seqs": 64, "n_lo": 1, "n_hi": 1, "len_hi": 2000, "block": 64, "ends": 0.1, "spare": 1.0},
        # prompts and generated tokens of many requests, more of them than the pool has blocks for
        {"name": "extend-prompts", "op": "extend", "seqs": 509, "n_lo": 1, "n_hi": 517, "len_hi": 8000, "block": 32, "ends": 0.05,
         "spare": 0.9},
        # one generated token for each of 8 requests of a small model (hidden 1,024)
        {"name": "rotary-step", "op": "rotary", "tokens": 8, "hq": 8, "hkv": 8, "d": 128, "dim": 128, "layout": "half", "dtype": "bf16",
         "far": 4096, "scaling": "none", "inverse": False, "packed": True},
        # the gradients of a training batch's queries and keys, part of each head turned, scaled for long contexts
        {"name": "rotary-gradient", "op": "rotary", "tokens": 15973, "hq": 16, "hkv": 16, "d": 64, "dim": 32, "layout": "interleaved",
         "dtype": "f32", "far": 131072, "scaling": "parts", "inverse": True, "packed": False},
        # a step of a large serving batch enters the cache
        {"name": "store-batch", **base, "op": "store", "seqs": 253, "n_lo": 1, "n_hi": 1, "len_lo": 1, "len_hi": 1024},
        # prompts of different lengths, some onto a prefix that ends inside a block
        {"name": "store-prompts", **base, "op": "store", "seqs": 9, "n_lo": 511, "n_hi": 4093, "len_lo": 4093, "len_hi": 4500,
         "dtype": "f16", "packed": True},
        # a few requests' state read back to be looked at, 32 bits
        {"name": "read-ragged", **base, "op": "read", "seqs": 8, "n_lo": 1, "n_hi": 512, "len_lo": 512, "len_hi": 512, "block": 32,
         "hkv": 16, "d": 64, "dtype": "f32"},
        # a long context read back whole
        {"name": "read-long", **base, "op": "read", "seqs": 1, "n_lo": 131071, "n_hi": 131071, "len_lo": 131071, "len_hi": 131071},
        # one request generates a token
        {"name": "attend-single", **base, "op": "attend", "seqs": 1, "n_lo": 1, "n_hi": 1, "len_lo": 512, "len_hi": 512, "block": 32,
         "hq": 8, "packed": True},
        # a step of a serving batch of ragged lengths, one of them still empty
        {"name": "attend-batch", **base, "op": "attend", "seqs": 64, "n_lo": 1, "n_hi": 1, "len_lo": 0, "len_hi": 8191},
        # two very long contexts, which 4 bits are for
        {"name": "attend-long", **base, "op": "attend", "seqs": 2, "n_lo": 1, "n_hi": 1, "len_lo": 250001, "len_hi": 262144, "lse": True},
        # pieces of prompts over the context before them
        {"name": "attend-chunk", **base, "op": "attend", "seqs": 3, "n_lo": 300, "n_hi": 512, "len_lo": 4000, "len_hi": 16384,
         "packed": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A case within the listed ones' ranges: sizes over their logarithm, any ragged spread, heads and blocks from small sets."""
    op = rng.choice(["extend", "rotary", "rotary", "store", "read", "attend", "attend", "attend"])
    if op == "extend":
        n = rng.choice([1, rng.randint(2, 16), _log(rng, 17, 600)])
        return {"op": op, "seqs": _log(rng, 1, max(1, min(600, 300_000 // n))), "n_lo": rng.choice([0, 1, n]), "n_hi": n,
                "len_hi": _log(rng, 1, 8192), "block": rng.choice([32, 64, 96, 128]), "ends": rng.choice([0.0, 0.1, 0.5]),
                "spare": rng.choice([0.5, 0.9, 1.0, 1.5])}
    hkv, group = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 1, 2, 3, 4, 4, 6, 8])
    d = rng.choice([64, 128])
    if op == "rotary":
        dtype = rng.choice(["bf16", "f16", "f32"])
        row = (hkv * group + hkv) * d
        return {"op": op, "tokens": _log(rng, 1, min(16384, 32_000_000 // row)), "hq": hkv * group, "hkv": hkv, "d": d,
                "dim": rng.choice([d, d, d // 2, d // 4, 40]), "layout": rng.choice(["half", "interleaved"]), "dtype": dtype,
                "far": _log(rng, 16, 1 << 20), "scaling": rng.choice(["none", "linear", "base", "parts", "bands"]),
                "inverse": rng.random() < 0.4, "packed": rng.random() < 0.5}
    c = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "block": rng.choice([32, 64, 96, 128]), "hq": hkv * group, "hkv": hkv, "d": d,
         "packed": rng.random() < 0.5, "causal": True, "window": 0, "lse": rng.random() < 0.3}
    if op != "attend":
        c["dtype"] = rng.choice(["bf16", "f16", "f32"])
        n = _log(rng, 1, 16384)
        seqs = _log(rng, 1, max(1, min(256, 40_000_000 // (n * hkv * d))))
        before = rng.choice([0, _log(rng, 1, 1000)])
        c |= {"seqs": seqs, "n_lo": max(1, int(n * rng.uniform(0.2, 1))), "n_hi": n, "len_lo": n, "len_hi": n + before}
        return c
    kind = rng.choice(["step", "step", "few", "chunk", "cross"])
    n = {"step": 1, "few": rng.randint(2, 16), "chunk": _log(rng, 17, 4096), "cross": _log(rng, 17, 512)}[kind]
    length = _log(rng, 16, 512) if kind == "cross" else max(n, _log(rng, 16, 131072 if n <= 16 else 8192))
    most = min(134_000_000 // (length * hkv * d), 800_000_000 // (n * c["hq"] * length))
    c |= {"seqs": _log(rng, 1, max(1, min(128, most))), "n_lo": max(1, int(n * rng.uniform(0.3, 1))), "n_hi": n,
          "len_lo": int(length * rng.uniform(0, 1)), "len_hi": length, "causal": kind != "cross"}
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log(rng, 16, length)
    return c


def _spread(i, step, lo, hi):
    return lo + int((hi - lo + 1) * ((i + 1) * step % 1))


def _lengths(case):
    """Tokens held and new tokens of every sequence: spread over their ranges, the last sequence at the low end of both."""
    held, new = [], []
    for b in range(case["seqs"]):
        last = b == case["seqs"] - 1 and b > 1
        n = case["n_lo"] if last else _spread(b, 0.7548776662, case["n_lo"], case["n_hi"])
        length = case["len_lo"] if last else _spread(b, 0.6180339887, case["len_lo"], case["len_hi"])
        held.append(length)
        new.append(n if case["op"] == "attend" else min(n, length))
    return held, new


def _requests(case):
    """Tokens held and new tokens (-1: done) of every request."""
    held = [_spread(b, 0.6180339887, 0, case["len_hi"]) for b in range(case["seqs"])]
    new = [-1 if (b + 1) * 0.5698402909 % 1 < case["ends"] else _spread(b, 0.7548776662, case["n_lo"], case["n_hi"])
           for b in range(case["seqs"])]
    return held, new


def _blocks(n, block):
    return -(-n // block)


def _seen(case, length, n):
    """[first, past the last) position seen by each of the n last tokens of a sequence."""
    for i in range(n):
        past = length - n + i + 1 if case["causal"] else length
        yield max(0, past - case["window"]) if case["window"] else 0, max(0, past)


def work(case):
    if case["op"] == "extend":
        held, new = _requests(case)
        block = case["block"]
        moved = sum(_blocks(a, block) if n < 0 else _blocks(a + n, block) - _blocks(a, block) for a, n in zip(held, new))
        return {"bytes": 28 * case["seqs"] + 8 * moved + 12 * sum(max(n, 0) for n in new), "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotary":
        row = case["hq"] + case["hkv"]
        return {"bytes": case["tokens"] * (2 * row * case["d"] * size + 4), "flops": 3 * case["tokens"] * row * case["dim"]}
    held, new = _lengths(case)
    row, tokens = case["hkv"] * case["d"], sum(new)
    if case["op"] != "attend":
        return {"bytes": int((2 if case["op"] == "store" else 1) * 2 * tokens * row * (size + 17 / 32)), "flops": 0}
    pairs = cached = 0
    for length, n in zip(held, new):
        spans = [s for s in _seen(case, length, n) if s[1] > s[0]]
        pairs += sum(b - a for a, b in spans)
        cached += max(b for _, b in spans) - min(a for a, _ in spans) if spans else 0
    return {"bytes": cached * row * 17 // 16 + 4 * tokens * case["hq"] * case["d"] + (4 * tokens * case["hq"] if case["lse"] else 0),
            "flops": 4 * pairs * case["hq"] * case["d"]}


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    return {"extend": _prepare_extend, "rotary": _prepare_rotary}.get(case["op"], _prepare_cache)(case, gen)


def _ids(gen, n):
    return torch.randperm(n, generator=gen, device="cuda").to(torch.int32)


def _prepare_extend(case, gen):
    """What a server keeps of its requests between steps: their blocks and lengths, and the stack of free blocks."""
    held, new = _requests(case)
    block = case["block"]
    have = [_blocks(a, block) for a in held]
    need = sum(_blocks(a + n, block) - h for a, n, h in zip(held, new, have) if n > 0)
    back = sum(h for n, h in zip(new, have) if n < 0)
    n_free = max(0, int(need * case["spare"]) - back)
    n_blocks, width = sum(have) + n_free, max(1, max(_blocks(a + max(n, 0), block) for a, n in zip(held, new)))
    s = SimpleNamespace(case=case, block=block, width=width, n_blocks=n_blocks)
    ids = _ids(gen, max(1, n_blocks))
    ends = torch.tensor([0] + have, device="cuda").cumsum(0)
    j = torch.arange(width, device="cuda")
    s.table = torch.where(j < (ends[1:] - ends[:-1])[:, None], ids[(ends[:-1, None] + j).clamp(max=max(0, n_blocks - 1))], -1).to(torch.int32)
    s.lens, s.new = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (held, new))
    s.free = torch.full((max(1, n_blocks),), -1, dtype=torch.int32, device="cuda")
    s.free[:n_free] = ids[sum(have):sum(have) + n_free]
    s.n_free = torch.tensor([n_free], dtype=torch.int32, device="cuda")
    s.tokens, s.most = sum(max(n, 0) for n in new), max(0, max(new))
    # the step's results go beside what it begins from, as for a step that may be taken back
    s.next_lens, s.next_free = torch.empty_like(s.lens), torch.empty_like(s.n_free)
    if own:
        import paper_2203_00448_gb300 as mp

        s.blocks = mp.KvBlocks(case["seqs"], width, block, n_blocks=n_blocks, table=s.table, lens=s.lens, free=s.free, n_free=s.n_free)
    return s


def _scaling(case):
    """The scaling's own parameters, by its kind."""
    return {"none": None, "linear": {"kind": "linear", "factor": 4.0}, "base": {"kind": "base", "factor": 4.0},
            "parts": {"kind": "parts", "factor": 16.0, "original": 8192, "fast": 32.0, "slow": 1.0},
            "bands": {"kind": "bands", "factor": 8.0, "original": 8192, "low": 1.0, "high": 4.0}}[case["scaling"]]


BASE = 10000.0


def _frequencies(case):
    """Radians a position of each pair, in 64 bits, and the amplitude."""
    dim, scaling = case["dim"], _scaling(case)
    i = torch.arange(0, dim, 2, dtype=torch.float64)
    f = BASE ** (-i / dim)
    if scaling is None:
        return f, 1.0
    factor = scaling["factor"]
    if scaling["kind"] == "linear":
        return f / factor, 1.0
    if scaling["kind"] == "base":
        return (BASE * factor ** (dim / (dim - 2))) ** (-i / dim), 1.0
    turns = scaling["original"] * f / (2 * math.pi)  # that a pair makes over the original length
    if scaling["kind"] == "bands":
        keep = ((turns - scaling["low"]) / (scaling["high"] - scaling["low"])).clamp(0, 1)
        return keep * f + (1 - keep) * f / factor, 1.0
    # the pairs (by index) that turn `fast` and `slow` times are the ends of a ramp
    index = [dim * math.log(scaling["original"] / (t * 2 * math.pi)) / (2 * math.log(BASE)) for t in (scaling["fast"], scaling["slow"])]
    low, high = max(0, math.floor(index[0])), min(dim - 1, math.ceil(index[1]))
    away = ((i / 2 - low) / max(high - low, 0.001)).clamp(0, 1)
    return (1 - away) * f + away * f / factor, 0.1 * math.log(factor) + 1


def _prepare_rotary(case, gen):
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["tokens"]
    dt = TYPES[case["dtype"]]
    s = SimpleNamespace(case=case)
    width = hq + 2 * hkv if case["packed"] else hq + hkv
    x = torch.randn(n, width * d, generator=gen, device="cuda").to(dt)
    if case["packed"]:
        s.q, s.k = (p.view(n, -1, d) for p in x.split([hq * d, hkv * d, hkv * d], dim=1)[:2])
    else:
        s.q, s.k = x[:, :hq * d].contiguous().view(n, hq, d), x[:, hq * d:].contiguous().view(n, hkv, d)
    # runs of neighbours, as prompts have them, from anywhere in the context
    run = torch.randint(0, case["far"], (n // 100 + 1,), generator=gen, device="cuda")
    at = torch.arange(n, device="cuda")
    s.positions = ((run[at // 100] + at % 100) % case["far"]).to(torch.int32)
    frequencies, s.amplitude = _frequencies(case)
    s.frequencies = frequencies.cuda()
    if own:
        import paper_2203_00448_gb300 as mp

        s.rotary = mp.Rotary(case["dim"], base=BASE, layout=case["layout"], scaling=_scaling(case))
    return s


def _prepare_cache(case, gen):
    """The pool with what the sequences hold, their tables (blocks in no order, -1 past the end), and the new tokens."""
    held, new = _lengths(case)
    block, hkv, hq, d = case["block"], case["hkv"], case["hq"], case["d"]
    dt = TYPES[case["dtype"]]
    cols = [_blocks(length, block) for length in held]
    n_blocks, width = max(1, sum(cols)), max(1, max(cols))
    s = SimpleNamespace(case=case, held=held, new=new, width=width)
    shuffled = _ids(gen, n_blocks)
    ends = torch.tensor([0] + cols, device="cuda").cumsum(0)
    j = torch.arange(width, device="cuda")
    there = j < (ends[1:] - ends[:-1])[:, None]
    s.table = torch.where(there, shuffled[(ends[:-1, None] + j).clamp(max=n_blocks - 1)], -1).to(torch.int32)
    s.lens = torch.tensor(held, dtype=torch.int32, device="cuda")
    s.token_ptr = torch.tensor([0] + new, device="cuda").cumsum(0)
    s.tokens, s.most = sum(new), max(new)

    # codes of about normal values under scales of a few sizes, one group of the keys' values larger than the others
    groups = d // GROUP
    s.k, s.v = (torch.empty(n_blocks, hkv, block // GROUP, 17 * d, dtype=torch.uint8, device="cuda") for _ in range(2))
    for pool in (s.k, s.v):
        step = max(1, (1 << 26) // (hkv * block * d))
        for at in range(0, n_blocks, step):
            some = pool[at:at + step]
            x = torch.randn(*some.shape[:3], 16 * d, 2, generator=gen, device="cuda").mul_(2.6).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
            some[..., :16 * d] = x[..., 0] | x[..., 1] << 4
            some[..., 16 * d:] = torch.randint(80, 104, some[..., 16 * d:].shape, generator=gen, device="cuda", dtype=torch.uint8)
        if pool is s.k:
            pool[..., 16 * d:].view(*pool.shape[:3], 8, groups, 4)[..., 1, :] += 12
    # slots past a sequence's end hold anything, here bytes that stand for no number
    b = torch.tensor([b for b, length in enumerate(held) for _ in range(cols[b] * block - length)], dtype=torch.int64, device="cuda")
    at = torch.tensor([p for b, length in enumerate(held) for p in range(length, cols[b] * block)], dtype=torch.int64, device="cuda")
    if at.numel():
        page, granule, t = s.table[b, at // block].long(), at % block // GROUP, at % GROUP
        s.k[..., 16 * d:].view(n_blocks, hkv, -1, 8, groups, 4)[page, :, granule, t % 8, :, t // 8] = 0xFF
        s.v[..., 16 * d:].view(n_blocks, hkv, -1, groups, 4, 4, 2)[page, :, granule, :, t // 2 % 4, t // 8, t % 2] = 0xFF
    s.k, s.v = (pool.view(n_blocks, hkv, -1) for pool in (s.k, s.v))

    size = {"store": 2 * hkv, "read": 0, "attend": hq}[case["op"]]
    if size:
        heads = (hq, hkv, hkv) if case["packed"] else (hq, 0, 0) if case["op"] == "attend" else (0, hkv, hkv)
        if case["packed"]:
            parts = torch.randn(s.tokens, sum(heads) * d, generator=gen, device="cuda").to(dt).split([h * d for h in heads], dim=1)
        else:
            parts = [torch.randn(s.tokens, h * d, generator=gen, device="cuda").to(dt) for h in heads]
        s.q, s.new_k, s.new_v = (p.view(s.tokens, -1, d) if p.numel() else None for p in parts)
    s.scale = 1 / math.sqrt(d)
    if own:
        import paper_2203_00448_gb300 as mp

        s.cache = mp.KvCache4(n_blocks, block, hkv, d, k=s.k, v=s.v)
        s.batch = mp.KvBatch(s.table, s.lens, s.token_ptr, n_tokens=s.tokens, max_tokens=s.most, max_len=max(held))
    return s


def run(s):
    c = s.case
    if own:
        import paper_2203_00448_gb300 as mp

        if c["op"] == "extend":
            step = mp.kv_extend(s.blocks, s.new, n_tokens=s.tokens, max_tokens=s.most, lens=s.next_lens, n_free=s.next_free)
            return {"table": s.table, "lens": s.next_lens, "n_free": s.next_free, "free": s.free, "step_lens": step.batch.lens,
                    "token_ptr": step.batch.token_ptr, "positions": step.positions, "slots": step.slots, "status": step.status}
        if c["op"] == "rotary":
            return mp.rotary(s.rotary, s.positions, s.q, s.k, inverse=c["inverse"])
        if c["op"] == "store":
            mp.kv_write(s.cache, s.batch, s.new_k, s.new_v)
            return mp.kv_read(s.cache, s.batch, dtype=TYPES[c["dtype"]])[:2]
        if c["op"] == "read":
            return mp.kv_read(s.cache, s.batch, dtype=TYPES[c["dtype"]])[:2]
        return mp.kv_attend(s.cache, s.batch, s.q, scale=s.scale, causal=c["causal"], window=c["window"], want_lse=c["lse"])[:2]
    return {"extend": _extend, "rotary": _rotary, "store": _store, "read": _read, "attend": _attend}[c["op"]](s)


# The plain forms.


def _extend(s):
    """Done requests push their blocks, in order; the others take theirs from the top, as long as those before them got theirs."""
    block, old, new = s.block, s.lens.long(), s.new.long()
    take = new.clamp(min=0)
    ptr = torch.cat([take.new_zeros(1), take.cumsum(0)])
    have = (old + block - 1) // block
    done = new < 0
    need = torch.where(done, 0, (old + take + block - 1) // block - have)
    j = torch.arange(s.width, device=old.device)
    back = done[:, None] & (j < have[:, None])
    place = torch.where(back, s.n_free + (back.flatten().cumsum(0) - 1).view_as(back), 0)
    at, row = back.nonzero(as_tuple=True)
    s.free[place[at, row]] = s.table[at, row]
    top = s.n_free.long() + back.sum()
    want = need.cumsum(0)
    fine = done | (need == 0) | (want <= top)
    given = torch.where(fine, need, 0)
    s.next_free.copy_(top - given.sum())
    # column j of a request is new where its blocks end before it
    k = (want - need)[:, None] + j - have[:, None]
    fresh = fine[:, None] & ~done[:, None] & (j >= have[:, None]) & (j < (have + need)[:, None])
    picked = s.free[(top - 1 - k).clamp(0, len(s.free) - 1)]
    s.table.copy_(torch.where(fresh, picked, s.table))
    s.next_lens.copy_(torch.where(done, 0, torch.where(fine, old + take, old)))
    step = torch.where(fine & ~done, old + take, -1).to(torch.int32)
    seq = torch.repeat_interleave(torch.arange(len(old), device=old.device), take, output_size=s.tokens)
    at = old[seq] + torch.arange(s.tokens, device=old.device) - ptr[seq]
    slot = s.table[seq, (at // block).clamp(max=s.width - 1)].long() * block + at % block
    there = fine[seq]
    return {"table": s.table, "lens": s.next_lens, "n_free": s.next_free, "free": s.free, "step_lens": step, "token_ptr": ptr,
            "positions": torch.where(there, at, -1).to(torch.int32), "slots": torch.where(there, slot, -1),
            "status": torch.where(fine, 0, 5).to(torch.int32)}


def _rotary(s):
    c = s.case
    dim = c["dim"]
    angle = s.positions[:, None].double() * s.frequencies
    cos, sin = (f(angle).mul(s.amplitude).float()[:, None] for f in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin
    out = []
    for x in (s.q, s.k):
        y = x.float()
        a, b = (y[..., :dim // 2], y[..., dim // 2:dim]) if c["layout"] == "half" else (y[..., :dim:2], y[..., 1:dim:2])
        turned = a * cos - b * sin, a * sin + b * cos
        turned = torch.cat(turned, -1) if c["layout"] == "half" else torch.stack(turned, -1).flatten(-2)
        out.append(torch.cat([turned, y[..., dim:]], -1).to(x.dtype))
    return tuple(out)


def _scale_of(byte):
    """What a scale's bytes stand for: 5 bits of exponent and 3 of fraction, those of an f16."""
    return (byte.to(torch.int16) << 7).view(torch.float16).float()


def _values(pool, block, d, keys):
    """A pool's (or some of its blocks') values as [blocks, heads, tokens, d]."""
    n, h = pool.shape[:2]
    pool = pool.view(n, h, block // GROUP, 17 * d)
    code, scale = pool[..., :16 * d], _scale_of(pool[..., 16 * d:])
    code = torch.stack([code & 15, code >> 4], -1).float() - 8
    groups = d // GROUP
    if keys:  # a token's codes lie in a row; scales as [token % 8][group][token / 8]
        code = code.view(n, h, -1, GROUP, d)
        scale = scale.view(n, h, -1, 8, groups, 4).permute(0, 1, 2, 5, 3, 4)
    else:  # codes as [token / 8][d / (D / 8)][token / 2 % 4][d / 4][token % 2][d % 4]; scales as [group][token / 2 % 4][token / 8][token % 2]
        code = code.view(n, h, -1, 4, 8, 4, groups, 2, 4).permute(0, 1, 2, 3, 5, 7, 4, 6, 8)
        scale = scale.view(n, h, -1, groups, 4, 4, 2).permute(0, 1, 2, 5, 4, 6, 3)
    scale = scale.reshape(n, h, -1, GROUP, groups)[..., None]
    return (code.reshape(n, h, -1, GROUP, groups, GROUP) * scale).reshape(n, h, block, d)


def _places(s):
    """Every new token's sequence, pool block and slot."""
    new, block = s.token_ptr[1:] - s.token_ptr[:-1], s.case["block"]
    seq = torch.repeat_interleave(torch.arange(len(s.new), device=s.lens.device), new, output_size=s.tokens)
    at = torch.arange(s.tokens, device=s.lens.device) - s.token_ptr[seq] + (s.lens - new)[seq]
    return s.table[seq, at // block].long(), at % block


def _quantised(x):
    """Codes [tokens, heads, groups, 32] and the scales' bytes [tokens, heads, groups] of values."""
    n, h, d = x.shape
    x = x.double().view(n, h, d // GROUP, GROUP)
    most = x.abs().amax(-1)
    grid = _scale_of(torch.arange(184, device=x.device, dtype=torch.uint8)).double()
    byte = torch.bucketize(most, 7.5 * grid).clamp(max=183)  # the least scale with most <= 7.5 of it
    code = torch.round(x / torch.where(byte > 0, grid[byte], 1.0)[..., None]).clamp(-7, 7)
    return (torch.where(byte[..., None] > 0, code, 0) + 8).to(torch.uint8), byte.to(torch.uint8)


def _store(s):
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    page, slot = _places(s)
    granule, t = slot // GROUP, slot % GROUP
    n_blocks, groups = s.k.shape[0], d // GROUP
    for pool, x, keys in ((s.k, s.new_k, True), (s.v, s.new_v, False)):
        code, byte = _quantised(x)
        code = code.view(s.tokens, hkv, d // 2, 2)
        code = code[..., 0] | code[..., 1] << 4  # two neighbours in a byte
        pool = pool.view(n_blocks, hkv, block // GROUP, 17 * d)
        codes, scales = pool[..., :16 * d], pool[..., 16 * d:]
        if keys:
            codes.view(n_blocks, hkv, -1, GROUP, d // 2)[page, :, granule, t] = code
            scales.view(n_blocks, hkv, -1, 8, groups, 4)[page, :, granule, t % 8, :, t // 8] = byte
        else:
            codes = codes.view(n_blocks, hkv, -1, 4, 8, 4, groups, 2, 2)
            codes[page, :, granule, t // 8, :, t // 2 % 4, :, t % 2] = code.view(s.tokens, hkv, 8, groups, 2)
            scales.view(n_blocks, hkv, -1, groups, 4, 4, 2)[page, :, granule, :, t // 2 % 4, t // 8, t % 2] = byte
    return _read(s)


def _read(s):
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    page, slot = _places(s)
    granule, t = slot // GROUP, slot % GROUP
    n_blocks, groups = s.k.shape[0], d // GROUP
    out = []
    for pool, keys in ((s.k, True), (s.v, False)):
        pool = pool.view(n_blocks, hkv, block // GROUP, 17 * d)
        codes, scales = pool[..., :16 * d], pool[..., 16 * d:]
        if keys:
            code = codes.view(n_blocks, hkv, -1, GROUP, d // 2)[page, :, granule, t]
            byte = scales.view(n_blocks, hkv, -1, 8, groups, 4)[page, :, granule, t % 8, :, t // 8]
        else:
            code = codes.view(n_blocks, hkv, -1, 4, 8, 4, groups, 2, 2)[page, :, granule, t // 8, :, t // 2 % 4, :, t % 2]
            byte = scales.view(n_blocks, hkv, -1, groups, 4, 4, 2)[page, :, granule, :, t // 2 % 4, t // 8, t % 2]
        code = code.reshape(s.tokens, hkv, d // 2)
        code = torch.stack([code & 15, code >> 4], -1).float() - 8
        x = code.view(s.tokens, hkv, groups, GROUP) * _scale_of(byte)[..., None]
        out.append(x.reshape(s.tokens, hkv, d).to(TYPES[c["dtype"]]))
    return tuple(out)


def _attend(s):
    c = s.case
    block, d, hkv, hq, n = c["block"], c["d"], c["hkv"], c["hq"], s.most
    group, seqs = hq // hkv, c["seqs"]
    pages = s.table.clamp(min=0).long()
    full = s.width * block
    k, v = (_values(pool[pages].flatten(0, 1), block, d, pool is s.k).view(seqs, -1, hkv, block, d) for pool in (s.k, s.v))
    k, v = (x.transpose(1, 2).reshape(seqs, hkv, full, d) for x in (k, v))
    new = s.token_ptr[1:] - s.token_ptr[:-1]
    seq = torch.repeat_interleave(torch.arange(seqs, device=new.device), new, output_size=s.tokens)
    i = torch.arange(s.tokens, device=seq.device) - s.token_ptr[seq]
    q = torch.zeros(seqs, n, hq, d, device=seq.device)
    q[seq, i] = s.q.float()
    q = q.view(seqs, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, group * n, d)
    j = torch.arange(full, device=seq.device)
    sees = (j < s.lens[:, None])[:, None, :].expand(seqs, n, full)
    v = torch.where(sees[:, :1, :, None], v, 0)
    if c["causal"]:
        place = (s.lens - new)[:, None] + torch.arange(n, device=seq.device)
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


def _held(s, b, first, past, keys):
    """Positions [first, past) of sequence b as stored, in 64 bits: [tokens, heads, d]."""
    c = s.case
    block, d, hkv = c["block"], c["d"], c["hkv"]
    at = torch.arange(first, past, device=s.lens.device)
    page, t = s.table[b, at // block].long()[:, None, None], (at % block)[:, None, None]
    h, i = torch.arange(hkv, device=at.device)[:, None], torch.arange(d, device=at.device)
    base, t = t // 32 * 17 * d, t % 32
    if keys:
        where, scale = t * (d // 2) + i // 2, t % 8 * (d // 8) + i // 32 * 4 + t // 8
    else:
        e = d // 8
        where = ((t // 8 * 8 + i // e) * 4 + t % 8 // 2) * e + i % e // 4 * 4 + t % 2 * 2 + i % 4 // 2
        scale = (i // 32 * 4 + t // 2 % 4) * 8 + t // 8 * 2 + t % 2
    pool = s.k if keys else s.v
    code = pool[page, h, base + where].long() >> (i % 2 * 4) & 15
    byte = pool[page, h, base + 16 * d + scale].long()
    exponent, part = byte >> 3, (byte & 7).double() / 8
    size = torch.where(exponent > 0, (1 + part) * torch.exp2((exponent - 15).double()), part * 2.0 ** -14)
    return (code - 8).double() * size


def _stored(x):
    """What 4 bits hold of [tokens, heads, d] values."""
    x = x.double().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    # steps of an eighth of a power of two, of 2^-17 below 2^-14
    least = most / 7.5
    _, e = torch.frexp(least)
    step = torch.exp2((e - 4).clamp(min=-17).double())
    scale = (torch.ceil(least / step) * step).clamp(max=240.0)
    code = torch.round(x / torch.where(scale > 0, scale, 1)).clamp(-7, 7)
    return (code * scale).flatten(-2)


def exact(case, seed):
    if case["op"] == "extend":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(s)
    if case["op"] == "store":
        return _stored(s.new_k), _stored(s.new_v)
    if case["op"] == "read":
        return tuple(torch.cat([_held(s, b, length - n, length, keys) for b, (length, n) in enumerate(zip(s.held, s.new))])
                     for keys in (True, False))
    return _exact_attend(s)


def _exact_rotary(s):
    c = s.case
    dim, way = c["dim"], -1 if c["inverse"] else 1
    frequencies, amplitude = _frequencies(c)
    out = []
    for x in (s.q, s.k):
        y = x.double().clone()
        for i, f in enumerate(frequencies.tolist()):
            a, b = (i, i + dim // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            angle = (way * f * s.positions.double())[:, None]
            z = torch.complex(x[..., a].double(), x[..., b].double()) * torch.polar(torch.full_like(angle, amplitude), angle)
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
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
        k, v = (_held(s, b, 0, length, keys) for keys in (True, False))
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
