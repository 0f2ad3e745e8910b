"""Block tables from request lengths and rotary positions against plain implementations, and steps of all the operators that
a server calls together."""
import numpy as np
import pytest
import torch

from tests import kv4_refs as R4

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def run_extend(mp, table, lens, new, block, n_tokens, max_tokens, max_len, free=None, n_free=0, n_blocks=0, first=None, room=None,
               inplace=True):
    dev = lambda x: None if x is None else torch.tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    kw = dict(first=dev(first), room=dev(room)) if first is not None else dict(free=dev(free), n_free=dev([n_free]))
    blocks = mp.KvBlocks(len(lens), table.shape[1], block, n_blocks, table=dev(table), lens=dev(lens).reshape(-1), **kw)
    outs = {} if inplace else dict(lens=torch.empty_like(blocks.lens), n_free=None if first is not None else torch.empty_like(blocks.n_free))
    step = mp.KvStep(blocks, n_tokens, max_tokens, max_len)
    step.positions.fill_(-77), step.slots.fill_(-77)
    got = mp.kv_extend(blocks, dev(new).reshape(-1), n_tokens, max_tokens, max_len, step=step, **outs)
    assert got is step
    want_table, want_free = table.copy(), None if free is None else np.array(free, np.int32)
    want = R4.extend(want_table, lens, new, block, n_tokens, max_tokens, max_len, want_free, n_free, n_blocks, first, room)
    after = blocks.lens if inplace else outs["lens"]
    assert step.status.tolist() == want["status"]
    assert after.tolist() == want["lens"] and step.batch.lens.tolist() == want["step_lens"]
    assert np.array_equal(step.batch.token_ptr.cpu().numpy(), want["token_ptr"])
    assert np.array_equal(step.positions.cpu().numpy(), want["positions"])
    assert np.array_equal(step.slots.cpu().numpy(), want["slots"])
    if first is None:
        assert (blocks.n_free if inplace else outs["n_free"]).item() == want["n_free"]
        assert np.array_equal(blocks.free.cpu().numpy(), want_free)
        if not inplace:
            assert blocks.n_free.item() == n_free and blocks.lens.tolist() == list(lens)
    assert np.array_equal(blocks.table.cpu().numpy(), want_table)
    return want


def requests(rng, B, block, len_hi, n_hi, ends, spare, width=None):
    lens = rng.integers(0, len_hi + 1, B)
    new = np.where(rng.random(B) < ends, -rng.integers(1, 4, B), rng.integers(0, n_hi + 1, B))
    have = -(-lens // block)
    need = -(-(lens + np.maximum(new, 0)) // block) - have
    width = width or max(1, int((have + need).max(initial=0)))
    n_free = int(need.sum() * spare)
    n_blocks = int(have.sum()) + n_free
    ids = rng.permutation(n_blocks)
    table, at = np.full((B, width), -5, np.int32), 0
    for b in range(B):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    free = np.full(n_blocks, -9, np.int32)
    free[:n_free] = ids[at:]
    return table, [int(x) for x in lens], [int(x) for x in new], free, n_free, n_blocks


@pytest.mark.parametrize("B,block,len_hi,n_hi,ends,spare", [
    (1, 32, 0, 1, 0, 1), (1, 64, 100, 70, 0, 1), (7, 32, 200, 1, 0.3, 1), (64, 64, 2000, 1, 0.1, 0.5), (33, 96, 500, 90, 0.2, 0.7),
    (1024, 32, 90, 2, 0.1, 0.9), (1025, 32, 300, 3, 0.5, 0.2), (3000, 128, 400, 12, 0.2, 0.6), (200, 32, 3000, 500, 0.05, 0.9),
    (3, 256, 100000, 20000, 0.4, 1.2), (40, 32, 64, 33, 1.0, 1)])
@pytest.mark.parametrize("inplace", [True, False])
def test_extend(cuda_lib, B, block, len_hi, n_hi, ends, spare, inplace):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(B + block)
    for _ in range(2):
        table, lens, new, free, n_free, n_blocks = requests(rng, B, block, len_hi, n_hi, ends, spare)
        total, most = sum(max(n, 0) for n in new), max(0, max(new))
        run_extend(mp, table, lens, new, block, total + 3, most, table.shape[1] * block, free, n_free, n_blocks, inplace=inplace)


@pytest.mark.parametrize("B,n_hi", [(9, 3), (700, 40)])
def test_extend_runs_of_a_plan(cuda_lib, B, n_hi):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(B)
    lens, new = rng.integers(0, 300, B), rng.integers(-1, n_hi, B)
    room = rng.integers(1, 12, B)
    lens = np.minimum(lens, room * 32)
    first = np.concatenate([[0], np.cumsum(room)[:-1]])
    first[1], first[2] = -1, int(room.sum()) - 1
    run_extend(mp, np.full((B, 14), -5, np.int32), lens.tolist(), new.tolist(), 32, int(np.maximum(new, 0).sum()), n_hi, 14 * 32,
               first=first.tolist(), room=room.tolist(), n_blocks=int(room.sum()))


@pytest.mark.parametrize("many", [False, True])
def test_extend_refuses_requests_one_by_one(cuda_lib, many):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(3)
    table, lens, new, free, n_free, n_blocks = requests(rng, 60, 32, 400, 200 if many else 5, 0.2, 0.8, width=20)
    total = sum(max(n, 0) for n in new)
    lens[3], lens[4], lens[50] = -1, 20 * 32 + 1, 2 ** 31 - 1
    new[7] = 2 ** 31 - 1
    args = (32, total, 200 if many else 5, 20 * 32 - 8, free, n_free, n_blocks)
    run_extend(mp, table, lens, new, *args)
    new[7] = 201 if many else 6  # above max_tokens; rows of the last requests are past n_tokens
    want = run_extend(mp, table, lens, new, *args)
    assert 1 in want["status"] and 0 in want["status"]
    for bad in (-1, n_blocks + 1, 2 ** 31 - 1, -2 ** 31):  # a stack of no such height: nobody is answered
        want = run_extend(mp, table, lens, new, *args[:4], free, bad, n_blocks)
        assert set(want["status"]) == {1}
    # a request that ends may have held more than the step's others may
    new[7] = 0
    long, gone = [a if 0 <= a <= 640 else 0 for a in lens], list(new)
    most = max(range(60), key=lambda b: long[b])
    gone[most] = -1
    want = run_extend(mp, table, long, gone, 32, sum(max(n, 0) for n in gone), 200 if many else 5, long[most] - 1, free, n_free, n_blocks)
    assert want["status"][most] == 0 and want["lens"][most] == 0
    # blocks that come back to a stack that is full already
    done = [-1 if a > 0 else 0 for a in lens]
    want = run_extend(mp, table, lens, done, *args[:4], free, n_blocks - 3, n_blocks)
    assert want["n_free"] <= n_blocks and 1 in want["status"]


def test_extend_of_nothing(cuda_lib):
    """No requests, requests without tokens or columns, and a pool without blocks."""
    import paper_2203_00448_gb300 as mp

    run_extend(mp, np.zeros((0, 3), np.int32), [], [], 32, 0, 0, 96, np.zeros(0, np.int32), 0, 0)
    for n_tokens in (0, 5, 5000):
        run_extend(mp, np.zeros((3, 0), np.int32), [0, 0, 0], [0, -1, 2], 32, n_tokens, 2, 0, np.zeros(0, np.int32), 0, 0)
        run_extend(mp, np.zeros((3, 2), np.int32), [0, 0, 0], [0, -1, 2], 32, n_tokens, 2, 64, np.zeros(0, np.int32), 0, 0)


def test_extend_step_after_step(cuda_lib):
    """Requests come, grow and go in a pool that is sometimes short; no block is ever anybody's twice."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(8)
    B, block, cols, n_blocks = 24, 32, 6, 60
    blocks = mp.KvBlocks(B, cols, block, n_blocks)
    held, refused = np.zeros(B, int), 0
    for _ in range(60):
        new = np.where(held > 0, np.where(rng.random(B) < 0.15, -1, rng.integers(0, 4, B)), rng.integers(0, 80, B))
        new = np.minimum(new, cols * block - held)
        step = mp.kv_extend(blocks, torch.from_numpy(new.astype(np.int32)).cuda(), int(np.maximum(new, 0).sum()))
        status = step.status.cpu().numpy()
        assert set(status) <= {0, 5}
        refused += int((status == 5).sum())
        held = np.where(status != 0, held, np.where(new < 0, 0, held + new))
        assert np.array_equal(blocks.lens.cpu().numpy(), held)
        table, n_free = blocks.table.cpu().numpy(), blocks.n_free.item()
        mine = [table[b, :-(-held[b] // block)] for b in range(B)] + [blocks.free.cpu().numpy()[:n_free]]
        assert np.array_equal(np.sort(np.concatenate(mine)), np.arange(n_blocks))
    assert refused


CASES = [
    # tokens, q heads, k heads, head_dim, dim, layout, dtype, rows
    (1, 8, 2, 128, 128, "half", "bf16", "plain"), (5, 4, 4, 64, 64, "interleaved", "f16", "plain"),
    (9, 3, 1, 64, 32, "half", "f32", "packed"), (33, 2, 2, 128, 40, "interleaved", "bf16", "packed"),
    (17, 5, 1, 128, 40, "half", "f16", "plain"), (4, 2, 1, 128, 2, "half", "f32", "plain"), (3, 1, 1, 6, 4, "interleaved", "bf16", "plain"),
    (7, 6, 2, 80, 80, "half", "f32", "odd"), (6, 2, 3, 128, 128, "interleaved", "bf16", "odd"), (11, 1, 0, 256, 64, "half", "f16", "heads"),
    (2500, 1, 1, 64, 48, "interleaved", "f32", "plain"), (2, 0, 3, 1024, 1024, "half", "bf16", "plain"),
]


def layout_rows(x, how):
    n, h, d = x.shape
    if how == "packed":
        return torch.cat([torch.zeros_like(x[:, :1]), x, x[:, :1]], 1)[:, 1:1 + h]
    if how == "odd":
        return torch.nn.functional.pad(x.reshape(n, -1), (1, 2))[:, 1:1 + h * d].view(n, h, d)
    return x.transpose(0, 1).contiguous().transpose(0, 1) if how == "heads" else x


@pytest.mark.parametrize("n,hq,hk,d,dim,layout,dtype,how", CASES)
def test_rotary(cuda_lib, n, hq, hk, d, dim, layout, dtype, how):
    """Both ways, out of place and in place.  A product of two numbers of 24 bits (x, and a cosine that is off by 2^-23 at most:
    the argument's rounding of 2^-25 of a turn's eighth times pi, the function's two and the amplitude's) and their sum: 2^-21 of
    the pair's size, and half a step of the output's type."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(n + d)
    positions = rng.choice([0, 1, 7, 4095, 131071, 10 ** 6 + 1, 2 ** 28 - 1, 2 ** 31 - 1, -3], n).astype(np.int32)
    if n > 100:
        positions = np.arange(n, dtype=np.int32)
    scaling = {"kind": "parts", "factor": 8.0, "original": 4096, "fast": 32.0, "slow": 1.0} if dim >= 40 else None
    r = mp.Rotary(dim, layout=layout, scaling=scaling)
    t = TYPES[dtype]
    q, k = (None if not h else layout_rows(torch.from_numpy(rng.standard_normal((n, h, d)) * 3).to(t).cuda(), how) for h in (hq, hk))
    at = torch.from_numpy(positions).cuda()
    keep = [None if x is None else x.double().cpu().numpy() for x in (q, k)]
    for inverse in (False, True):
        outs = mp.rotary(r, at, q, k, inverse=inverse)
        for x, had, out in zip((q, k), keep, outs):
            if x is None:
                assert out is None
                continue
            some = slice(None) if n < 100 else slice(n - 60, n)
            want = R4.rotary(had[some], positions[some], r.frequencies.tolist(), r.amplitude, layout, inverse)
            got = out.double().cpu().numpy()[some]
            pairs = np.abs(want).copy()
            a, b = (slice(0, dim // 2), slice(dim // 2, dim)) if layout == "half" else (slice(0, dim, 2), slice(1, dim, 2))
            pairs[..., a] = pairs[..., b] = np.hypot(want[..., a], want[..., b])
            bound = pairs * 2.0 ** -21 + np.abs(want) * torch.finfo(t).eps / 2 + torch.finfo(t).tiny
            assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / bound)
            assert np.array_equal(got[..., dim:], had[some][..., dim:])
            assert torch.equal(x.double().cpu(), torch.from_numpy(had))
        a, b = (None if x is None else layout_rows(x.clone(), how) for x in (q, k))
        mp.rotary(r, at, a, b, q_out=a, k_out=b, inverse=inverse)
        for x, y in zip((a, b), outs):
            assert x is None or torch.equal(x, y)


def test_rotary_gradient(cuda_lib):
    """The call with inverse=True on the outputs' gradients against differences of the call itself: it is linear, so a difference
    over a step of 1 has no error but the roundings (three of 2^-24 a product, terms of size up to 4, sums of 2 x 3 x 32 x 2)."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(2)
    for layout in ("half", "interleaved"):
        r = mp.Rotary(24, layout=layout, amplitude=1.25)
        x, w = (torch.from_numpy(rng.standard_normal((2, 3, 32))).float().cuda() for _ in range(2))
        at = torch.tensor([5, 70000], dtype=torch.int32, device="cuda")
        grad = mp.rotary(r, at, w, inverse=True)[0]
        base = (mp.rotary(r, at, x)[0].double() * w).sum()
        for i in ((0, 0, 0), (1, 2, 23), (0, 1, 13), (1, 0, 30), (1, 1, 6)):
            y = x.clone()
            y[i] += 1
            step = (y[i] - x[i]).double()
            difference = ((mp.rotary(r, at, y)[0].double() * w).sum() - base) / step
            assert abs(difference - grad[i]) <= 192 * 3 * 4 * 2.0 ** -24


def test_rotary_past_32_bit_offsets(cuda_lib):
    """Rows that are 2^30 values apart."""
    import paper_2203_00448_gb300 as mp

    wide = torch.empty(3, 1 << 30, dtype=torch.bfloat16, device="cuda")
    x = wide[:, 40:104].view(3, 1, 64)
    x.copy_(torch.randn(3, 1, 64, device="cuda"))
    r, at = mp.Rotary(64), torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    want = mp.rotary(r, at, x.contiguous())[0]
    assert torch.equal(mp.rotary(r, at, x)[0], want)
    mp.rotary(r, at, x, q_out=x)
    assert torch.equal(x, want)


def test_rotary_captured_and_on_another_stream(cuda_lib):
    import paper_2203_00448_gb300 as mp

    r = mp.Rotary(64)
    x = torch.randn(20, 4, 64, device="cuda")
    at = torch.arange(20, dtype=torch.int32, device="cuda")
    want = mp.rotary(r, at, x)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = mp.rotary(r, at, x, stream=s)[0]
    s.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        z = mp.rotary(r, at, x)[0]
    at += 3
    g.replay()
    assert torch.equal(z, mp.rotary(r, at, x)[0]) and not torch.equal(z, want)
    assert mp.rotary(r, at[:0], x[:0])[0].shape == (0, 4, 64)


@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_of_no_heads(cuda_lib, inverse):
    """Queries or keys without heads leave the other to be turned, as a call without them does."""
    import paper_2203_00448_gb300 as mp

    r, at = mp.Rotary(64, layout="interleaved"), torch.arange(5, 12, dtype=torch.int32, device="cuda")
    x = torch.randn(7, 3, 64, device="cuda")
    want = mp.rotary(r, at, x, inverse=inverse)[0]
    assert not torch.equal(want, x)
    none = x[:, :0]
    for q, k in ((none, x), (x, none)):
        outs = mp.rotary(r, at, q, k, inverse=inverse)
        assert [y.shape for y in outs] == [q.shape, k.shape] and torch.equal(outs[0] if k is none else outs[1], want)
    y = x.clone()
    mp.rotary(r, at, none, y, q_out=none, k_out=y, inverse=inverse)
    assert torch.equal(y, want)
    assert [y.shape for y in mp.rotary(r, at, none, none)] == [none.shape] * 2


@pytest.mark.parametrize("bits", [4, 8])
def test_steps_together(cuda_lib, bits):
    """What a server does each step: blocks, positions, rotated queries and keys, the cache, attention; against plain attention
    over the tokens themselves as the cache holds them, and captured."""
    import paper_2203_00448_gb300 as mp
    from tests import kv_refs as R

    rng = np.random.default_rng(bits)
    B, block, heads, group, d = 5, 32, 2, 3, 64
    cache = (mp.KvCache4 if bits == 4 else mp.KvCache)(40, block, heads, d)
    blocks, r = mp.KvBlocks(B, 12, block, 40), mp.Rotary(d, layout="interleaved")
    held = np.zeros(B, int)
    graph = fixed = None
    for turn in range(12):
        new = np.ones(B, int) if turn else np.array([40, 1, 33, 64, 100])
        if turn == 3:
            new[2] = -1
        if turn == 4:
            new[2] = 20
        n = int(np.maximum(new, 0).sum())
        q, k, v = (torch.from_numpy(rng.standard_normal((n, h, d))).to(torch.bfloat16).cuda() for h in (heads * group, heads, heads))
        start = held.copy()
        held = np.where(new < 0, 0, held + new)
        if turn >= 6:  # the same sizes from here on: one graph
            if graph is None:
                count = torch.ones(B, dtype=torch.int32, device="cuda")
                fixed = [x.clone() for x in (q, k, v)]
                graph = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(graph):
                    step = mp.kv_extend(blocks, count, n)
                    qr, kr = mp.rotary(r, step.positions, fixed[0], fixed[1])
                    wrote = mp.kv_write(cache, step.batch, kr, fixed[2])
                    out, _, status = mp.kv_attend(cache, step.batch, qr)
            for x, y in zip(fixed, (q, k, v)):
                x.copy_(y)
            graph.replay()
        else:
            step = mp.kv_extend(blocks, torch.from_numpy(new.astype(np.int32)).cuda(), n)
            qr, kr = mp.rotary(r, step.positions, q, k)
            wrote = mp.kv_write(cache, step.batch, kr, v)
            out, _, status = mp.kv_attend(cache, step.batch, qr)
        gone = (new < 0).astype(int).tolist()
        assert step.status.tolist() == [0] * B and wrote.tolist() == gone and status.tolist() == gone
        assert step.positions.tolist() == [start[b] + i for b in range(B) for i in range(max(new[b], 0))]
        # the plain form over what the slots of each request hold
        whole = mp.KvBatch(blocks.table, blocks.lens, torch.from_numpy(np.concatenate([[0], np.cumsum(held)])).cuda(), int(held.sum()))
        kk, vv, _ = mp.kv_read(cache, whole, torch.float32)
        row = past = 0
        for b in range(B):
            m = max(new[b], 0)
            K, V = (x[past:past + held[b]].double().repeat_interleave(group, 1).transpose(0, 1) for x in (kk, vv))
            x = qr[row:row + m].double().transpose(0, 1) @ K.transpose(1, 2) * d ** -0.5
            x = x.masked_fill(torch.arange(held[b], device="cuda") > (start[b] + torch.arange(m, device="cuda"))[:, None], -torch.inf)
            w = torch.softmax(x, -1)
            want, mag = (w @ V).transpose(0, 1).cpu().numpy(), (w @ V.abs()).transpose(0, 1).cpu().numpy()
            lse = torch.logsumexp(x, -1).transpose(0, 1).cpu().numpy()
            size = ((qr[row:row + m].double().abs().transpose(0, 1) @ K.abs().transpose(1, 2)).amax(-1) * d ** -0.5).transpose(0, 1).cpu().numpy() \
                if held[b] else np.zeros(lse.shape)
            if m:
                bound, _ = R.attend_bounds(torch.bfloat16, want, lse, mag, size)
                assert (np.abs(out[row:row + m].double().cpu().numpy() - want) <= bound).all()
            row, past = row + m, past + held[b]


def test_example_serves_from_four_bits(cuda_lib):
    """The example's loop over the 4-bit cache; bounds as for 8 bits: bf16's last rounding, 2^-9, and the weights' 2^-11."""
    from examples.serve_requests import serve

    done = serve(n=12, prompt=150, generate=8, spread=15, heads=2, group=4, dim=64, block_tokens=32, check=True, bits=4)
    assert done["pool_blocks"] < done["blocks"] and 0 < done["worst"] <= 2.0 ** -9 + 2.0 ** -11
