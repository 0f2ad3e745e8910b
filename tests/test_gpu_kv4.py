"""The cache in 4 bits against plain 64-bit implementations: lengths of 0 and 1, blocks that end inside a granule, pairs of
tokens of which one is new, values beside rounding borders, slots full of bytes that stand for no number."""
import numpy as np
import pytest
import torch

from tests import kv4_refs as R4
from tests import kv_refs as R
from tests.test_gpu_kv import ATTENDS, BF16, F16, F32, WRITES, batch_of, rows
from tests.test_gpu_kv_timeout import hooks  # noqa: F401

pytestmark = pytest.mark.gpu


def same(cache, pool):
    got = pool.from_stored(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    return all(np.array_equal(x, y) for x, y in zip(got, (pool.k, pool.ks, pool.v, pool.vs)))


@pytest.mark.parametrize("block,heads,d,dtype,how,seqs", WRITES)
def test_write_and_read(cuda_lib, block, heads, d, dtype, how, seqs):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(11)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, block, rng)
    pool = R4.Pool(n, block, heads, d, rng)
    s = torch.from_numpy(np.exp2(rng.integers(-20, 7, (sum(new), heads, 1)))).cuda()
    k, _ = rows(rng, sum(new), heads, d, dtype, how)
    v, _ = rows(rng, sum(new), heads, d, dtype, how)
    k.copy_(k.double() * s)
    v.copy_(v.double() * s * 0.03)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    status = mp.kv_write(cache, batch, k, v)
    assert np.array_equal(R4.write(pool, table, lens, new, k.double().cpu().numpy(), v.double().cpu().numpy()), status.cpu().numpy())
    assert same(cache, pool)  # what is not written is as it was
    for out_dtype in (F16, BF16, F32):
        ko, _ = rows(rng, sum(new), heads, d, out_dtype, how)
        vo, _ = rows(rng, sum(new), heads, d, out_dtype, how)
        _, _, st = mp.kv_read(cache, batch, out_dtype, k=ko, v=vo)
        assert not st.any()
        want = [np.concatenate(x) for x in zip(*(R4.held(pool, table, b, lens[b] - new[b], lens[b]) for b in range(len(lens))))]
        for x, y in ((ko, want[0]), (vo, want[1])):  # exact in every type
            assert torch.equal(x.double().cpu(), torch.from_numpy(y))
    mp.kv_write(cache, batch, k, v)  # a second call with the same tokens changes nothing
    assert same(cache, pool)


@pytest.mark.parametrize("tokens", [9, 40])
def test_write_beside_borders(cuda_lib, tokens):
    """Largest magnitudes and values a rounding of 32 bits around 7.5 s and (n + 1/2) s, for every scale; zeros; the smallest."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(tokens)
    every = np.concatenate([R4.SCALES[1:], [2.0 ** -30, 1e-40, 240.0]])
    x = np.zeros((tokens * 4 * 4, 32), np.float32)
    for row in range(len(x)):
        s = every[(row * 7 + tokens) % len(every)]
        n = rng.integers(-8, 8, 32) + 0.5
        x[row] = np.clip(n, -7.5, 7.5) * s
        x[row, 0] = 7.5 * s
        off = rng.integers(-1, 2, 32)
        x[row] = np.where(off == 0, x[row], np.nextafter(x[row], np.float32(np.inf) * np.where(off > 0, 1, -1).astype(np.float32)))
        x[row, 0] = min(x[row, 0], np.float32(1800))
    x[5], x[6, 1:] = 0, 0
    k = torch.from_numpy(np.clip(x, -1800, 1800).reshape(tokens, 4, 128)).cuda()
    table, n = R.make_table([tokens + 3], 64, rng)
    pool = R4.Pool(n, 64, 4, 128, rng)
    cache, batch = pool.cache(), batch_of(mp, table, [tokens + 3], [tokens])
    assert not mp.kv_write(cache, batch, k, k.flip(0)).any()
    R4.write(pool, table, [tokens + 3], [tokens], k.double().cpu().numpy(), k.flip(0).double().cpu().numpy())
    assert same(cache, pool)


def test_write_non_finite_and_large_values(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(5)
    lens, new = [40, 40, 3, 40, 35], [8, 40, 3, 40, 20]
    for dtype, few in ((BF16, False), (F32, True), (F16, False)):
        if few:
            new = [8, 5, 3, 4, 16]
        at = np.concatenate([[0], np.cumsum(new)])
        table, n = R.make_table(lens, 32, rng)
        pool = R4.Pool(n, 32, 2, 64, rng)
        k, _ = rows(rng, sum(new), 2, 64, dtype)
        v, _ = rows(rng, sum(new), 2, 64, dtype)
        k[3, 0, 5], k[at[1] + 1, 1, 6] = float("nan"), float("inf")
        v[at[1], 1, 7] = float("-inf")
        v[at[2]:at[3]] = 1800.0
        k[at[3]] = 1808.0  # in every type the next number above
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        status = mp.kv_write(cache, batch, k, v)
        want = R4.write(pool, table, lens, new, k.double().cpu().numpy(), v.double().cpu().numpy())
        assert want.tolist() == [1, 1, 0, 1, 0] and np.array_equal(want, status.cpu().numpy())
        assert same(cache, pool)


def check_attend(mp, pool, table, lens, new, q, qx, scale, causal, window, **kw):
    cache, batch = pool.cache(), batch_of(mp, table, lens, new, **kw)
    out, lse, status = mp.kv_attend(cache, batch, q, scale=scale, causal=causal, window=window, want_lse=True)
    want, want_lse, mag, size = R4.attend(pool, table, lens, new, qx, scale, causal, window)
    bound, lse_bound = R.attend_bounds(q.dtype, want, want_lse, mag, size)
    assert not status.any()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
    assert (out[np.isneginf(want_lse)] == 0).all()
    assert (np.abs(out - want) <= bound).all(), np.max(np.abs(out - want) / bound)
    fine = np.isfinite(want_lse)
    assert (np.abs(lse[fine] - want_lse[fine]) <= lse_bound[fine]).all()


@pytest.mark.parametrize("block,hq,heads,d,dtype,how,causal,window,seqs", ATTENDS)
def test_attend(cuda_lib, block, hq, heads, d, dtype, how, causal, window, seqs):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(7)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, block, rng)
    pool = R4.Pool(n, block, heads, d, rng)
    for b, length in enumerate(lens):  # slots past the end hold bytes that stand for no number
        if length % block:
            for scales in (pool.ks, pool.vs):
                scales[table[b, length // block], :, length % block:] = 0xFF
    q, qx = rows(rng, sum(new), hq, d, dtype, how)
    check_attend(mp, pool, table, lens, new, q, qx, d ** -0.5, causal, window)


@pytest.mark.parametrize("group,d,dtype", [(4, 128, BF16), (4, 64, F16), (3, 128, F16), (1, 64, BF16), (8, 128, BF16)])
@pytest.mark.parametrize("kind", ["prompts", "few", "singles"])
def test_attend_ragged(cuda_lib, group, d, dtype, kind):
    """Batches whose work is cut between CTAs, from scratch memory that holds anything; the definition in 64 bits on the GPU."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(group * d)
    heads, block = 3, 32
    most = {"prompts": 700, "few": 128 // group + 1, "singles": 2}[kind]
    for count in (3, 24):
        new = [int(n) for n in rng.integers(1, most, count)]
        lens = [n + int(x) for n, x in zip(new, rng.integers(0, 900 if kind == "prompts" else 6000, count))]
        lens[0] = new[0]
        table, n = R.make_table(lens, block, rng)
        pool = R4.Pool(n, block, heads, d, rng)
        pool.vs[:] = rng.integers(40, 150, pool.vs.shape)
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        q, qx = rows(rng, sum(new), heads * group, d, dtype)
        k, v, _ = mp.kv_read(cache, batch_of(mp, table, lens, lens), F32)
        want, mag, want_lse, size, row, past = [], [], [], [], 0, 0
        for length, m in zip(lens, new):
            kk, vv = (x[past:past + length].double().repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
            qq = q[row:row + m].double().transpose(0, 1)
            x = qq @ kk.transpose(1, 2) * d ** -0.5
            j = torch.arange(length, device="cuda")
            x = x.masked_fill(j > (length - m + torch.arange(m, device="cuda"))[:, None], -torch.inf)
            w = torch.softmax(x, -1)
            want.append((w @ vv).transpose(0, 1)), mag.append((w @ vv.abs()).transpose(0, 1))
            want_lse.append(torch.logsumexp(x, -1).transpose(0, 1))
            size.append(((qq.abs() @ kk.abs().transpose(1, 2)).amax(-1) * d ** -0.5).transpose(0, 1))
            row, past = row + m, past + length
        want, mag, want_lse, size = (torch.cat(x).cpu().numpy() for x in (want, mag, want_lse, size))
        bound, lse_bound = R.attend_bounds(dtype, want, want_lse, mag, size)
        first = None
        for fill in (0, 255, 0, 255):
            ws = mp.Workspace("cuda")
            ws.get(max(mp.kv_attend_workspace_bytes(cache, batch, heads * group), 1))
            ws.buf.fill_(fill)
            out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True, workspace=ws)
            assert not status.any()
            assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
            assert (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_bound).all()
            first = out if first is None else first
            assert torch.equal(out, first)


def test_attend_sharp_and_flat_rows_and_scales_far_apart(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(9)
    for new in ([1, 90], [2, 3]):
        lens = [3000, 700]
        table, n = R.make_table(lens, 64, rng)
        pool = R4.Pool(n, 64, 2, 128, rng)
        pool.vs[:] = rng.integers(0, 184, pool.vs.shape)  # every scale there is, zeros among them
        pool.ks[table[1, 3]] = 0
        q, _ = rows(rng, sum(new), 4, 128, F16)
        q[0] *= 60
        q[1] = 0
        q[2, 1] *= 1e-6
        q[-1, 2:] *= 100
        check_attend(mp, pool, table, lens, new, q, q.double().cpu().numpy(), 128 ** -0.5, True, 0)


def test_non_finite_queries_stay_in_their_rows(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(19)
    for lens, new in (([100, 50], [1, 2]), ([300, 100], [100, 70]), ([5000, 100], [2, 2])):
        table, n = R.make_table(lens, 64, rng)
        pool = R4.Pool(n, 64, 2, 64, rng)
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        q, _ = rows(rng, sum(new), 4, 64, F16)
        clean, _, _ = mp.kv_attend(cache, batch, q)
        q[1, 2, 3], q[0, 1, 5] = float("nan"), float("inf")
        out, _, status = mp.kv_attend(cache, batch, q)
        assert torch.isnan(out[1, 2]).all() and torch.isnan(out[0, 1]).all() and not status.any()
        clean[1, 2] = clean[0, 1] = out[1, 2] = out[0, 1] = 0
        assert torch.equal(out, clean)


def test_pools_past_32_bit_offsets(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(29)
    block, heads, d = 128, 8, 128
    n = (1 << 32) // (block * heads * d * 17 // 32) + 40
    cache = mp.KvCache4(n, block, heads, d)
    lens = [200, 300]
    ids, local = np.array([[n - 1, n - 3, -1], [n - 2, n - 7, n - 5]], np.int32), np.array([[7, 5, -1], [6, 1, 3]], np.int32)
    small = R4.Pool(8, block, heads, d, rng)
    for x, y in zip((cache.k, cache.v), small.stored()):
        x[n - 8:] = torch.from_numpy(y).cuda()
    for new in ([200, 1], [1, 2]):
        batch = batch_of(mp, ids, lens, new)
        k, kx = rows(rng, sum(new), heads, d, BF16)
        v, vx = rows(rng, sum(new), heads, d, BF16)
        assert not mp.kv_write(cache, batch, k, v).any()
        R4.write(small, local, lens, new, kx, vx)
        got = small.from_stored(cache.k[n - 8:].cpu().numpy(), cache.v[n - 8:].cpu().numpy())
        assert all(np.array_equal(x, y) for x, y in zip(got, (small.k, small.ks, small.v, small.vs)))
        ko, vo, _ = mp.kv_read(cache, batch, F32)
        want = R4.held(small, local, 0, 200 - new[0], 200)
        assert torch.equal(ko[:new[0]].double().cpu(), torch.from_numpy(want[0]))
        q, qx = rows(rng, sum(new), heads, d, BF16)
        out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
        want, want_lse, mag, size = R4.attend(small, local, lens, new, qx, d ** -0.5)
        bound, _ = R.attend_bounds(BF16, want, want_lse, mag, size)
        assert not status.any() and (np.abs(out.double().cpu().numpy() - want) <= bound).all()


def test_bad_sequences_are_reported_and_leave_others_alone(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(31)
    lens = [100, 90, 80, 70, 64, 60]
    table, n = R.make_table(lens, 32, rng)
    for count in (3, 40):
        new = [count] * 6
        pool = R4.Pool(n, 32, 2, 64, rng)
        cache = pool.cache()
        q, _ = rows(rng, sum(new), 4, 64, F16)
        k, kx = rows(rng, sum(new), 2, 64, F16)
        bad_lens, bad_table = list(lens), table.copy()
        bad_lens[1], bad_lens[2] = 101, -1  # past max_len, negative
        bad_table[3, 1:], bad_table[4, 1:] = n, -1  # outside the pool
        bad = batch_of(mp, bad_table, bad_lens, new, max_len=100)
        clean, _, _ = mp.kv_attend(cache, batch_of(mp, table, lens, new, max_len=100), q)
        out, _, status = mp.kv_attend(cache, bad, q)
        assert status.tolist() == [0, 1, 1, 1, 1, 0]
        for s in (slice(0, count), slice(5 * count, 6 * count)):
            assert torch.equal(out[s], clean[s])
        before_k, _, st = mp.kv_read(cache, bad, F32)
        assert st.tolist() == [0, 1, 1, 1, 1, 0]
        assert mp.kv_write(cache, bad, k, k).tolist() == [0, 1, 1, 1, 1, 0]
        for b in (0, 5):
            part = [x[b:b + 1] for x in (table, np.array(lens), np.array(new))]
            R4.write(pool, *part, kx[b * count:(b + 1) * count], kx[b * count:(b + 1) * count])
        got = pool.from_stored(cache.k.cpu().numpy(), cache.v.cpu().numpy())
        for b in (0, 5):
            pages = table[b, :-(-lens[b] // 32)]
            for x, y in zip(got, (pool.k, pool.ks, pool.v, pool.vs)):
                assert np.array_equal(x[pages], y[pages])


def test_empty_pool_and_empty_batch(cuda_lib):
    import paper_2203_00448_gb300 as mp

    none = mp.KvCache4(0, 32, 2, 64)
    q = torch.ones(3, 4, 64, dtype=F16, device="cuda")
    batch = batch_of(mp, np.zeros((2, 2)), [0, 40], [1, 2])
    out, lse, status = mp.kv_attend(none, batch, q, want_lse=True)
    assert status.tolist() == [0, 1] and (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    cache = mp.KvCache4(3, 32, 2, 64)
    empty = batch_of(mp, np.zeros((0, 2)), [], [])
    assert mp.kv_write(cache, empty, q[:0, :2], q[:0, :2]).numel() == 0
    assert mp.kv_attend(cache, empty, q[:0])[0].numel() == 0


def test_captured_calls_and_other_streams(cuda_lib):
    """Graphs replayed after their inputs have changed, two of them at once, beside eager calls on another stream."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(41)
    lens, new = [6000, 333, 64], [1, 2, 1]
    table, n = R.make_table(lens, 64, rng)
    pool = R4.Pool(n, 64, 2, 128, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, 4, 8, 128, BF16)
    k, _ = rows(rng, 4, 2, 128, BF16)
    other, _ = rows(rng, 4, 8, 128, BF16)
    mp.kv_write(cache, batch, k, k)
    mp.kv_attend(cache, batch, q)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in (q, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mp.kv_write(cache, batch, k, k)
            outs.append(mp.kv_attend(cache, batch, x)[0])
        graphs.append(g)
    k.mul_(2)
    q.mul_(0.5)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = mp.kv_read(cache, batch, F32, stream=streams[2])[0]
    torch.cuda.synchronize()
    assert eager.shape == (4, 2, 128)
    for x, y in zip(outs, (q, other)):
        assert torch.equal(x, mp.kv_attend(cache, batch, y)[0])


@pytest.mark.parametrize("d,lens,new", [(128, [6000, 700, 3000], [600, 40, 200]), (64, [60000, 700, 30000], [30, 20, 25])])
def test_attention_wait_runs_out(hooks, d, lens, new):  # noqa: F811
    """A unit held back in the kernel for many rows, as in tests/test_gpu_kv_timeout.py: the call ends, says so, and the next is
    right."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(53)
    table, n = R.make_table(lens, 64, rng)
    pool = R4.Pool(n, 64, 2, d, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, sum(new), 8, d, BF16)
    want, _, status = mp.kv_attend(cache, batch, q)
    assert not status.any()
    for unit in (0, 2):
        hooks(unit)
        _, _, status = mp.kv_attend(cache, batch, q)
        torch.cuda.synchronize()
        hooks(-1)
        assert status.tolist() == [mp.ETIMEOUT] * 3
        out, _, status = mp.kv_attend(cache, batch, q)
        assert not status.any() and torch.equal(out, want)


@pytest.mark.parametrize("group,d", [(4, 128), (1, 64)])
def test_attend_by_both_long_kernels(cuda_lib, group, d):
    """A batch of single tokens over long contexts with pieces of prompts, large enough for both kernels, one joining launch, and one
    that the second takes alone; the definition in 64 bits on the GPU."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(d)
    heads, block = 4, 64
    for lens in ([30000, 17, 40000, 300, 0, 25000, 64, 900], [3000, 17, 4000, 300, 0, 2500, 64, 900]):
        new = [1, 2, 100, 290, 1, 2, 33, 1]
        table, n = R.make_table(lens, block, rng)
        pool = R4.Pool(n, block, heads, d, rng)
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        q, _ = rows(rng, sum(new), heads * group, d, BF16)
        out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
        assert not status.any()
        k, v, _ = mp.kv_read(cache, batch_of(mp, table, lens, lens), F32)
        row = past = 0
        for length, m in zip(lens, new):
            mine, mine_lse = out[row:row + m].double().cpu().numpy(), lse[row:row + m].double().cpu().numpy()
            kk, vv = (x[past:past + length].double().repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
            qq = q[row:row + m].double().transpose(0, 1)
            row, past = row + m, past + length
            if length == 0:
                assert (mine == 0).all() and np.isneginf(mine_lse).all()
                continue
            x = qq @ kk.transpose(1, 2) * d ** -0.5
            x = x.masked_fill(torch.arange(length, device="cuda") > (length - m + torch.arange(m, device="cuda"))[:, None], -torch.inf)
            w = torch.softmax(x, -1)
            want, mag = (w @ vv).transpose(0, 1).cpu().numpy(), (w @ vv.abs()).transpose(0, 1).cpu().numpy()
            want_lse = torch.logsumexp(x, -1).transpose(0, 1).cpu().numpy()
            size = ((qq.abs() @ kk.abs().transpose(1, 2)).amax(-1) * d ** -0.5).transpose(0, 1).cpu().numpy()
            bound, lse_bound = R.attend_bounds(BF16, want, want_lse, mag, size)
            assert (np.abs(mine - want) <= bound).all() and (np.abs(mine_lse - want_lse) <= lse_bound).all()


@pytest.mark.parametrize("new,size", [(1, 1e4), (1, 1e7), (1, 1e12), (40, 1e3), (40, 1e5)])
def test_attend_scores_of_any_size(cuda_lib, new, size):
    """Scores of up to 1e12 and more (2^23 in calls of many rows): one token of each row outweighs all others by far, so the row is
    that token's values, but for rounding to the output's type and for the others, whose weights are e^-40 at most each; in every
    kernel."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(3)
    for lens in ([100, 60], [5000, 60]):
        table, n = R.make_table(lens, 64, rng)
        pool = R4.Pool(n, 64, 2, 64, rng)
        q = torch.from_numpy(rng.standard_normal((2 * new, 4, 64))).to(BF16).cuda()
        assert new == 1 or size * 64 * 8 * float(R4.SCALES[pool.ks.max()]) * 0.2 < 2.0 ** 23  # |q| |k| of 64 values, a fifth of the most
        out, lse, status = mp.kv_attend(pool.cache(), batch_of(mp, table, lens, [new, new]), q, scale=size, want_lse=True)
        assert not status.any() and torch.isfinite(lse).all()
        for b, length in enumerate(lens):
            k, v = R4.held(pool, table, b, 0, length)
            for i in range(new):
                for h in range(4):
                    x = k[:length - new + i + 1, h // 2] @ q[b * new + i, h].double().cpu().numpy()
                    order = np.sort(x)
                    if len(x) > 1 and (order[-1] - order[-2]) * size < 40 + 2.0 ** -16 * order[-1] * size:
                        continue  # two that rounding may bring together
                    want = v[np.argmax(x), h // 2]
                    others = len(x) * np.exp(-40.0) * np.abs(v).max()
                    assert (np.abs(out[b * new + i, h].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + others).all()


@pytest.mark.parametrize("rows_a_head", [4, 12])
@pytest.mark.parametrize("length,later", [(1000, 16), (2560, 1)])
@pytest.mark.parametrize("unit,ahead", [(3.2, 2), (6.5, 1), (9.0, 1)])
def test_attend_large_scores_a_step_apart(cuda_lib, unit, ahead, length, later, rows_a_head):
    """Two tokens whose scores of 13,762,560 and `ahead` more (as the kernels for few rows multiply them, one step of 32 bits is 1
    there) are a few powers of two apart, the larger one in a later granule of the same warp: the larger score may not pass the
    reference by more than weights of 16 bits have room for.  Weights are off by 2^-11, the exponential and its argument by less
    than 2^-18; the log-sum has seven roundings of 2^-24 of itself."""
    import paper_2203_00448_gb300 as mp

    heads, group, d = 2, 4, 64
    new = rows_a_head // group
    table = np.arange(-(-length // 64), dtype=np.int32)[None]
    pool = R4.Pool(table.size, 64, heads, d, np.random.default_rng(61))
    pool.k[:], pool.ks[:] = 8, 120  # zeros under the scale 1
    for granule, more in ((0, 0), (later, ahead)):
        at = (granule * 32 // 64, slice(None), granule * 32 % 64 + 5)
        pool.k[at][:, :8], pool.ks[at][:, 0] = 15, 183  # 8 values of 7 * 240
        pool.k[at][:, 32] = 8 + more
    cache, batch = pool.cache(), batch_of(mp, table, [length], [new])
    for dtype in (BF16, F16):
        q = torch.zeros(new, heads * group, d, dtype=dtype, device="cuda")
        q[..., :8], q[..., 32] = 1.0, 2.0 ** -10  # times 2^14 in the kernels, and keys a sixteenth
        scale = float(np.float32(unit * 2.0 ** 10 / np.log2(np.e)))
        out, lse, status = mp.kv_attend(cache, batch, q, scale=scale, want_lse=True)
        assert not status.any()
        w = np.exp(-scale * ahead * 2.0 ** -10)
        _, v = R4.held(pool, table, 0, 0, length)
        low, high = (v[granule * 32 + 5].repeat(group, 0) for granule in (0, later))
        want, mag = (w * low + high) / (w + 1), (w * np.abs(low) + np.abs(high)) / (w + 1)
        near = mag * (2.0 ** -11 + 2.0 ** -18)
        bound = near + (np.abs(want) + near) * torch.finfo(dtype).eps / 2
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
        want_lse = scale * (13762560 + ahead) * 2.0 ** -10 + np.log1p(w)
        assert (np.abs(lse.double().cpu().numpy() - want_lse) <= want_lse * 2.0 ** -21).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("new,lens", [(1, [100, 90]), (1, [5000, 4000]), (3, [900, 2600]), (40, [900, 5000])])
def test_attend_scores_near_the_limit(cuda_lib, bits, new, lens):
    """Scores of just under 2^23, all of a row's within 4.5 of each other: 32 bits leave them off by less than 1 each (1.45 as powers of
    two), so weights are off by e at most and outputs are means of the values all the same, whichever value of a row is the
    reference: between the least and the largest, but for the weights' 2^-11 and the output's rounding."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(67)
    heads, group, d, block = 2, 4, 64, 64
    table, n = R.make_table(lens, block, rng)
    kind = R4 if bits == 4 else R
    pool = kind.Pool(n, block, heads, d, rng)
    code = rng.integers(0, 8, pool.k.shape[:3])
    if bits == 4:
        pool.k[:], pool.ks[:] = 8, 120  # zeros under the scale 1
        pool.k[..., :8], pool.ks[..., 0] = 15, 183  # 8 values of 7 * 240
        pool.k[..., 32] = 8 + code
        most, step = 8 * 1680.0, 2.0 ** -10
    else:
        pool.k[:], pool.ks[:] = 0, 4.0
        pool.k[..., :8] = 0x7e  # 448
        pool.k[..., 32] = R.to_byte(code.astype(float))
        most, step = 8 * 1792.0, 2.0 ** -12
    scale = (2.0 ** 23 - 8) / most
    assert 7 * step * float(pool.ks.flat[0] if bits == 8 else 1) * scale < 4.5
    q = torch.zeros(2 * new, heads * group, d, dtype=BF16, device="cuda")
    q[..., :8], q[..., 32] = 1.0, step
    out, lse, status = mp.kv_attend(pool.cache(), batch_of(mp, table, lens, [new, new]), q, scale=scale, want_lse=True)
    assert not status.any() and (torch.abs(lse / 2.0 ** 23 - 1) < 2.0 ** -18).all()
    out = out.double().cpu().numpy()
    for b, length in enumerate(lens):
        _, v = kind.held(pool, table, b, 0, length)
        low, high, size = (x.repeat(group, 0) for x in (v.min(0), v.max(0), np.abs(v).max(0)))
        for i in range(new):
            mine = out[b * new + i]
            assert (mine >= low - size * 2.0 ** -7).all() and (mine <= high + size * 2.0 ** -7).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("new,lens", [(1, [100, 90]), (1, [5000, 4000]), (3, [900, 2600]), (40, [900, 5000])])
def test_attend_zero_queries_under_any_scale(cuda_lib, bits, new, lens):
    """Scores of 0 are 0 under the largest scale too: every value that a row sees weighs the same.  Sums of 5,000 values under
    equal weights in 32 bits, 16 at a time, each off by 2^-22 of the sum of magnitudes: 2^-13."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(71)
    heads, group, d = 2, 4, 64
    table, n = R.make_table(lens, 64, rng)
    kind = R4 if bits == 4 else R
    pool = kind.Pool(n, 64, heads, d, rng)
    q = torch.zeros(2 * new, heads * group, d, dtype=BF16, device="cuda")
    for scale in (1e36, 1e38, 3.4e38):
        out, lse, status = mp.kv_attend(pool.cache(), batch_of(mp, table, lens, [new, new]), q, scale=scale, want_lse=True)
        assert not status.any()
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for b, length in enumerate(lens):
            _, v = kind.held(pool, table, b, 0, length)
            for i in range(new):
                seen = v[:length - new + i + 1].repeat(group, 1)
                want, size = seen.mean(0), np.abs(seen).mean(0)
                assert (np.abs(out[b * new + i] - want) <= size * (2.0 ** -13 + 2.0 ** -20) + np.abs(want) * 2.0 ** -8).all()
                assert (np.abs(lse[b * new + i] - np.log(len(seen))) <= 2.0 ** -18).all()
