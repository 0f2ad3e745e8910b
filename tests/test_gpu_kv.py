"""The key/value cache operators against plain 64-bit implementations, at the sizes, masks and layouts where they can go
wrong: lengths of 0 and 1, blocks that end inside a granule or tile, queries that see nothing, unused slots full of bytes
that stand for no number, groups that are no power of two, strided and unaligned rows, scales far apart."""
import numpy as np
import pytest
import torch

from tests import kv_refs as R

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def batch_of(mp, table, lens, new, **kw):
    ptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    dev = [torch.from_numpy(np.asarray(x, t)).cuda() for x, t in ((table, np.int32), (lens, np.int32), (ptr, np.int64))]
    kw.setdefault("max_tokens", max([0] + list(new)))
    return mp.KvBatch(*dev, n_tokens=int(ptr[-1]), **kw)


def rows(rng, tokens, heads, d, dtype, how="plain", scale=1.0):
    """A tensor [tokens, heads, d] of `dtype`, laid out as asked, and its values in float64."""
    x = torch.from_numpy(rng.standard_normal((tokens, heads, d)) * scale).to(dtype).cuda()
    if how == "packed":  # columns of a wider projection
        wide = torch.zeros(tokens, (heads + 3) * d, dtype=dtype, device="cuda")
        view = wide[:, 2 * d:(heads + 2) * d].view(tokens, heads, d)
    elif how == "odd":  # rows that start off any 16-byte boundary
        wide = torch.zeros(tokens * (heads * d + 3) + 5, dtype=dtype, device="cuda")
        view = wide[1:1 + tokens * (heads * d + 3)].view(tokens, -1)[:, :heads * d].view(tokens, heads, d)
    elif how == "heads":  # heads before tokens
        view = torch.zeros(heads, tokens, d, dtype=dtype, device="cuda").transpose(0, 1)
    else:
        return x, x.double().cpu().numpy()
    view.copy_(x)
    return view, x.double().cpu().numpy()


WRITES = [
    # block, heads, d, dtype, rows' layout, (held, new) of each sequence
    (32, 8, 128, BF16, "plain", [(1, 1), (33, 1), (64, 1), (500, 1)]),
    (64, 2, 64, F16, "packed", [(1, 1), (65, 2), (70, 7), (0, 0), (128, 16)]),
    (96, 3, 128, F32, "odd", [(5, 5), (97, 3), (96, 1)]),
    (256, 1, 64, BF16, "heads", [(300, 10)]),
    (32, 2, 128, F16, "plain", [(17, 17), (500, 100), (333, 333), (40, 0), (33, 32)]),
    (64, 5, 64, BF16, "odd", [(129, 129), (64, 64), (63, 62)]),
    (128, 1, 128, F32, "heads", [(1000, 999), (20, 18)]),
    (256, 2, 64, F32, "packed", [(511, 300)]),
]


@pytest.mark.parametrize("block,heads,d,dtype,how,seqs", WRITES)
def test_write_and_read(cuda_lib, block, heads, d, dtype, how, seqs):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(11)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, block, rng)
    pool = R.Pool(n, block, heads, d, rng)
    # sizes a thousandfold apart, so that some blocks' scales grow and some do not
    size = np.exp2(rng.integers(-8, 4, (sum(new), heads, 1)))
    k, kx = rows(rng, sum(new), heads, d, dtype, how)
    v, vx = rows(rng, sum(new), heads, d, dtype, how)
    s = torch.from_numpy(size).cuda()
    k.copy_(k.double() * s)
    v.copy_(v.double() * s * 0.03)
    kx, vx = k.double().cpu().numpy(), v.double().cpu().numpy()
    cache = pool.cache()
    batch = batch_of(mp, table, lens, new)
    status = mp.kv_write(cache, batch, k, v)
    assert np.array_equal(R.write(pool, table, lens, new, kx, vx), status.cpu().numpy())
    got = pool.from_stored(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    assert np.array_equal(cache.k_scale.cpu().numpy(), pool.ks) and np.array_equal(cache.v_scale.cpu().numpy(), pool.vs)
    # the sign of a zero is kept, so bytes are equal, not only values
    assert np.array_equal(got[0], pool.k) and np.array_equal(got[1], pool.v)
    # a second call with the same tokens changes nothing
    mp.kv_write(cache, batch, k, v)
    again = pool.from_stored(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    assert np.array_equal(again[0], pool.k) and np.array_equal(again[1], pool.v)

    for out_dtype in (F16, BF16, F32):
        ko, _ = rows(rng, sum(new), heads, d, out_dtype, how)
        vo, _ = rows(rng, sum(new), heads, d, out_dtype, how)
        _, _, st = mp.kv_read(cache, batch, out_dtype, k=ko, v=vo)
        assert not st.any()
        want = [np.concatenate(x) for x in zip(*(R.held(pool, table, b, lens[b] - new[b], lens[b]) for b in range(len(lens))))]
        for x, y in ((ko, want[0]), (vo, want[1])):
            assert torch.equal(x.cpu(), torch.from_numpy(y).to(out_dtype))


def test_read_everything_and_random_bytes(cuda_lib):
    """All finite bytes under scales that are no power of two, read whole and from the middle of a block."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(3)
    lens = [700, 1, 0, 63]
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 3, 64, rng)
    for x in (pool.k, pool.v):
        x[:] = rng.integers(0, 256, x.shape)
        x[x & 127 == 127] = 0x7E
    pool.ks[:], pool.vs[:] = (rng.uniform(1e-3, 10, pool.ks.shape) for _ in range(2))
    cache = pool.cache()
    for new in ([700, 1, 0, 63], [13, 0, 0, 31]):
        k, v, st = mp.kv_read(cache, batch_of(mp, table, lens, new), F32)
        want = [np.concatenate(x) for x in zip(*(R.held(pool, table, b, lens[b] - new[b], lens[b]) for b in range(4)))]
        assert torch.equal(k.cpu(), torch.from_numpy(want[0]).float()) and not st.any()
        assert torch.equal(v.cpu(), torch.from_numpy(want[1]).float())


def test_write_non_finite_and_extreme_values(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(5)
    lens, new = [40, 40, 3, 40, 35], [8, 40, 3, 40, 20]
    for dtype in (BF16, F32):
        table, n = R.make_table(lens, 32, rng)
        pool = R.Pool(n, 32, 2, 64, rng)
        k, _ = rows(rng, sum(new), 2, 64, dtype)
        v, _ = rows(rng, sum(new), 2, 64, dtype)
        k[3, 0, 5], k[4, 1, 6] = float("nan"), float("inf")
        v[9, 1, 7] = float("-inf")
        k[48:51] = 0  # nothing but zeros
        v[51:91] *= 3e38 if dtype == F32 else 1e38  # the largest values there are
        v[60, 0, 0] = torch.finfo(dtype).max
        k[91:] *= 1e-30  # below the least scale
        kx, vx = k.double().cpu().numpy(), v.double().cpu().numpy()
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        status = mp.kv_write(cache, batch, k, v)
        want = R.write(pool, table, lens, new, kx, vx)
        assert want[0] == 1 and want[1] == 1
        assert np.array_equal(want, status.cpu().numpy())
        got = pool.from_stored(cache.k.cpu().numpy(), cache.v.cpu().numpy())
        assert np.array_equal(cache.k_scale.cpu().numpy(), pool.ks) and np.array_equal(cache.v_scale.cpu().numpy(), pool.vs)
        assert np.array_equal(got[0], pool.k) and np.array_equal(got[1], pool.v)


def check_attend(mp, pool, table, lens, new, q, qx, scale, causal, window, **kw):
    cache, batch = pool.cache(), batch_of(mp, table, lens, new, **kw)
    out, lse, status = mp.kv_attend(cache, batch, q, scale=scale, causal=causal, window=window, want_lse=True)
    want, want_lse, mag, size = R.attend(pool, table, lens, new, qx, scale, causal, window)
    bound, lse_bound = R.attend_bounds(q.dtype, want, want_lse, mag, size)
    assert not status.any()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
    assert (out[np.isneginf(want_lse)] == 0).all()
    assert (np.abs(out - want) <= bound).all(), np.max(np.abs(out - want) / bound)
    fine = np.isfinite(want_lse)
    assert (np.abs(lse[fine] - want_lse[fine]) <= lse_bound[fine]).all()
    return out


ATTENDS = [
    # block, query heads, heads, d, dtype, layout, causal, window, (held, new) of each sequence
    (32, 8, 8, 128, BF16, "plain", True, 0, [(1, 1)]),
    (32, 8, 8, 128, BF16, "packed", True, 0, [(512, 1)]),
    (64, 32, 8, 128, BF16, "plain", True, 0, [(0, 1), (1, 1), (31, 1), (32, 1), (33, 1), (700, 1), (5, 0)]),
    (96, 6, 2, 64, F16, "odd", True, 0, [(97, 2), (5, 2), (1, 2), (64, 1), (300, 2)]),  # one query before the start
    (32, 20, 4, 64, F16, "heads", True, 40, [(100, 3), (45, 3), (41, 3), (40, 1), (2, 2)]),
    (128, 5, 1, 128, F16, "plain", True, 1, [(200, 3), (1, 1)]),
    (64, 16, 2, 64, BF16, "plain", True, 0, [(50, 2), (1000, 1), (64, 2)]),  # groups of 8: two tiles of rows
    (256, 12, 4, 64, BF16, "packed", True, 100, [(513, 5), (99, 4)]),
    (64, 8, 2, 128, F16, "plain", False, 0, [(130, 4), (1, 3), (0, 2), (64, 4)]),
    # many rows: prompts, pieces of them, pieces before the start, no causal order
    (64, 8, 2, 128, BF16, "packed", True, 0, [(200, 200)]),
    (32, 4, 4, 64, F16, "plain", True, 0, [(127, 127), (129, 129), (128, 128), (1, 1), (0, 0)]),
    (96, 6, 2, 128, F16, "odd", True, 0, [(400, 70), (60, 64), (300, 1)]),
    (64, 3, 1, 128, BF16, "heads", True, 0, [(385, 100), (500, 33)]),
    (32, 10, 2, 64, BF16, "plain", True, 50, [(300, 120), (49, 40), (400, 2)]),
    (64, 4, 2, 128, F16, "plain", True, 130, [(600, 260)]),
    (64, 8, 8, 64, F16, "packed", False, 0, [(37, 100), (300, 129), (1, 64), (0, 20)]),
    (128, 7, 1, 128, BF16, "plain", False, 0, [(257, 61)]),
]


@pytest.mark.parametrize("block,hq,heads,d,dtype,how,causal,window,seqs", ATTENDS)
def test_attend(cuda_lib, block, hq, heads, d, dtype, how, causal, window, seqs):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(7)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, block, rng)
    pool = R.Pool(n, block, heads, d, rng)
    for b, length in enumerate(lens):  # slots past the end hold bytes that stand for no number
        if length % block:
            page = table[b, length // block]
            pool.k[page, :, length % block:] = 0x7F
            pool.v[page, :, length % block:] = 0xFF
    q, qx = rows(rng, sum(new), hq, d, dtype, how)
    check_attend(mp, pool, table, lens, new, q, qx, d ** -0.5, causal, window)


@pytest.mark.parametrize("group,d,dtype", [(4, 128, BF16), (4, 64, F16), (3, 128, F16), (1, 64, BF16)])
def test_attend_many_ragged_prompts(cuda_lib, group, d, dtype):
    """Pairs of row tiles with one tile in use follow and precede pairs with both, in batches whose work is cut between
    CTAs, from scratch memory that holds anything; the definition in 64 bits on the GPU."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(group * d)
    heads, block = 3, 32
    for seqs in ([(500, 460), (1300, 408), (700, 300)], [(int(n) + int(x), int(n)) for n, x in
                                                      zip(rng.integers(30, 700, 24), rng.integers(0, 900, 24))]):
        lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
        table, n = R.make_table(lens, block, rng)
        pool = R.Pool(n, block, heads, d, rng)
        pool.vs[:] = np.exp2(rng.integers(-12, 3, pool.vs.shape))  # scales that are not the next unit's
        pool.ks[:] = np.exp2(rng.integers(-9, -5, pool.ks.shape))
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        q, qx = rows(rng, sum(new), heads * group, d, dtype)
        k, v, _ = mp.kv_read(cache, batch_of(mp, table, lens, lens), F32)
        want, mag, row, past = [], [], 0, 0
        want_lse, size = [], []
        for length, m in seqs:
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
        for fill in (0, 255, 0, 255):
            ws = mp.Workspace("cuda")
            need = mp.kv_attend_workspace_bytes(cache, batch, heads * group)
            ws.get(need)
            ws.buf.fill_(fill)
            out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True, workspace=ws)
            assert not status.any()
            assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
            assert (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_bound).all()


@pytest.mark.parametrize("group,d,dtype,causal,window", [
    (4, 128, BF16, True, 0), (4, 64, F16, True, 0), (3, 128, F16, False, 0), (8, 64, BF16, True, 700),
    (1, 128, BF16, True, 130)])
def test_attend_one_row_tile(cuda_lib, group, d, dtype, causal, window):
    """17 to 128 rows a sequence and head, which two halves of a CTA share by the granules: contexts that give one half
    nothing, that end in either half's turn, that are cut between CTAs, next to prompts of both row tiles."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(1000 * group + d + window)
    heads, block = 3, 64
    news = [17 // group + 1, 128 // group, 40 // group + 1]
    seqs = [(max(n, length), n) for length in (1, 40, 128, 129, 256, 257, 384, 400, 640) for n in news]
    seqs += [(int(n), news[i % 3]) for i, n in enumerate(rng.integers(1500, 6000, 12))]
    seqs += [(900, 300), (1400, 130 // group + 1), (4000, 20)]
    order = rng.permutation(len(seqs))
    lens, new = [seqs[i][0] for i in order], [seqs[i][1] for i in order]
    table, n = R.make_table(lens, block, rng)
    pool = R.Pool(n, block, heads, d, rng)
    pool.vs[:] = np.exp2(rng.integers(-12, 3, pool.vs.shape))
    pool.ks[:] = np.exp2(rng.integers(-9, -5, pool.ks.shape))
    q, qx = rows(rng, sum(new), heads * group, d, dtype)
    check_attend(mp, pool, table, lens, new, q, qx, d ** -0.5, causal, window)


def test_attend_contexts_of_millions(cuda_lib):
    """A piece of a prompt over ten million positions that share four blocks: a CTA spends a tenth of a second and more on
    each of several heads, and no wait may take that for a fault.  As the last block is whole and every row sees each of the
    four nearly equally often, the result is attention over the four."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(5)
    block, heads, group, d, n = 256, 5, 8, 64, 4864
    columns = 40000
    pool = R.Pool(4, block, heads, d, rng)
    q, _ = rows(rng, n, heads * group, d, BF16)
    table = np.tile(np.arange(4, dtype=np.int32), columns // 4)[None]
    out, _, status = mp.kv_attend(pool.cache(), batch_of(mp, table, [columns * block], [n]), q)
    assert not status.any()
    small = np.arange(4, dtype=np.int32)[None].repeat(n, 0)  # each row on its own over the four blocks
    want, _, status = mp.kv_attend(pool.cache(), batch_of(mp, small, [4 * block] * n, [1] * n), q)
    assert not status.any()
    v = mp.kv_read(pool.cache(), batch_of(mp, small[:1], [4 * block], [4 * block]), F32)[1].double().abs().amax((0, 2))
    # f32 sums of as many steps of 16 tokens, each cut off at 24 bits; weights as f16 and the last rows' uneven share of the
    # four below 2^-8 together; both results rounded to bf16
    steps = columns * block / 16
    bound = (steps * 2.0 ** -24 + 2.0 ** -8) * v.repeat_interleave(group)[None, :, None] + 2.0 ** -7 * want.abs().double()
    assert ((out.double() - want.double()).abs() <= bound).all()


def test_attend_sharp_and_flat_rows(cuda_lib):
    """Scores hundreds apart, one token that outweighs thousands, and queries of zeros (all weights equal)."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(9)
    lens, new = [3000, 700], [1, 90]
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 2, 128, rng)
    q, _ = rows(rng, sum(new), 4, 128, F16)
    q[0] *= 60
    q[1:30] = 0
    q[30:60, 1] *= 1e-6
    q[60:, 2:] *= 100
    pool.v[:, 1] = R.to_byte(np.abs(R.VALUES[pool.v[:, 1]]))  # values of one sign: lost weights would show
    check_attend(mp, pool, table, lens, new, q, q.double().cpu().numpy(), 128 ** -0.5, True, 0)


def test_attend_scales_far_apart(cuda_lib):
    """Blocks whose scales differ by 2^40, scales that are no power of two, and scales of zero."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(13)
    for seqs in ([(300, 1), (33, 2)], [(300, 80), (65, 64)]):
        lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
        table, n = R.make_table(lens, 32, rng)
        pool = R.Pool(n, 32, 2, 64, rng)
        pool.vs[:] = rng.uniform(0.5, 1, pool.vs.shape) * np.exp2(rng.integers(-20, 21, pool.vs.shape))
        pool.ks[:] = rng.uniform(0.2, 1, pool.ks.shape) * 2.0 ** -5
        pool.vs[table[0, 1]] = 0
        pool.ks[table[0, 2]] = 0
        q, qx = rows(rng, sum(new), 4, 64, BF16)
        check_attend(mp, pool, table, lens, new, q, qx, 0.2, True, 0)


def test_attend_many_short_sequences(cuda_lib):
    """More sequences than threads of a CTA, some empty: each warp's stretch covers several."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(17)
    lens = [int(x) for x in rng.integers(0, 70, 700)]
    new = [int(x) for x in rng.integers(0, 3, 700)]
    table, n = R.make_table(lens, 32, rng)
    pool = R.Pool(n, 32, 1, 64, rng)
    q, qx = rows(rng, sum(new), 2, 64, BF16)
    check_attend(mp, pool, table, lens, new, q, qx, 0.125, True, 0)


def test_non_finite_queries_stay_in_their_rows(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(19)
    for lens, new in (([100, 50], [1, 2]), ([300, 100], [100, 70])):
        table, n = R.make_table(lens, 64, rng)
        pool = R.Pool(n, 64, 2, 64, rng)
        cache, batch = pool.cache(), batch_of(mp, table, lens, new)
        q, _ = rows(rng, sum(new), 4, 64, F16)
        clean, _, _ = mp.kv_attend(cache, batch, q)
        q[1, 2, 3] = float("nan")
        q[0, 1, 5] = float("inf")
        out, _, status = mp.kv_attend(cache, batch, q)
        assert torch.isnan(out[1, 2]).all() and torch.isnan(out[0, 1]).all() and not status.any()
        clean[1, 2] = clean[0, 1] = out[1, 2] = out[0, 1] = 0
        assert torch.equal(out, clean)


def test_attend_same_result_every_time(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(23)
    lens, new = [5000, 333, 64], [1, 40, 1]
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 2, 128, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, sum(new), 8, 128, BF16)
    first, first_lse, _ = mp.kv_attend(cache, batch, q, want_lse=True)
    for _ in range(20):
        out, lse, _ = mp.kv_attend(cache, batch, q, want_lse=True)
        assert torch.equal(out, first) and torch.equal(lse, first_lse)


def test_pools_past_32_bit_offsets(cuda_lib):
    """Blocks whose bytes lie past 2^32 in the pool."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(29)
    block, heads, d = 128, 8, 128
    n = (1 << 32) // (block * heads * d) + 40
    cache = mp.KvCache(n, block, heads, d)
    lens, new = [200, 300], [200, 1]
    ids = np.array([[n - 1, n - 3, -1], [n - 2, n - 7, n - 5]], np.int32)
    small = R.Pool(8, block, heads, d, rng)
    local = np.array([[7, 5, -1], [6, 1, 3]], np.int32)
    for x, y in zip((cache.k, cache.v), small.stored()):
        x[n - 8:] = torch.from_numpy(y).cuda()
    cache.k_scale[n - 8:] = torch.from_numpy(small.ks).cuda()
    cache.v_scale[n - 8:] = torch.from_numpy(small.vs).cuda()
    batch = batch_of(mp, ids, lens, new)
    k, kx = rows(rng, 201, heads, d, BF16)
    v, vx = rows(rng, 201, heads, d, BF16)
    assert not mp.kv_write(cache, batch, k, v).any()
    R.write(small, local, lens, new, kx, vx)
    got = small.from_stored(cache.k[n - 8:].cpu().numpy(), cache.v[n - 8:].cpu().numpy())
    assert np.array_equal(got[0], small.k) and np.array_equal(got[1], small.v)
    ko, vo, _ = mp.kv_read(cache, batch, F32)
    want = R.held(small, local, 0, 0, 200)
    assert torch.equal(ko[:200].cpu(), torch.from_numpy(want[0]).float())
    assert torch.equal(vo[:200].cpu(), torch.from_numpy(want[1]).float())
    q, qx = rows(rng, 201, heads, d, BF16)
    out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
    want, want_lse, mag, size = R.attend(small, local, lens, new, qx, d ** -0.5)
    bound, _ = R.attend_bounds(BF16, want, want_lse, mag, size)
    assert not status.any() and (np.abs(out.double().cpu().numpy() - want) <= bound).all()


def test_bad_sequences_are_reported_and_leave_others_alone(cuda_lib):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(31)
    lens, new = [100, 90, 80, 70, 64, 60], [3, 3, 3, 3, 3, 3]
    table, n = R.make_table(lens, 32, rng)
    pool = R.Pool(n, 32, 2, 64, rng)
    for many in (False, True):
        if many:
            new = [40, 40, 40, 40, 40, 40]
        cache = pool.cache()
        good = batch_of(mp, table, lens, new, max_len=100)
        q, _ = rows(rng, sum(new), 4, 64, F16)
        k, _ = rows(rng, sum(new), 2, 64, F16)
        clean, _, _ = mp.kv_attend(cache, good, q)
        bad_lens, bad_table = list(lens), table.copy()
        bad_lens[1] = 101  # past max_len
        bad_lens[2] = -1
        bad_table[3, 1] = n  # outside the pool
        bad_table[4, 1] = -1
        ptr = np.concatenate([[0], np.cumsum(new)])
        bad = batch_of(mp, bad_table, bad_lens, new, max_len=100)
        out, _, status = mp.kv_attend(cache, bad, q)
        assert status.tolist() == [0, 1, 1, 1, 1, 0]
        for b in (0, 5):
            assert torch.equal(out[ptr[b]:ptr[b + 1]], clean[ptr[b]:ptr[b + 1]])
        # 3 tokens of sequence 3 lie past the block that is outside the pool: nothing is read or written there
        _, _, status = mp.kv_read(cache, bad, F16)
        assert status.tolist() == [0, 1, 1, int(many), 1, 0]
        other = pool.cache()
        assert mp.kv_write(cache, bad, k, k).tolist() == [0, 1, 1, int(many), 1, 0]
        assert not mp.kv_write(other, good, k, k).any()
        for b in (0, 5):
            for page in table[b][table[b] >= 0]:
                assert torch.equal(cache.k[page], other.k[page]) and torch.equal(cache.v[page], other.v[page])
        # token ranges that go back or past the end, and more tokens than the declared bound or than are held
        twisted = batch_of(mp, table, lens, new, max_len=100)
        twisted.token_ptr[2] = ptr[1] - 1
        status = mp.kv_attend(cache, twisted, q)[2]
        assert status[1] == 1 and status[0] == 0
        twisted.token_ptr.copy_(torch.from_numpy(ptr))
        twisted.token_ptr[6] = int(ptr[-1]) + 1
        assert mp.kv_attend(cache, twisted, q)[2].tolist() == [0, 0, 0, 0, 0, 1]
        assert mp.kv_write(cache, twisted, k, k).tolist() == [0, 0, 0, 0, 0, 1]
        held = torch.tensor([2, 100, 100, 100, 100, 100], dtype=torch.int32)
        short = batch_of(mp, table, held.numpy(), new, max_len=100)
        assert mp.kv_read(cache, short, F16)[2][0] == 1
        assert mp.kv_write(cache, short, k, k)[0] == 1


def test_empty_calls(cuda_lib):
    import paper_2203_00448_gb300 as mp

    cache = mp.KvCache(0, 32, 2, 64)
    none = batch_of(mp, np.zeros((0, 1)), [], [])
    q = torch.zeros(0, 4, 64, dtype=F16, device="cuda")
    assert mp.kv_attend(cache, none, q)[0].shape == (0, 4, 64)
    assert mp.kv_write(cache, none, q[:, :2], q[:, :2]).shape == (0,)
    assert mp.kv_read(cache, none)[0].shape == (0, 2, 64)
    idle = batch_of(mp, np.full((2, 1), -1), [0, 0], [0, 0])  # sequences, but no tokens
    assert mp.kv_attend(cache, idle, q)[2].tolist() == [0, 0]
    assert mp.kv_write(cache, idle, q[:, :2], q[:, :2]).tolist() == [0, 0]
    assert mp.kv_read(cache, idle)[2].tolist() == [0, 0]
    first = batch_of(mp, np.full((1, 1), -1), [0], [3], max_tokens=3)  # queries over nothing, no block at all
    out, lse, st = mp.kv_attend(cache, first, torch.ones(3, 4, 64, dtype=F16, device="cuda"), causal=False, want_lse=True)
    assert not out.any() and torch.isneginf(lse).all() and st.tolist() == [0]


def test_streams_and_graphs(cuda_lib):
    """Calls on two streams at once, each with its own scratch, and a captured step that follows lens on the device."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(37)
    lens, new = [2000, 900], [1, 1]
    table, n = R.make_table([2100, 1000], 64, rng)
    pool = R.Pool(n, 64, 2, 128, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, 2, 8, 128, BF16)
    r, _ = rows(rng, 2, 8, 128, BF16)
    want, want_r = mp.kv_attend(cache, batch, q)[0], mp.kv_attend(cache, batch, r)[0]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [(mp.kv_attend(cache, batch, q, stream=s1)[0], mp.kv_attend(cache, batch, r, stream=s2)[0]) for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) and torch.equal(b, want_r) for a, b in got)

    k, _ = rows(rng, 2, 2, 128, BF16)
    out, status = torch.empty_like(q), torch.empty(2, dtype=torch.int32, device="cuda")
    ws = mp.Workspace("cuda")
    mp.kv_attend(cache, batch, q, out=out, status=status, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        batch.lens += 1
        mp.kv_write(cache, batch, k, k, status=status)
        mp.kv_attend(cache, batch, q, out=out, status=status, workspace=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert batch.lens.tolist() == [2003, 903]
    twin = pool.cache()
    for step in range(1, 4):
        at = batch_of(mp, table, [2000 + step, 900 + step], new)
        mp.kv_write(twin, at, k, k)
    assert torch.equal(twin.k, cache.k) and torch.equal(twin.v_scale, cache.v_scale)
    assert torch.equal(mp.kv_attend(twin, at, q)[0], out)


def test_example_serves_planned_requests(cuda_lib):
    """The example's loop: requests' blocks from one plan, prompts and single tokens mixed in a call.  An output may be off
    by bf16's last rounding, 2^-9 of it, and by the weights' 2^-11 (both at most, in the 2-norm)."""
    from examples.serve_requests import serve

    for kw in (dict(n=12, prompt=150, generate=8, spread=15, heads=2, group=4, dim=64, block_tokens=32),
               dict(n=6, prompt=400, generate=5, spread=4, heads=1, group=3, dim=128, block_tokens=96, dtype=F16)):
        done = serve(check=True, **kw)
        assert done["pool_blocks"] < done["blocks"] or kw["spread"] < 10
        assert 0 < done["worst"] <= 2.0 ** -9 + 2.0 ** -11


@pytest.mark.parametrize("lens,new", [([40, 0, 33], [1, 1, 0]), ([9000, 0, 1], [1, 2, 2]), ([300, 0, 5], [100, 40, 3]),
                                      ([120000, 0, 70000, 1], [40, 40, 1, 0])])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_empty_pool(cuda_lib, lens, new, causal):
    """A pool without blocks: sequences that see a position are refused by every route, the others get their zeros."""
    import paper_2203_00448_gb300 as mp

    for heads, dtype in ((1, F16), (8, BF16)):
        cache = mp.KvCache(0, 32, heads, 128)
        for entry in (0, -1, 7):
            table = np.full((len(lens), -(-max(lens) // 32)), entry)
            q = torch.ones(sum(new), 4 * heads, 128, dtype=dtype, device="cuda")
            out = torch.full_like(q, 5)
            _, lse, status = mp.kv_attend(cache, batch_of(mp, table, lens, new), q, causal=causal, out=out, want_lse=True)
            assert status.tolist() == [int(n > 0 and length > 0) for length, n in zip(lens, new)]
            at = new[0]
            assert not out[at:at + new[1]].any() and torch.isneginf(lse[at:at + new[1]]).all()


def equal_weights(mp, rng, lens, new, vs, heads=2, group=4, d=64, dtype=BF16, blocks=4):
    """Attention of queries of zeros over sequences that share a few blocks under value scales vs: out and lse."""
    block = 256
    pool = R.Pool(blocks, block, heads, d, rng)
    pool.vs[:] = vs
    columns = -(-max(lens) // block)
    table = np.tile(np.arange(columns, dtype=np.int32) % blocks, (len(lens), 1))
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q = torch.zeros(sum(new), heads * group, d, dtype=dtype, device="cuda")
    out, lse, status = mp.kv_attend(cache, batch, q, causal=False, want_lse=True)
    assert not status.any()
    return out, lse.double().cpu().numpy()


@pytest.mark.parametrize("lens,new", [([1500], [1]), ([16384, 40000], [1, 2]), ([3_000_000], [1]),
                                      ([2_500_000, 2_100_000], [40, 20])])
@pytest.mark.parametrize("d,dtype", [(64, F16), (128, BF16)])
def test_attend_values_all_of_scale_zero(cuda_lib, lens, new, d, dtype):
    """Scales of 0, and below 2^-84, where they count as 0: outputs are 0 and the log-sums are those of the scores, however
    many tokens share the weight.  A log-sum's terms are below 128 in units of log 2, where 32 bits keep 2^-18; four of them."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(41)
    for vs in (0.0, 2.0 ** -85, 2.0 ** -149):
        out, lse = equal_weights(mp, rng, lens, new, vs, d=d, dtype=dtype)
        want = np.repeat(np.log(lens), new)[:, None]
        assert not out.any()
        assert (np.abs(lse - want) <= 2.0 ** -16 + 2.0 ** -20 * (1 + want)).all()


@pytest.mark.parametrize("seqs", [[(300, 1), (33, 2)], [(5000, 2), (4000, 1)], [(300, 80), (65, 64)], [(4500, 300), (129, 20)]])
def test_attend_scales_of_zero_among_others(cuda_lib, seqs):
    """Blocks of scale 0, whose bytes are no small numbers, take part in the softmax and add nothing to the outputs."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(43)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, 32, rng)
    pool = R.Pool(n, 32, 2, 128, rng)
    pool.vs[:] = np.exp2(rng.integers(-60, -55, pool.vs.shape))
    for b in range(2):
        pool.vs[table[b, ::3]] = 0
        pool.vs[table[b, 1::6]] = 2.0 ** -84 * 0.999  # counts as 0
    q, qx = rows(rng, sum(new), 4, 128, BF16)
    small, pool.vs = pool.vs, np.where(pool.vs < 2.0 ** -84, np.float32(0), pool.vs)
    want = R.attend(pool, table, lens, new, qx, 0.09)
    pool.vs = small
    out, lse, status = mp.kv_attend(pool.cache(), batch_of(mp, table, lens, new), q, scale=0.09, want_lse=True)
    bound, lse_bound = R.attend_bounds(BF16, *want)
    assert not status.any()
    assert (np.abs(out.double().cpu().numpy() - want[0]) <= bound).all()
    assert (np.abs(lse.double().cpu().numpy() - want[1]) <= lse_bound + 2.0 ** -16).all()


@pytest.mark.parametrize("lens,new", [([100, 50], [1, 2]), ([6000, 2500], [3, 1]), ([300, 100], [100, 70]), ([30000, 700], [90, 20])])
@pytest.mark.parametrize("d", [64, 128])
def test_log_sums_of_non_finite_queries(cuda_lib, lens, new, d):
    """A query row of which no score is a number has no log-sum either: NaN, not that of a row that sees nothing, by which
    whoever merges parts of an attention would leave it out.  All other rows keep theirs."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(19)
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 2, d, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, sum(new), 8, d, F16)
    _, clean, _ = mp.kv_attend(cache, batch, q, want_lse=True)
    bad = [(0, 1), (new[0] - 1, 7), (sum(new) - 1, 2)]
    for i, h in bad:
        q[i, h, 5] = float("nan")
    out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
    assert not status.any()
    for i, h in bad:
        assert torch.isnan(lse[i, h]) and torch.isnan(out[i, h]).all()
        clean[i, h] = lse[i, h] = 0
    assert torch.equal(lse, clean)


def test_captured_calls_have_scratch_of_their_own(cuda_lib):
    """Graphs captured without scratch of the caller's: later and larger calls on the stream of the capture do not take
    theirs away, and two that were captured on one stream run at once on two."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(47)
    lens, new = [60000, 30000], [1, 1]
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 2, 128, rng)
    cache, step = pool.cache(), batch_of(mp, table, lens, new)
    prompt = batch_of(mp, table, [60000, 700], [600, 600])
    q, _ = rows(rng, 2, 8, 128, BF16)
    r, _ = rows(rng, 2, 8, 128, BF16)
    long, _ = rows(rng, 1200, 8, 128, BF16)
    ws = mp.Workspace("cuda")
    want = [mp.kv_attend(cache, step, x, workspace=ws)[0] for x in (q, r)]
    want_long = mp.kv_attend(cache, prompt, long, workspace=ws)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs, outs = [], [torch.empty_like(q) for _ in range(2)]
    status = [torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(2)]
    with torch.cuda.stream(side):  # an eager step first, as a warm-up
        mp.kv_attend(cache, step, q)
    torch.cuda.synchronize()
    for x, out, st in zip((q, r), outs, status):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            mp.kv_attend(cache, step, x, out=out, status=st)
    with torch.cuda.stream(side):
        got = mp.kv_attend(cache, prompt, long)[0]
        torch.cuda.synchronize()
        # whatever scratch was given up on that stream is other tensors' now
        theirs = [torch.full((size,), 3, dtype=torch.uint8, device="cuda") for size in [1 << 20] * 64 + [16 << 20] * 4]
    torch.cuda.synchronize()
    assert torch.equal(got, want_long)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert all(bool((x == 3).all()) for x in theirs)


@pytest.mark.parametrize("group,d,dtype,causal,window", [
    (4, 128, BF16, True, 0), (4, 64, F16, True, 0), (3, 128, F16, True, 900), (1, 64, BF16, False, 0), (8, 128, BF16, True, 0)])
def test_attend_by_both_long_kernels(cuda_lib, group, d, dtype, causal, window):
    """Batches whose bound on what is cached passes 256 MB: sequences of up to 16 rows a head go to one kernel, the others to
    the second, and the joining has rows of the first and cuts of the second at once.  On either side of the 16 rows, of one
    row tile and of two, contexts cut between warps and between CTAs, sequences without tokens and without a past."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(100 * group + d)
    heads, block = 2, 64
    most = 16 // group
    seqs = [(5000, 1), (700, most), (900, most + 1), (0, 0), (3100, 300), (0, 2), (1, 1), (2500, 128 // group), (40, 0),
            (64, 64), (1300, 128 // group + 1), (33, most), (2, 5)]
    seqs += [(int(n), 1) for n in rng.integers(1, 6000, 12)] + [(int(n), 18) for n in rng.integers(18, 3000, 4)]
    order = rng.permutation(len(seqs))
    lens, new = [seqs[i][0] for i in order], [seqs[i][1] for i in order]
    table, n = R.make_table(lens, block, rng)
    bound = (256 << 20) // (len(lens) * heads * d * 2) // block * block + block  # tokens a sequence might hold
    wide = np.full((len(lens), bound // block), -1, np.int32)
    wide[:, :table.shape[1]] = table
    assert len(lens) * bound * heads * d * 2 > 256 << 20 and sum(new) != len(new) * max(new)
    pool = R.Pool(n, block, heads, d, rng)
    pool.vs[:] = np.exp2(rng.integers(-12, 3, pool.vs.shape))
    pool.ks[:] = np.exp2(rng.integers(-9, -5, pool.ks.shape))
    q, qx = rows(rng, sum(new), heads * group, d, dtype)
    out = check_attend(mp, pool, wide, lens, new, q, qx, d ** -0.5, causal, window, max_len=bound)
    # the same result from scratch that holds anything, and status of its own for either kind of sequence
    cache = pool.cache()
    few, many = order.tolist().index(0), order.tolist().index(4)
    wide[few, 0], wide[many, 0] = n, -1
    if window:  # what a window does not reach is not looked at
        wide[few, lens[few] // block], wide[many, lens[many] // block] = n, -1
    batch = batch_of(mp, wide, lens, new, max_len=bound)
    ptr = np.concatenate([[0], np.cumsum(new)])
    for fill in (0, 255):
        ws = mp.Workspace("cuda")
        ws.get(mp.kv_attend_workspace_bytes(cache, batch, heads * group))
        ws.buf.fill_(fill)
        again, _, status = mp.kv_attend(cache, batch, q, causal=causal, window=window, workspace=ws)
        assert status.tolist() == [int(b in (few, many)) for b in range(len(lens))]
        for b in range(len(lens)):
            if b not in (few, many):
                assert np.array_equal(again[ptr[b]:ptr[b + 1]].double().cpu().numpy(), out[ptr[b]:ptr[b + 1]])


def test_read_follows_the_tensor_that_is_given(cuda_lib):
    """kv_read with one of k and v, whatever type and layout it has: the other comes in the same type."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(59)
    lens, new = [100, 7], [33, 7]
    table, n = R.make_table(lens, 32, rng)
    pool = R.Pool(n, 32, 3, 64, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    want = [np.concatenate(x) for x in zip(*(R.held(pool, table, b, lens[b] - new[b], lens[b]) for b in range(2)))]
    for dtype in (F16, BF16, F32):
        for how in ("plain", "heads"):
            mine, _ = rows(rng, sum(new), 3, 64, dtype, how)
            for name in ("k", "v"):
                k, v, status = mp.kv_read(cache, batch, **{name: mine})
                assert (k if name == "k" else v) is mine and k.dtype == v.dtype == dtype and not status.any()
                for x, y in ((k, want[0]), (v, want[1])):
                    assert torch.equal(x.cpu(), torch.from_numpy(y).to(dtype))


@pytest.mark.parametrize("seqs", [[(300, 1), (90, 4)], [(6000, 3), (5000, 1)], [(400, 90), (65, 64)], [(5000, 300), (3000, 20)]])
@pytest.mark.parametrize("d,dtype", [(64, F16), (128, BF16)])
def test_attend_value_scales_as_far_apart_as_they_may_be(cuda_lib, seqs, d, dtype):
    """Value scales of 2^-80 among 2^20 (2^3 with outputs in f16), the small ones' tokens holding most of the weight, before
    and after the large ones': each weight counts in the sum although its values do not in the output."""
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(61)
    lens, new = [s[0] for s in seqs], [s[1] for s in seqs]
    table, n = R.make_table(lens, 32, rng)
    pool = R.Pool(n, 32, 2, d, rng)
    pool.ks[:] = 2.0 ** -8
    large, small = (2.0 ** 3 if dtype == F16 else 2.0 ** 20), 2.0 ** -80
    pool.vs[:] = small
    for b in range(2):
        pool.vs[table[b, 1::4]] = large
        pool.vs[table[b, 0]] = (large, small)[b]
    q, qx = rows(rng, sum(new), 4, d, dtype)
    want, want_lse, mag, size = R.attend(pool, table, lens, new, qx, d ** -0.5)
    out, lse, status = mp.kv_attend(pool.cache(), batch_of(mp, table, lens, new), q, want_lse=True)
    bound, lse_bound = R.attend_bounds(dtype, want, want_lse, mag, size)
    assert not status.any()
    # exponents of up to 2^7 in units of log 2 keep 2^-18: twice in a weight, and in the log-sum's two terms
    assert (np.abs(out.double().cpu().numpy() - want) <= bound + 2.0 ** -16 * mag).all()
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_bound + 2.0 ** -16).all()
