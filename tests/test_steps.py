"""Checks of arguments of the 4-bit cache, of kv_extend and of rotary, and the tests' own plain forms, without a GPU."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2203_00448_gb300 as mp
from paper_2203_00448_gb300 import _lib, build
from tests import kv4_refs as R4
from tests.test_kv import BAD_BATCHES, BAD_TOKENS, P, batch, tokens

E = _lib.EINVAL


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def made(base, **kw):
    for k, v in kw.items():
        setattr(base, k, v)
    return ctypes.byref(base)


def cache(**kw):
    return made(_lib.MpKv4Cache(10, 32, 2, 64, P, P), **kw)


def blocks(**kw):
    return made(_lib.MpKvBlocks(4, 3, 32, 20, P, P, None, None), **kw)


def step(**kw):
    return made(_lib.MpKvExtension(20, 8, 96, *[P] * 10), **kw)


def rotation(**kw):
    return made(_lib.MpRotation(32, 0, P, 1.0), **kw)


def test_cache_argument_errors(lib):
    bad = [dict(n_blocks=-1), dict(block_tokens=0), dict(block_tokens=48), dict(block_tokens=288), dict(n_heads=0), dict(head_dim=96),
           dict(k=None), dict(v=P + 8)]
    for c, b in [(cache(**x), batch()) for x in bad] + [(cache(), batch(**x)) for x in BAD_BATCHES] + [(None, batch()), (cache(), None)]:
        assert lib.mp_kv_four_write(c, b, tokens(), tokens(), P, None) == E
        assert lib.mp_kv_four_read(c, b, tokens(), tokens(), P, None) == E
        assert lib.mp_kv_four_attend(c, b, tokens(4), 0.1, 1, 0, tokens(4), None, P, P, 1 << 40, None) == E
        assert lib.mp_kv_four_attend_workspace_bytes(c, b, 4) == 0
    for t in BAD_TOKENS:
        for f in (lib.mp_kv_four_write, lib.mp_kv_four_read):
            assert f(cache(), batch(), t, tokens(), P, None) == E and f(cache(), batch(), tokens(), t, P, None) == E
        assert lib.mp_kv_four_attend(cache(), batch(), t, 0.1, 1, 0, tokens(4), None, P, P, 1 << 40, None) == E
    for f in (lib.mp_kv_four_write, lib.mp_kv_four_read):
        assert f(cache(), batch(), tokens(dtype=0), tokens(dtype=1), P, None) == E
        assert f(cache(), batch(), tokens(), tokens(), None, None) == E
    long = dict(max_blocks=1000, max_len=32000)

    def call(q=None, scale=0.1, causal=1, window=0, out=None, lse=None, ws=P, room=1 << 40):
        return lib.mp_kv_four_attend(cache(), batch(**long), q or tokens(4), scale, causal, window, out or tokens(4), lse, P, ws, room, None)

    assert call(q=tokens(4, dtype=2), out=tokens(4, dtype=2)) == E and call(out=tokens(2)) == E and call(q=tokens(5), out=tokens(5)) == E
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=scale) == E
    assert call(window=-1) == E and call(window=5, causal=0) == E and call(lse=P + 2) == E and call(ws=None) == E
    need = lib.mp_kv_four_attend_workspace_bytes(cache(), batch(**long), 4)
    assert need > 0 and call(room=need - 1) == _lib.ENOMEM
    assert lib.mp_kv_four_attend_workspace_bytes(cache(n_blocks=0, k=None, v=None), batch(**long), 4) == 0


def test_extend_argument_errors(lib):
    def call(b, s, ws=P, room=1 << 40):
        return lib.mp_kv_extend(b, s, ws, room, None)

    for bad in (dict(n_seqs=-1), dict(n_seqs=(1 << 28) + 1), dict(max_blocks=-1), dict(n_blocks=-1), dict(block_tokens=0), dict(block_tokens=40), dict(block_tokens=288),
                dict(table=None), dict(table=P + 2), dict(free=None), dict(first=P), dict(first=P + 1, room=P), dict(first=P, room=P + 2)):
        assert call(blocks(**bad), step()) == E and lib.mp_kv_extend_workspace_bytes(blocks(**bad)) == 0
    names = ("lens", "n_free", "n_new", "lens_out", "n_free_out", "step_lens", "token_ptr", "positions", "slots", "seq_status")
    for bad in [dict(n_tokens=-1), dict(max_tokens=-1), dict(max_len=-1), dict(max_len=97), dict(max_tokens=(1 << 28) + 1)] + \
            [{n: None} for n in names] + [{n: P + 2} for n in names]:
        assert call(blocks(), step(**bad)) == E
    assert call(None, step()) == E and call(blocks(), None) == E
    need = lib.mp_kv_extend_workspace_bytes(blocks())
    assert need > 0 and call(blocks(), step(), room=need - 1) == _lib.ENOMEM and call(blocks(), step(), ws=None) == E


def test_rotary_argument_errors(lib):
    def rows(heads=2, dtype=1, data=P):
        return ctypes.byref(_lib.MpTokens(data, heads * 64, 64, heads, dtype))

    def call(r=None, positions=P, n=4, d=64, q=rows(), k=rows(), qo=rows(), ko=rows()):
        return lib.mp_rotary(r or rotation(), positions, n, d, q, k, qo, ko, 0, None)

    for bad in (dict(dim=0), dict(dim=3), dict(dim=66), dict(dim=-2), dict(layout=2), dict(layout=-1), dict(turns=None), dict(turns=P + 4),
                dict(amplitude=math.nan), dict(amplitude=math.inf)):
        assert call(rotation(**bad)) == E
    assert lib.mp_rotary(None, P, 4, 64, rows(), rows(), rows(), rows(), 0, None) == E
    for bad in (dict(positions=None), dict(positions=P + 1), dict(n=-1), dict(d=63), dict(d=1026), dict(d=0), dict(q=None), dict(qo=None), dict(k=None),
                dict(ko=None), dict(q=None, qo=None, k=None, ko=None), dict(q=rows(3)), dict(qo=rows(dtype=0)), dict(k=rows(dtype=2)),
                dict(q=rows(dtype=3), qo=rows(dtype=3)), dict(q=rows(data=P + 1)), dict(ko=rows(data=None)), dict(q=rows(0), qo=rows(0))):
        assert call(**bad) == E


def test_binding_refusals():
    for bad in (dict(block_tokens=48), dict(head_dim=80), dict(n_heads=0), dict(k=torch.zeros(4, 2, 100, dtype=torch.uint8)),
                dict(k=torch.zeros(4 * 2 * 1088 + 16, dtype=torch.uint8)[8:-8].view(4, 2, 1088))):
        with pytest.raises(ValueError):
            mp.KvCache4(**{**dict(n_blocks=4, block_tokens=32, n_heads=2, head_dim=64, device="cpu"), **bad})
    c = mp.KvCache4(3, 64, 5, 128, "cpu")
    assert 3 * mp.KvCache4.block_bytes(64, 5, 128) == c.k.numel() + c.v.numel()
    with pytest.raises(AttributeError):
        c.k = c.v
    i32 = dict(dtype=torch.int32)
    for bad in (dict(block_tokens=40), dict(n_seqs=-1), dict(first=torch.zeros(4, **i32)), dict(free=torch.zeros(20, **i32)),
                dict(lens=torch.zeros(3, **i32)), dict(table=torch.zeros(4, 3)),
                dict(first=torch.zeros(4, **i32), room=torch.zeros(4, **i32), free=torch.zeros(20, **i32), n_free=torch.zeros(1, **i32))):
        with pytest.raises(ValueError):
            mp.KvBlocks(**{**dict(n_seqs=4, max_blocks=3, block_tokens=32, n_blocks=20, device="cpu"), **bad})
    b = mp.KvBlocks(4, 3, 32, 20, device="cpu")
    assert b.free.tolist() == list(range(19, -1, -1)) and b.n_free.item() == 20 and not b.lens.any()
    with pytest.raises(ValueError, match="run on a GPU"):
        mp.kv_extend(b, torch.zeros(4, **i32), 0)
    r = mp.Rotary(32, device="cpu")
    with pytest.raises(ValueError, match="run on a GPU"):
        mp.rotary(r, torch.zeros(2, **i32), torch.zeros(2, 2, 64))
    for bad in (dict(dim=3), dict(dim=0), dict(layout="other"), dict(base=0.0), dict(scaling={"kind": "none"}), dict(scaling={"kind": "linear"}),
                dict(scaling={"kind": "linear", "factor": 0.0}), dict(amplitude=math.inf), dict(frequencies=[1.0]),
                dict(scaling={"kind": "bands", "factor": 2.0, "original": 100, "low": 4.0, "high": 1.0}),
                dict(frequencies=[math.nan] * 16), dict(frequencies=[1.0] * 16, scaling={"kind": "linear", "factor": 2.0})):
        with pytest.raises(ValueError):
            mp.Rotary(**{**dict(dim=32, device="cpu"), **bad})


def test_calls_check_their_tensors(monkeypatch):
    """With a library that does nothing: what reaches it, and what is refused before."""
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: (reached.append(name), 256 if name.endswith("_bytes") else 0)[1]

    monkeypatch.setattr(_lib, "load", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    i32 = dict(dtype=torch.int32)
    r = mp.Rotary(32, device="cpu")
    r._index = 0
    at, q = torch.zeros(2, **i32), torch.zeros(2, 3, 64)
    for args, kw in (((at.long(), q), {}), ((at[:1], q), {}), ((at, q[0]), {}), ((at, q.double()), {}), ((at, None), {}), ((at, q, q.half()), {}),
                     ((at, q, q[..., :32]), {}), ((at, q[..., :16]), {}), ((at, q), dict(k_out=q)), ((at, q), dict(q_out=q[:1])),
                     ((at, q.transpose(1, 2)), {}), ((at, q), {})):  # the last: tensors of another device than the frequencies'
        with pytest.raises(ValueError):
            mp.rotary(r, *args, **kw)
    b = mp.KvBlocks(4, 3, 32, 20, device="cpu")
    b._index = 0
    new = torch.zeros(4, **i32)
    ws = type("W", (), {"get": lambda self, n: (P, n)})()
    for args, kw in (((new.long(), 4), {}), ((new[:2], 4), {}), ((new, -1), {}), ((new, 4), dict(max_len=97)), ((new, 4), dict(max_len=-1)),
                     ((new, 4), dict(max_tokens=-1)), ((new, 4), dict(max_tokens=1 << 40)), ((new, 4), dict(lens=new[:1])), ((new, 4), dict(n_free=new))):
        with pytest.raises(ValueError):
            mp.kv_extend(b, *args, workspace=ws, **kw)
    assert "mp_kv_extend" not in reached and "mp_rotary" not in reached
    first = mp.kv_extend(b, new, 4, workspace=ws)
    assert reached[-1] == "mp_kv_extend" and first.batch.max_len == 96 and first.batch.max_tokens == 4
    assert mp.kv_extend(b, new, 4, step=first, workspace=ws) is first
    with pytest.raises(ValueError):
        mp.kv_extend(b, new, 5, step=first, workspace=ws)
    with pytest.raises(ValueError):
        mp.kv_extend(mp.KvBlocks(4, 3, 32, 20, device="cpu"), new, 4, step=first, workspace=ws)


@pytest.mark.parametrize("kind", [mp.KvCache, mp.KvCache4])
def test_steps_go_with_caches_of_their_block_size(kind):
    """Blocks of another size are other tokens' places, even where the step's lengths fit into the table's columns."""
    blocks = mp.KvBlocks(2, 4, 64, 10, device="cpu")
    step = mp.KvStep(blocks, 3, 2, 100)
    assert step.batch._for(kind(10, 64, 2, 64, "cpu"))[1] == (3, 2, 64)
    for other in (32, 96, 128):
        with pytest.raises(ValueError, match="blocks of 64 tokens"):
            step.batch._for(kind(10, other, 2, 64, "cpu"))
    # a batch of the user's own tables may be of any
    own = mp.KvBatch(blocks.table, blocks.lens, step.batch.token_ptr, 3, 2, 100)
    for other in (32, 64):
        own._for(kind(10, other, 2, 64, "cpu"))


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("hq,hk", [(0, 3), (3, 0), (0, 0), (2, 3)])
def test_rotary_of_no_heads(monkeypatch, hq, hk, inverse):
    """A tensor without heads has nothing to turn; the other one is turned all the same."""
    from paper_2203_00448_gb300 import rotation

    reached = []

    class Library:
        def mp_rotary(self, *args):
            reached.append(args[4:8])
            return 0

    monkeypatch.setattr(_lib, "load", Library)
    monkeypatch.setattr(rotation, "_away", lambda *args: False)
    monkeypatch.setattr(rotation, "_stream", lambda *args: 0)
    at, q, k = torch.zeros(2, dtype=torch.int32), torch.zeros(2, hq, 64), torch.zeros(2, hk, 64)
    for given in ({}, dict(q_out=q, k_out=k)):
        reached.clear()
        outs = mp.rotary(mp.Rotary(32, device="cpu"), at, q, k, inverse=inverse, **given)
        assert [x.shape for x in outs] == [q.shape, k.shape]
        if hq == hk == 0:
            assert not reached
            continue
        (qi, ki, qo, ko), = reached
        for heads, x, i, o in ((hq, q, qi, qo), (hk, k, ki, ko)):
            assert (i is None) == (o is None) == (heads == 0)
            assert heads == 0 or i.data == x.data_ptr()
        for o, out in ((qo, outs[0]), (ko, outs[1])):
            assert o is None or o.data == out.data_ptr()


def test_frequencies():
    """Each kind against its definition at single pairs, and what the integer turns stand for."""
    f, a = mp.rotary_frequencies(128)
    assert a == 1 and f[0] == 1 and abs(f[-1] - 10000 ** (-126 / 128)) < 1e-18
    g, _ = mp.rotary_frequencies(128, scaling={"kind": "linear", "factor": 4.0})
    assert torch.equal(g, f / 4)
    g, _ = mp.rotary_frequencies(128, scaling={"kind": "base", "factor": 4.0})
    assert g[0] == 1 and abs(g[-1] / f[-1] - 0.25) < 1e-12
    g, a = mp.rotary_frequencies(128, scaling={"kind": "parts", "factor": 8.0, "original": 4096, "fast": 32.0, "slow": 1.0})
    turns = 4096 * f / (2 * math.pi)
    assert abs(a - (0.1 * math.log(8) + 1)) < 1e-15
    assert torch.allclose(g[turns > 40], f[turns > 40], rtol=1e-12) and torch.allclose(g[turns < 0.9], f[turns < 0.9] / 8, rtol=1e-12)
    assert ((g <= f * (1 + 1e-12)) & (g >= f / 8 * (1 - 1e-12))).all()
    g, a = mp.rotary_frequencies(128, scaling={"kind": "bands", "factor": 8.0, "original": 4096, "low": 1.0, "high": 4.0})
    assert a == 1 and torch.equal(g[turns > 4], f[turns > 4]) and torch.allclose(g[turns < 1], f[turns < 1] / 8, rtol=1e-15)
    r = mp.Rotary(4, frequencies=[math.pi, -math.pi / 2], device="cpu")
    assert [int(t) % (1 << 64) for t in r.turns] == [1 << 63, 3 << 62]


def test_amplitude_of_parts_is_1_up_to_a_factor_of_1():
    """Only longer contexts need the larger amplitude: ln of a factor below 1 would make it less than 1."""
    for factor, want in ((0.25, 1.0), (1.0, 1.0), (1.5, 0.1 * math.log(1.5) + 1), (16.0, 0.1 * math.log(16) + 1)):
        scaling = {"kind": "parts", "factor": factor, "original": 4096, "fast": 32.0, "slow": 1.0}
        assert mp.rotary_frequencies(64, scaling=scaling)[1] == want and mp.Rotary(64, scaling=scaling, device="cpu").amplitude == want


def test_turns_are_as_near_as_doubles():
    """Turns a position times 2^64, against pi from its series 16 atan(1/5) - 4 atan(1/239) in whole numbers of 400 bits: the
    division in doubles and the double of 2 pi leave less than 2^-52 of a frequency's turns, the last rounding half a unit."""
    one = 1 << 400

    def atan(n):
        total, power, k = 0, one // n, 0
        while power:
            total += (-1) ** k * (power // (2 * k + 1))
            power //= n * n
            k += 1
        return total

    two_pi = 2 * (16 * atan(5) - 4 * atan(239))
    given = mp.rotary_frequencies(128)[0].tolist() + [-f for f in mp.rotary_frequencies(40, base=500000.0)[0].tolist()] + \
        [0.0, 3.0, math.pi, -math.pi / 2, 1e-300, 2.0 ** -70, 12345.678]
    r = mp.Rotary(2 * len(given), frequencies=given, device="cpu")
    for f, t in zip(given, r.turns.tolist()):
        n, d = f.as_integer_ratio()
        want = Fraction(n << 464, d * two_pi)
        off = abs((t - want + (1 << 63)) % (1 << 64) - (1 << 63))
        assert off <= abs(want) / 2 ** 52 + Fraction(1, 2), f


def test_plain_quantisation():
    rng = np.random.default_rng(0)
    assert R4.SCALES[183] == 240 and (np.diff(R4.SCALES) > 0).all()
    assert np.array_equal(R4.SCALES, (np.arange(184, dtype=np.uint16) << 7).view(np.float16).astype(float))
    x = rng.standard_normal((200, 32)) * np.exp2(rng.integers(-22, 8, (200, 1)))
    code, byte = R4.quantise(x)
    for i in range(0, 200, 9):
        assert byte[i] == R4.scale_byte(np.abs(x[i]).max())
    off = np.abs((code - 8.0) * R4.SCALES[byte][:, None] - x)
    assert (off <= R4.SCALES[byte][:, None] / 2 * (1 + 1e-12)).all()


def test_plain_layout_is_a_layout():
    for d in (64, 128):
        pool = R4.Pool(2, 64, 3, d, np.random.default_rng(1))
        for keys in (True, False):
            at, half, scale = pool.places(keys)
            assert sorted((2 * at + half).reshape(-1)) == list(range(32 * d)) and sorted(scale.reshape(-1)) == list(range(16 * d, 17 * d))
        got = pool.from_stored(*pool.stored())
        assert all(np.array_equal(x, y) for x, y in zip(got, (pool.k, pool.ks, pool.v, pool.vs)))
