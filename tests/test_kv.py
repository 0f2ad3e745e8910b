"""The key/value cache operators' checks of arguments and the tests' own plain forms, without a GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2203_00448_gb300 as mp
from paper_2203_00448_gb300 import _lib, build
from tests import kv_refs as R

P = 0x10000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def cache(**kw):
    c = _lib.MpKvCache(10, 32, 2, 64, P, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def batch(**kw):
    b = _lib.MpKvBatch(4, 3, 8, 96, 20, P, P, P)
    for k, v in kw.items():
        setattr(b, k, v)
    return ctypes.byref(b)


def tokens(heads=2, dtype=1, data=P):
    return ctypes.byref(_lib.MpTokens(data, heads * 64, 64, heads, dtype))


BAD_CACHES = [dict(n_blocks=-1), dict(block_tokens=0), dict(block_tokens=48), dict(block_tokens=288), dict(n_heads=0),
              dict(head_dim=96), dict(head_dim=256), dict(k=None), dict(v=P + 8), dict(k_scale=None), dict(v_scale=P + 2)]
BAD_BATCHES = [dict(n_seqs=-1), dict(max_blocks=-1), dict(max_tokens=-1), dict(max_len=97), dict(max_len=-1),
               dict(n_tokens=-1), dict(table=None), dict(lens=P + 1), dict(token_ptr=P + 4), dict(token_ptr=None),
               dict(max_tokens=(1 << 28) + 1), dict(max_blocks=1 << 24, max_len=(1 << 28) + 1)]
BAD_TOKENS = [tokens(3), tokens(0), tokens(dtype=3), tokens(dtype=-1), tokens(data=None), tokens(data=P + 1), None]


def test_host_argument_errors(lib):
    """Fake device addresses: every call fails its checks before anything could be enqueued."""
    E = _lib.EINVAL
    for c, b in [(cache(**x), batch()) for x in BAD_CACHES] + [(cache(), batch(**x)) for x in BAD_BATCHES] + \
            [(None, batch()), (cache(), None)]:
        assert lib.mp_kv_write(c, b, tokens(), tokens(), P, None) == E
        assert lib.mp_kv_read(c, b, tokens(), tokens(), P, None) == E
        assert lib.mp_kv_attend(c, b, tokens(4), 0.1, 1, 0, tokens(4), None, P, P, 1 << 40, None) == E
        assert lib.mp_kv_attend_workspace_bytes(c, b, 4) == 0
    for t in BAD_TOKENS:
        for f in (lib.mp_kv_write, lib.mp_kv_read):
            assert f(cache(), batch(), t, tokens(), P, None) == E
            assert f(cache(), batch(), tokens(), t, P, None) == E
        assert lib.mp_kv_attend(cache(), batch(), t, 0.1, 1, 0, tokens(4), None, P, P, 1 << 40, None) == E
        assert lib.mp_kv_attend(cache(), batch(), tokens(4), 0.1, 1, 0, t, None, P, P, 1 << 40, None) == E
    for f in (lib.mp_kv_write, lib.mp_kv_read):
        assert f(cache(), batch(), tokens(dtype=0), tokens(dtype=1), P, None) == E  # two types
        assert f(cache(), batch(), tokens(), tokens(), None, None) == E
        assert f(cache(), batch(), tokens(), tokens(), P + 2, None) == E


def test_attend_argument_errors(lib):
    E = _lib.EINVAL

    long = dict(max_blocks=1000, max_len=32000)  # a context that is shared among CTAs, which takes scratch

    def call(q=None, scale=0.1, causal=1, window=0, out=None, lse=None, status=P, ws=P, room=1 << 40):
        return lib.mp_kv_attend(cache(), batch(**long), q or tokens(4), scale, causal, window, out or tokens(4), lse, status, ws,
                                room, None)

    assert call(q=tokens(4, dtype=2), out=tokens(4, dtype=2)) == E  # 32-bit queries
    assert call(q=tokens(4, dtype=0)) == E  # another type than the output's
    assert call(out=tokens(2)) == E
    assert call(q=tokens(5), out=tokens(5)) == E  # no whole groups
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=scale) == E
    assert call(window=-1) == E and call(window=5, causal=0) == E
    assert call(lse=P + 2) == E and call(status=None) == E
    need = lib.mp_kv_attend_workspace_bytes(cache(), batch(**long), 4)
    assert need > 0
    assert call(room=need - 1) == _lib.ENOMEM
    assert call(ws=None) == E and call(ws=P + 8) == E
    assert lib.mp_kv_attend_workspace_bytes(cache(), batch(), 3) == 0
    assert lib.mp_kv_attend_workspace_bytes(cache(), batch(n_seqs=0), 4) == 0


def test_binding_refusals():
    with pytest.raises(ValueError):
        mp.KvCache(4, 48, 2, 64, "cpu")
    with pytest.raises(ValueError):
        mp.KvCache(4, 32, 2, 80, "cpu")
    with pytest.raises(ValueError):
        mp.KvCache(4, 32, 2, 64, k=torch.zeros(4, 2, 2047, dtype=torch.uint8))
    with pytest.raises(ValueError):
        mp.KvCache(4, 32, 2, 64, "cpu", k_scale=torch.zeros(4, 2, dtype=torch.float64))
    c = mp.KvCache(4, 32, 2, 64, "cpu")
    table, lens, ptr = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for bad in ((table.long(), lens, ptr), (table[0], lens, ptr), (table, lens.long(), ptr), (table, lens, ptr.int()),
                (table, lens, ptr[:2]), (table.t()[:, :1].expand(2, 2), lens, ptr)):
        with pytest.raises(ValueError):
            mp.KvBatch(*bad, n_tokens=2)
    b = mp.KvBatch(table, lens, ptr, n_tokens=2)
    x = torch.zeros(2, 2, 64)
    for bad in (x[:1], x[0], x[..., :32], x.double(), torch.zeros(2, 3, 64), torch.zeros(2, 64, 2).transpose(1, 2)):
        with pytest.raises(ValueError):
            mp.kv_write(c, b, bad, x)
        with pytest.raises(ValueError):
            mp.kv_write(c, b, x, bad)
    for bad in (x[:1], x[0], x[..., :32], x.double()):
        with pytest.raises(ValueError):
            mp.kv_attend(c, b, bad)


def test_block_bytes():
    c = mp.KvCache(3, 64, 5, 128, "cpu")
    assert 3 * mp.KvCache.block_bytes(64, 5, 128) == sum(t.numel() * t.element_size() for t in (c.k, c.v, c.k_scale, c.v_scale))


def test_plain_e4m3_rounding():
    """The tests' own rounding against a brute-force search, and its ties."""
    rng = np.random.default_rng(0)
    grid = R.VALUES[np.isfinite(R.VALUES)]
    x = np.concatenate([rng.standard_normal(2000) * np.exp2(rng.integers(-14, 9, 2000)), [0.0, 448.0, 500.0, -1e9, 2.0 ** -10]])
    got = R.VALUES[R.to_byte(x)]
    best = np.abs(np.minimum(np.abs(x), 448) * np.sign(x) - grid[:, None]).min(0)
    assert np.array_equal(np.abs(np.clip(x, -448, 448) - got), best)
    assert R.VALUES[R.to_byte(np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10]))].tolist() == [16.0, 20.0, 0.0, 2.0 ** -8]
    assert R.scale_of(448.0) == 1 and R.scale_of(448.1) == 2 and R.scale_of(224.0) == 0.5 and R.scale_of(0.0) == 2.0 ** -60


def test_empty_pool_needs_no_scratch(lib):
    """No kernel that walks a context may be launched over a pool without blocks, so none has scratch; each route's sizes."""
    none = dict(n_blocks=0, k=None, v=None, k_scale=None, v_scale=None)
    for sizes in (dict(max_tokens=1), dict(max_tokens=1, max_blocks=1000, max_len=32000), dict(max_tokens=40, n_tokens=160),
                  dict(max_tokens=40, n_tokens=44, max_blocks=1 << 18, max_len=1 << 23)):
        assert lib.mp_kv_attend_workspace_bytes(cache(**none), batch(**sizes), 4) == 0
    assert lib.mp_kv_attend_workspace_bytes(cache(), batch(max_tokens=40, n_tokens=160), 4) > 0


def test_attributes_are_not_replaced():
    """The C structs hold addresses and bounds: a tensor or bound put in place of another would not be seen by any call."""
    c = mp.KvCache(4, 32, 2, 64, "cpu")
    b = mp.KvBatch(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    for x, names in ((c, ("k", "v", "k_scale", "v_scale", "n_blocks", "block_tokens", "n_heads", "head_dim", "device")),
                     (b, ("table", "lens", "token_ptr", "n_tokens", "max_tokens", "max_len", "n_seqs", "device"))):
        for name in names:
            had = getattr(x, name)
            with pytest.raises(AttributeError):
                setattr(x, name, had.clone() if isinstance(had, torch.Tensor) else 77)
            with pytest.raises(AttributeError):
                delattr(x, name)
            assert getattr(x, name) is had
    at = b.lens.data_ptr()
    b.lens += 1  # in place: the same tensor
    b.lens[0] = 5
    assert b.lens.tolist() == [5, 1] and b.lens.data_ptr() == at
    c.note = b.note = 1  # what a program hangs on them is its own


def test_batch_and_cache_on_one_device():
    """A batch that has served a cache is still refused for one of the same shape on another device."""
    b = mp.KvBatch(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    near, far = (mp.KvCache(4, 32, 2, 64, device) for device in ("cpu", "meta"))
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    mp.kv_attend_workspace_bytes(near, b, 4)
    for _ in range(2):
        for call in (lambda: mp.kv_attend_workspace_bytes(far, b, 4), lambda: mp.kv_write(far, b, x, x),
                     lambda: mp.kv_read(far, b), lambda: mp.kv_attend(far, b, x)):
            with pytest.raises(ValueError, match="batch is on cpu, the cache on meta"):
                call()


def test_tensors_in_host_memory_are_refused(monkeypatch):
    """No call hands a kernel an address of host memory: with a cache, batch and tokens on the CPU, each stops before the
    library is called."""

    class Library:
        def __getattr__(self, name):
            def call(*args):
                launched.append(name)
                return _lib.OK if name != "mp_kv_attend_workspace_bytes" else 0

            return call

    launched = []
    monkeypatch.setattr(_lib, "load", Library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    c = mp.KvCache(4, 32, 2, 64, "cpu")
    b = mp.KvBatch(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    for call in (lambda: mp.kv_write(c, b, x, x), lambda: mp.kv_read(c, b), lambda: mp.kv_read(c, b, x.dtype, k=x, v=x),
                 lambda: mp.kv_attend(c, b, x), lambda: mp.kv_attend(c, b, x, out=x, want_lse=True)):
        with pytest.raises(ValueError, match="run on a GPU"):
            call()
    assert not [name for name in launched if name != "mp_kv_attend_workspace_bytes"]


def test_import_without_cuda_in_pytorch():
    """A PyTorch built without CUDA has no raw streams; the package can be imported there all the same (its planner's
    host-side parts and checks need no GPU)."""
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "import torch; del torch._C._cuda_getCurrentRawStream; import paper_2203_00448_gb300 as mp; mp.KvCache(1, 32, 1, 64, 'cpu')"
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True, timeout=300)


def test_calls_run_on_the_device_of_the_cache(monkeypatch):
    """With another device current, a call makes the cache's current for its launch and puts the other back; a stream has to
    be the cache's device's.  Two devices, both made up."""
    from contextlib import contextmanager
    from types import SimpleNamespace

    from paper_2203_00448_gb300 import kv

    now, launches = [1], []

    @contextmanager
    def device(index):
        had, now[0] = now[0], index
        yield
        now[0] = had

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "mp_kv_attend_workspace_bytes":
                    return 0
                launches.append((name, now[0], args[-1]))
                return _lib.OK

            return call

    monkeypatch.setattr(_lib, "load", Library)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: device(s.device_index))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    monkeypatch.setattr(kv, "_tokens", lambda name, t, cache, shape: _lib.MpTokens(0, 64, 64, 2, 0))
    c = mp.KvCache(4, 32, 2, 64, "cpu")
    c._index = 0
    b = mp.KvBatch(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    calls = [lambda **kw: mp.kv_write(c, b, x, x, **kw), lambda **kw: mp.kv_read(c, b, **kw), lambda **kw: mp.kv_attend(c, b, x, **kw)]
    for call in calls:
        call()
        call(stream=SimpleNamespace(device_index=0))
        with pytest.raises(ValueError, match="stream is on device 1"):
            call(stream=SimpleNamespace(device_index=1))
    assert [x[0] for x in launches] == ["mp_kv_write"] * 2 + ["mp_kv_read"] * 2 + ["mp_kv_attend"] * 2
    assert all(x[1:] == (0, 100) for x in launches) and now == [1]


def test_caches_start_on_16_byte_boundaries(lib):
    """A pool that every call would refuse is refused at once: the size of the scratch asked for with it, 0, would otherwise
    be kept for valid ones of its shape."""
    shape = (4, 2, 32 * 64)
    room = torch.zeros(4 * 2 * 32 * 64 + 64, dtype=torch.uint8)
    start = -room.data_ptr() % 16
    at = [room[start + i:start + i + 4 * 2 * 32 * 64].view(shape) for i in (0, 8, 1, 16)]
    for bad in (dict(k=at[1], v=at[0]), dict(k=at[0], v=at[2]), dict(k=at[1])):
        with pytest.raises(ValueError, match="16-byte"):
            mp.KvCache(4, 32, 2, 64, "cpu", **bad)
    c = mp.KvCache(4, 32, 2, 64, k=at[0], v=at[3])
    b = mp.KvBatch(torch.zeros(2, 1000, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    assert mp.kv_attend_workspace_bytes(c, b, 4) > 0


def test_bounds_past_32_bits(monkeypatch):
    """Numbers that 32 bits do not hold do not come out of them as others: bounds are refused, a window is as good as none."""
    table, lens, ptr = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for bad in (dict(max_tokens=(1 << 32) + 5), dict(max_tokens=-1), dict(max_len=(1 << 32) + 64), dict(max_len=-1 << 32),
                dict(max_len=(1 << 28) + 1), dict(max_tokens=(1 << 28) + 1)):
        with pytest.raises(ValueError, match="2\\^28"):
            mp.KvBatch(table, lens, ptr, 2, **bad)
    c = mp.KvCache(4, 256, 2, 64, "cpu")
    wide = mp.KvBatch(torch.zeros(2, 1, dtype=torch.int32), lens, ptr, 2)
    assert wide._for(c)[0]._obj.max_len == 256
    # a table of 2^24 + 1 columns, which nobody reads here
    long = mp.KvBatch(torch.empty(2, (1 << 24) + 1, dtype=torch.int32), lens, ptr, 2)
    assert long._for(c)[0]._obj.max_len == 1 << 28

    windows = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "mp_kv_attend":
                    windows.append(args[5])
                return _lib.OK

            return call

    monkeypatch.setattr(_lib, "load", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(mp.kv, "_tokens", lambda name, t, cache, shape: _lib.MpTokens(0, 64, 64, 2, 0))
    c._index = 0
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    for window in (0, 7, (1 << 32) + 7, 1 << 63, -5, -(1 << 32) + 7):
        mp.kv_attend(c, wide, x, window=window)
    assert windows == [0, 7, (1 << 31) - 1, (1 << 31) - 1, -1, -1]


def test_scratch_of_an_empty_pool_is_not_kept_for_others(lib):
    """An empty pool takes no scratch; a pool with blocks of the same shape, asked for with the same batch, does."""
    b = mp.KvBatch(torch.zeros(2, 1000, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), 2)
    none, some = (mp.KvCache(n, 32, 2, 64, "cpu") for n in (0, 4))
    for _ in range(2):
        assert mp.kv_attend_workspace_bytes(none, b, 4) == 0
        assert mp.kv_attend_workspace_bytes(some, b, 4) > 0
