"""The attention kernels' bounded waits run out cleanly (MP_ETIMEOUT), on the GPU.

A test build of the library (paper_2203_00448_gb300.build.build_test_hooks: waits bounded at about 8 ms, and the entry point
mp_test_kv_hold) holds the bytes of one unit of the cache back, as if they never came.  The warps that wait for them give
up after the bound, the call returns, the sequences that they were at work on report MP_ETIMEOUT, and the same call right
after, with nothing held, is right (the context is still usable).
"""
import numpy as np
import pytest
import torch

from tests import kv_refs as R
from tests.test_gpu_kv import batch_of, rows

pytestmark = pytest.mark.gpu


@pytest.fixture
def hooks(cuda_lib):
    """The package on the test build; yields its mp_test_kv_hold."""
    import ctypes

    from paper_2203_00448_gb300 import _lib, build

    path = build.build_test_hooks()
    plain, _lib._lib = _lib._lib, None
    try:
        hold = _lib.load(path).mp_test_kv_hold
        hold.argtypes, hold.restype = [ctypes.c_int64], None
        yield hold
        hold(-1)
    finally:
        _lib._lib = plain


@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float16)])
@pytest.mark.parametrize("kernel,lens,new,units", [
    ("few", [60000, 500, 9000], [1, 1, 1], (0, 1, 5, 7)),          # of the first sequence, which many warps share
    ("few", [60000, 500, 9000], [4, 4, 3], (0, 3)),
    ("many", [6000, 700, 3000], [600, 40, 200], (0, 1, 2, 4)),     # units of both row tiles
    ("many", [60000, 700, 30000], [30, 20, 25], (0, 1, 2, 6)),     # the tiles in turn
])
def test_attention_wait_runs_out(hooks, kernel, lens, new, units, d, dtype):
    import paper_2203_00448_gb300 as mp

    rng = np.random.default_rng(53)
    table, n = R.make_table(lens, 64, rng)
    pool = R.Pool(n, 64, 2, d, rng)
    cache, batch = pool.cache(), batch_of(mp, table, lens, new)
    q, _ = rows(rng, sum(new), 8, d, dtype)
    want, want_lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
    assert not status.any()
    first = new[0]
    for unit in units:
        hooks(unit)
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
        end.record()
        hooks(-1)
        assert status.tolist() == ([mp.ETIMEOUT, 0, 0] if kernel == "few" else [mp.ETIMEOUT] * 3)
        if kernel == "few":  # one warp gave up; the others' sequences are whole
            assert torch.equal(out[first:], want[first:]) and torch.equal(lse[first:], want_lse[first:])
        # 2^24 cycles, twice at most (the wait, and what it leaves in flight), at 1 GHz or more, beside the call itself
        assert start.elapsed_time(end) < 40
        out, lse, status = mp.kv_attend(cache, batch, q, want_lse=True)
        assert not status.any() and torch.equal(out, want) and torch.equal(lse, want_lse)
