"""The 4-bit cache's refusals, on the host: no call here reaches a kernel.  And
the reference the GPU tests compare with, held to the definition's bounds."""
import ctypes

import numpy as np
import pytest

from tests import _kv_ref as ref
from tests.test_abi import _FakeBufs


@pytest.fixture(scope="module")
def L():
    import paper_2608_03839_amd as oil
    return oil.lib()


def test_sizes(L):
    assert L.oil_kv_bytes(1, 1, 128, 1) == 128 * 32 + 256
    assert L.oil_kv_bytes(1, 1, 128, 33) == 2 * (128 * 32 + 256)
    assert L.oil_kv_bytes(2, 3, 64, 64) == 6 * 2 * (64 * 32 + 256)
    assert L.oil_kv_bytes(1, 1, 72, 32) == 128 * 32 + 256
    assert L.oil_kv_bytes(5, 8, 128, 1 << 20) == 5 * 8 * (1 << 15) * (128 * 32 + 256)   # past 2^32
    for bad in ((0, 1, 64, 1), (1, 0, 64, 1), (1, 1, 0, 1), (1, 1, 60, 1), (1, 1, 136, 1), (1, 257, 64, 1),
                (1, 1, 64, 0), (65536, 1, 64, 1), (1, 1, 64, (1 << 30) + 1)):
        assert L.oil_kv_bytes(*bad) == 0, bad


def test_create_refuses(L):
    f = _FakeBufs()
    P, bad = f.aligned, f.misaligned
    h = ctypes.c_void_p()
    out = ctypes.byref(h)
    assert L.oil_kv_create(1, 1, 64, 32, P, P, P, P, None, None) == -1
    for args in ((0, 1, 64, 32), (1, 0, 64, 32), (1, 1, 65, 32), (1, 1, 64, 0), (70000, 1, 64, 32)):
        assert L.oil_kv_create(*args, P, P, P, P, None, out) == -1
    assert L.oil_kv_create(1, 300, 64, 32, P, P, P, P, None, out) == -3
    assert L.oil_kv_create(1, 1, 256, 32, P, P, P, P, None, out) == -3
    for i in range(4):
        bufs = [P] * 4
        bufs[i] = None
        assert L.oil_kv_create(1, 1, 64, 32, *bufs, None, out) == -1
    assert L.oil_kv_create(1, 1, 64, 32, bad, P, P, P, None, out) == -1
    assert L.oil_kv_create(1, 1, 64, 32, P, P, P, bad, None, out) == -1
    assert not h.value
    assert L.oil_kv_destroy(None) == -1


def test_calls_refuse_no_handle(L):
    f = _FakeBufs()
    P = f.aligned
    assert L.oil_kv_reset(None, None, 1, None) == -1
    assert L.oil_kv_append(None, None, 1, P, P, 1, 64, 1, None, None, None, None) == -1
    assert L.oil_kv_read(None, None, 1, 0, 1, P, P, 1, None) == -1
    assert L.oil_kv_attend_workspace_bytes(None, 1, 1, 1) == 0
    assert L.oil_kv_attend(None, None, 1, P, 64, 1, None, None, 0, None, None, 1, 1.0, P, 1 << 20, P, P, None) == -1
    assert L.oil_kv_weigh(None, None, 1, P, 64, 1, P, 1, None, None, 1.0, None) == -1
    assert L.oil_kv_evict_workspace_bytes(None, 1, 1) == 0
    assert L.oil_kv_evict(None, None, 1, 1, 0, P, 1 << 20, None) == -1


def test_reference_rows_are_near():
    """Every finite value of a held row is within half a step and the coverage
    of the row's range is whole: |x - held| <= s / 2 (1 + 2^-20)."""
    rng = np.random.default_rng(1)
    for size in (1e-3, 1.0, 1e4):
        x = (rng.standard_normal((500, 128)) * size + rng.standard_normal((500, 1)) * size * 3).astype(np.float32)
        c, s, z = ref.quantise(x)
        assert (z[:, 0] <= x.min(1)).all() and c.min() == 0 and c.max() == 15
        assert (np.abs(x - ref.held(x)) <= s.astype(np.float64) / 2 * (1 + 2.0 ** -20)).all()


def test_reference_evicts_lightest():
    rng = np.random.default_rng(2)
    c = ref.Cache(1, 1, 8, 20)
    x = rng.standard_normal((1, 20, 1, 8)).astype(np.float32)
    w = np.arange(20, dtype=np.float32)[None, None, ::-1].copy()
    c.append(x, x, weight=w)
    c.evict(6, 2)
    assert sorted(c.pos[0][0].tolist()) == [0, 1, 2, 3, 18, 19]
    assert c.pos[0][0].tolist() == [0, 1, 2, 3, 18, 19]
