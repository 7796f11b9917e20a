"""The 4-bit cache at the sizes where a call takes another path: many requests,
items cut into many parts, each number of row tiles, odd widths, budgets past
what LDS holds.  Bounds as in test_gpu_kv.py."""
import ctypes

import numpy as np
import pytest
import torch

from tests import _kv_ref as ref
from tests.test_gpu_kv import Both, _check_weights, _cu, _rows, _tree_mask, oil  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,G", [(65, 1, 4), (130, 1, 1), (200, 3, 2), (130, 7, 5)])
def test_many_requests(oil, B, N, G):  # noqa: F811
    """More than 64 requests at ragged lengths (empty ones among them), in slots of another order."""
    rng = np.random.default_rng(B + N)
    lens = rng.integers(0, 70, B)
    lens[B // 2] = 900
    lens[[0, 63, 64, B - 1]] = [0, 33, 0, 64]
    c = Both(oil, B, 1, 64, 900)
    k, v = _rows(rng, B, 70, 1, 64), _rows(rng, B, 70, 1, 64)
    c.append(k, v, count=np.minimum(lens, 70))
    c.append(_rows(rng, 1, 830, 1, 64), _rows(rng, 1, 830, 1, 64), slots=[B // 2])
    slots = rng.permutation(B)
    n_nodes = rng.integers(0, N + 1, B).astype(np.int32)
    q, k, v = _rows(rng, B, N, G, 64), _rows(rng, B, N, 1, 64), _rows(rng, B, N, 1, 64)
    c.attend(q, k, v, n_nodes, _tree_mask(rng, B, N, n_nodes), slots=slots)
    c.attend(q, None, None, n_nodes, slots=slots)
    lse = c.ref.attend(q, scale=0.1, slots=slots)[1].astype(np.float32)
    count = rng.integers(0, N + 1, B).astype(np.int32)
    c.own.weigh(_cu(q, torch.bfloat16), _cu(lse), None, _cu(count), 0.1, Both._i32(slots))
    c.ref.weigh(q, lse, None, count, 0.1, slots)
    _check_weights(c, None, q, lse, 0.1)
    c.own.evict(40, 8)
    c.ref.evict(40, 8)
    torch.cuda.synchronize()
    for s in range(B):       # float32 weights order as the reference's do: they are far apart
        n = c.ref.pos[s].shape[1]
        assert int(c.own.lengths[s]) == n


@pytest.mark.parametrize("D", [8, 24, 40, 72, 104, 120])
@pytest.mark.parametrize("N,G", [(3, 2), (20, 1), (40, 2)])
def test_odd_widths(oil, D, N, G):  # noqa: F811
    rng = np.random.default_rng(D + N)
    lens = [0, 50, 97]
    c = Both(oil, 3, 2, D, 100)
    c.fill(rng, lens)
    n_nodes = np.array([N, N - 1, N], np.int32)
    q, k, v = _rows(rng, 3, N, 2 * G, D), _rows(rng, 3, N, 2, D), _rows(rng, 3, N, 2, D)
    c.attend(q, k, v, n_nodes, _tree_mask(rng, 3, N, n_nodes))
    c.attend(q, k, v, n_nodes)


@pytest.mark.parametrize("N", [4, 20, 45])
def test_value_ranges_by_row_tiles(oil, N):  # noqa: F811
    """Value rows whose scales differ by any factor, constant ones and zero ones among
    them, in tiles of their own and mixed, with one, two and three row tiles."""
    rng = np.random.default_rng(90 + N)
    n = 500
    size = np.ones((1, n, 1, 1), np.float32)
    size[0, 64:96] = 2.0 ** -7                 # a tile below what binary16 operands are taken at
    size[0, 130:140] = 2.0 ** -12
    size[0, 200] = 300.0                       # every tile after it is far below
    size[0, 300:330] = (10.0 ** rng.integers(-20, 3, (30, 1, 1))).astype(np.float32)
    k = _rows(rng, 1, n, 1, 128)
    v = ref.bf16((rng.standard_normal((1, n, 1, 128)) * size).astype(np.float32))
    v[0, 400:404] = 0.0
    v[0, 410] = -7.0
    c = Both(oil, 1, 1, 128, n)
    c.append(k, v)
    c.attend(_rows(rng, 1, N, 3, 128), _rows(rng, 1, N, 1, 128), _rows(rng, 1, N, 1, 128))


@pytest.mark.parametrize("N,G", [(2, 4), (4, 4), (17, 1)])
def test_masked_rows_do_not_reach_small_trees(oil, N, G):  # noqa: F811
    rng = np.random.default_rng(91 + N)
    c = Both(oil, 3, 1, 64, 40)
    c.fill(rng, [40, 0, 7])
    n_nodes = np.array([N, N - 1, N], np.int32)
    mask = _tree_mask(rng, 3, N, n_nodes)
    mask[:, :, 0] &= ~np.uint32(1 << 1)          # node 1 is seen by nobody
    q, k, v = _rows(rng, 3, N, G, 64), _rows(rng, 3, N, 1, 64), _rows(rng, 3, N, 1, 64)
    clean = c.attend(q, k, v, n_nodes, mask)
    k[:, 1], v[:, 1] = np.nan, -np.inf
    k[1, N - 1:], v[1, N - 1:], q[1, N - 1:] = np.inf, np.nan, np.nan
    again = c.attend(q, k, v, n_nodes, mask)
    assert np.array_equal(clean[0], again[0]) and np.array_equal(clean[1], again[1])
    v[0, 0, 0, 3], v[2, 0, 0, 9] = np.inf, np.nan
    c.attend(q, k, v, n_nodes, mask)


def test_one_item_in_many_parts(oil):  # noqa: F811
    """A single head so long that hundreds of workgroups share it, beside nothing and beside short ones."""
    rng = np.random.default_rng(92)
    n = 40000
    c = Both(oil, 3, 1, 64, n)
    c.fill(rng, [n, 3, 0])
    for N, G in ((1, 1), (1, 6), (9, 2), (30, 2)):
        q, k, v = _rows(rng, 3, N, G, 64), _rows(rng, 3, N, 1, 64), _rows(rng, 3, N, 1, 64)
        c.attend(q[:1], k[:1], v[:1])
        c.attend(q, k, v)


def test_no_lse_and_no_nodes(oil):  # noqa: F811
    rng = np.random.default_rng(93)
    c = Both(oil, 2, 2, 128, 60)
    c.fill(rng, [60, 0])
    q = _cu(_rows(rng, 2, 3, 4, 128), torch.bfloat16)
    out, _ = c.own.attend(q)
    got = torch.full_like(out, 7.0)
    ws = torch.empty((c.own._ws["attend", (2, 3, 4)].numel(),), dtype=torch.uint8, device="cuda")
    L, p = oil.lib(), lambda t: ctypes.c_void_p(t.data_ptr())
    st = L.oil_kv_attend(c.own.handle, None, 2, p(q), 512, 4, None, None, 0, None, None, 3, 128 ** -0.5, p(ws),
                         ws.numel(), p(got), None, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(got, out) and not got[1].any()


def test_evict_past_lds(oil):  # noqa: F811
    """More rows than the selection holds in LDS, equal weights among them."""
    rng = np.random.default_rng(94)
    n = 40000
    c = Both(oil, 1, 1, 8, n)
    w = np.round(rng.random((1, 1, n)) * 3000).astype(np.float32)
    c.append(_rows(rng, 1, n, 1, 8), _rows(rng, 1, n, 1, 8), weight=w)
    for keep, recent in ((38011, 500), (20000, 0), (77, 13)):
        c.own.evict(keep, recent)
        c.ref.evict(keep, recent)
        c.same()


def test_evict_many_tiles(oil):  # noqa: F811
    """So many destination tiles that each is one wave's."""
    rng = np.random.default_rng(95)
    B, H, keep, n = 8, 8, 4130, 4300
    c = Both(oil, B, H, 8, n)
    w = rng.random((B, H, n)).astype(np.float32)
    c.append(_rows(rng, B, n, H, 8), _rows(rng, B, n, H, 8), weight=w)
    c.own.evict(keep, 100)
    c.ref.evict(keep, 100)
    c.same()


def test_weigh_many_rows(oil):  # noqa: F811
    """Committed rows past the 64 that stand in LDS at a time, some of them with nothing to add."""
    rng = np.random.default_rng(96)
    c = Both(oil, 2, 1, 128, 200)
    c.fill(rng, [200, 31], weights=True)
    N, G = 50, 3
    q = _rows(rng, 2, N, G, 128)
    lse = c.ref.attend(q, scale=0.09)[1].astype(np.float32)
    lse[0, 21:43] = -np.inf                    # the second 64 rows and some before
    c.own.weigh(_cu(q, torch.bfloat16), _cu(lse), scale=0.09)
    c.ref.weigh(q, lse, scale=0.09)
    _check_weights(c, None, q, lse, 0.09)


def test_append_of_many_tiles(oil):  # noqa: F811
    """Tickets end at 64 workgroups a request: both sides, twice each."""
    rng = np.random.default_rng(97)
    c = Both(oil, 2, 3, 64, 2000)
    for n in (600, 620, 700, 30, 2):
        c.append(_rows(rng, 2, n, 3, 64), _rows(rng, 2, n, 3, 64), count=[n, n - 1])
        c.same()
    c.own.reset()
    c.ref.reset()
    c.same()


@pytest.mark.parametrize("N,G", [(1, 4), (6, 2), (20, 1), (20, 3)])
@pytest.mark.parametrize("e", [-90, 60, 100])
def test_powers_of_two_pass_through(oil, N, G, e):  # noqa: F811
    """Keys times 2^e under queries times 2^-e: the same bits throughout (at 2^-90 the
    keys' codes come from divisions, the queries' factors from the end of their range)."""
    rng = np.random.default_rng(98)
    q, k, v = _rows(rng, 2, N, 2 * G, 128), _rows(rng, 2, N, 2, 128), _rows(rng, 2, N, 2, 128)
    ck, cv = _rows(rng, 2, 333, 2, 128), _rows(rng, 2, 333, 2, 128)
    got = []
    for by in (np.float32(1.0), np.float32(2.0) ** np.float32(e)):
        c = oil.KvCache(2, 2, 128, 400)
        c.append(_cu(ck * by, torch.bfloat16), _cu(cv, torch.bfloat16), count=_cu(np.array([333, 41], np.int32)))
        t = [_cu(q / by, torch.bfloat16), _cu(k * by, torch.bfloat16), _cu(v, torch.bfloat16)]
        out, lse = c.attend(*t)
        c.weigh(t[0], lse)
        torch.cuda.synchronize()
        got.append((out, lse, c.weights.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert got[0][2].any() and torch.isfinite(got[0][1]).all()
