"""The 4-bit cache at the limits of what it holds: rows that are not finite in long
slots, values up to binary32's range, probabilities of a tree's own nodes, large
offsets and batches, and inputs whose results are exact.  u = 2^-24 as in
test_gpu_kv.py, where the bound on the scores is derived."""
import numpy as np
import pytest
import torch

from tests import _kv_ref as ref
from tests.test_gpu_kv import U, Both, _check_weights, _cu, _rows, _tree_mask, oil  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rows that are not finite
@pytest.mark.parametrize("n", [20, 600, 3000, 40000])
@pytest.mark.parametrize("N,G", [(1, 1), (5, 2), (30, 2)])
def test_not_finite_value_row_reaches_whatever_outweighs_it(oil, n, N, G):  # noqa: F811
    """A value row that is not finite makes the output of every row that sees it NaN,
    also where another position outweighs it by 2^369: in one workgroup (20 rows), in
    a few parts and in many."""
    rng = np.random.default_rng(n + N)
    for bad, top in ((5, n - 3), (n - 3, 5), (n // 2, n - 3)):
        k = np.zeros((2, n, 1, 64), np.float32)
        k[:, top, 0, 0] = 16.0
        v = _rows(rng, 2, n, 1, 64)
        v[1, bad, 0, 7] = np.nan
        c = Both(oil, 2, 1, 64, n)
        c.append(k, v)
        q = np.zeros((2, N, G, 64), np.float32)
        q[..., 0] = 16.0
        out, lse = c.attend(q, scale=1.0)
        assert np.isfinite(out[0]).all() and np.isnan(out[1]).all() and np.isfinite(lse).all()


# ------------------------------------------------------------------ ranges of values
LARGEST = float(np.float32(3.3895314e38))    # of bf16


def _sized(rng, shape, size):
    return ref.bf16((size * rng.uniform(-1, 1, shape)).astype(np.float32))


@pytest.mark.parametrize("size", [1e30, 1e32, 1e36, 1.6e38])
@pytest.mark.parametrize("N,G", [(1, 4), (3, 2), (20, 1), (45, 1)])
def test_large_values(oil, size, N, G):  # noqa: F811
    """Outputs are means of values: they stay within binary32 wherever the values do."""
    rng = np.random.default_rng(N)
    n = 2048
    c = Both(oil, 3, 1, 64, n)
    c.append(_rows(rng, 3, n, 1, 64), _sized(rng, (3, n, 1, 64), size), count=[n, 77, 0])
    q = ref.bf16(_rows(rng, 3, N, G, 64) * np.float32(0.1))
    k, v = _rows(rng, 3, N, 1, 64), _sized(rng, (3, N, 1, 64), size)
    assert np.isfinite(c.attend(q * 0, k, v)[0]).all()       # every position weighs the same
    assert np.isfinite(c.attend(q, k, v)[0]).all()
    c.attend(q)
    c.attend(q, k, v / np.float32(2.0 ** 100))               # the nodes' far below the cached
    small = Both(oil, 3, 1, 64, n)
    small.append(_rows(rng, 3, n, 1, 64), _rows(rng, 3, n, 1, 64), count=[n, 77, 0])
    small.attend(q, k, v)                                     # and far above


@pytest.mark.parametrize("N,G", [(1, 1), (20, 1), (45, 1)])
def test_large_offsets_of_values(oil, N, G):  # noqa: F811
    """Rows of one value and rows far from zero, up to the largest bf16, beside small ones."""
    rng = np.random.default_rng(7 * N)
    n = 700
    v = _rows(rng, 2, n, 1, 128)
    v[0, 100:200] = LARGEST
    v[0, 200:300] = -LARGEST
    v[0, 300:420] = ref.bf16((1e38 * rng.uniform(2, 3.3, (120, 1, 128))).astype(np.float32))
    v[1] = ref.bf16((1e37 * rng.uniform(1, 1.01, (n, 1, 128))).astype(np.float32))
    v[1, 600:] = 3.0
    c = Both(oil, 2, 1, 128, n)
    c.append(_rows(rng, 2, n, 1, 128), v)
    q = ref.bf16(_rows(rng, 2, N, G, 128) * np.float32(0.05))
    own = np.full((2, N, 1, 128), LARGEST, np.float32)
    for k, w in ((None, None), (_rows(rng, 2, N, 1, 128), own), (_rows(rng, 2, N, 1, 128), _rows(rng, 2, N, 1, 128))):
        c.attend(q, k, w)
        c.attend(q * 0, k, w)


def test_many_large_values(oil):  # noqa: F811
    rng = np.random.default_rng(11)
    n = 262144
    c = Both(oil, 1, 1, 8, n)
    c.append(_rows(rng, 1, n, 1, 8), _sized(rng, (1, n, 1, 8), 1e37))
    c.attend(np.zeros((1, 1, 2, 8), np.float32))
    c.attend(np.zeros((1, 9, 2, 8), np.float32))


@pytest.mark.parametrize("N", [1, 20])
def test_large_values_of_no_weight(oil, N):  # noqa: F811
    """Value rows 2^90 above the others whose probability is nothing leave the others' output as it is."""
    rng = np.random.default_rng(12)
    n = 900
    k = np.zeros((1, n, 1, 64), np.float32)
    k[0, 300:340, 0, 0] = -32.0
    v = ref.bf16(_rows(rng, 1, n, 1, 64) * np.float32(2.0 ** -30))
    v[0, 300:340] *= np.float32(2.0 ** 90)
    c = Both(oil, 1, 1, 64, n)
    c.append(k, v)
    q = np.zeros((1, N, 2, 64), np.float32)
    q[..., 0] = 16.0
    c.attend(q, scale=1.0)
    c.attend(q, np.zeros((1, N, 1, 64), np.float32), ref.bf16(_rows(rng, 1, N, 1, 64) * np.float32(2.0 ** -30)), scale=1.0)


# ------------------------------------------------------------------ workspace, units of several tiles
def test_attend_workspace_is_bounded(oil):  # noqa: F811
    """A call's workspace holds two parts of 48 rows for each of its workgroups (512), or of
    16 for 768, whatever the requests and nodes."""
    for D, H in ((64, 2), (128, 2), (128, 8)):
        c = oil.KvCache(512, H, D, 40)
        W = 64 if D <= 64 else 128
        bound = 768 * 32 + 2 * 512 * 48 * (W + 2) * 4
        for B in (1, 7, 64, 512):
            for N in (1, 4, 17, 65, 256):
                for G in (1, 4, 8, 64):
                    need = oil.lib().oil_kv_attend_workspace_bytes(c.handle, B, N, H * G)
                    assert 0 < need <= bound, (D, H, B, N, G, need)


def test_units_of_several_tiles(oil):  # noqa: F811
    """A capacity at which a call's list is counted in units of two tiles (342 row blocks
    over 2^23 tiles), slots short and long."""
    rng = np.random.default_rng(14)
    c = oil.KvCache(1, 1, 64, 1 << 28)
    r = Both(oil, 1, 1, 64, 5000)
    for n in (5, 40, 1235, 1900):
        k, v = _rows(rng, 1, n, 1, 64), _rows(rng, 1, n, 1, 64)
        c.append(_cu(k, torch.bfloat16), _cu(v, torch.bfloat16))
        r.append(k, v)
        q, k, v = _rows(rng, 1, 256, 64, 64), _rows(rng, 1, 256, 1, 64), _rows(rng, 1, 256, 1, 64)
        t = [_cu(x, torch.bfloat16) for x in (q, k, v)]
        got = [c.attend(*t), r.own.attend(*t)]
        torch.cuda.synchronize()
        assert torch.allclose(*(g[1] for g in got), rtol=0, atol=1e-5)
        assert torch.allclose(*(g[0].float() for g in got), rtol=2 ** -7, atol=2 ** -7)


# ------------------------------------------------------------------ probabilities
def _half_spacing(x):
    """Half the distance between bf16 values at |x|."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 8)


def _close(c, q, k, v, n_nodes, mask, roundoff):
    """The output within half a spacing of bf16, `roundoff` of sum p |v|, and the scores' error."""
    scale = c.D ** -0.5
    t = [None if x is None else _cu(x, torch.bfloat16) for x in (q, k, v)]
    out, _ = c.own.attend(*t, Both._i32(n_nodes), None if mask is None else _cu(mask.view(np.int32)), scale)
    torch.cuda.synchronize()
    out = out.float().cpu().numpy().astype(np.float64)
    want, _, size, spread = c.ref.attend(q, k, v, n_nodes, mask, scale)
    ds = 4 * (c.D + 8) * U * (size + c._zero_size(q, scale, None))
    off = (roundoff + 2.0 ** -17 + 2 * ds[..., None]) * spread
    bound = off + _half_spacing(np.abs(want) + off)
    assert (np.abs(out - want) <= bound).all(), ((np.abs(out - want) - bound) / spread.clip(1e-30)).max()


@pytest.mark.parametrize("N,G,D", [(2, 4, 64), (5, 4, 128), (17, 1, 128), (17, 2, 64), (61, 4, 128), (256, 1, 128)])
def test_probabilities_of_nodes(oil, N, G, D):  # noqa: F811
    """Nodes over an empty cache hold all the mass: their probabilities are two bf16 (2^-16)."""
    rng = np.random.default_rng(N + G)
    c = Both(oil, 3, 2, D, 40)
    n_nodes = np.array([N, max(1, N - 1), N], np.int32)
    q = ref.bf16(rng.standard_normal((3, N, 2 * G, D)).astype(np.float32))
    k, v = (ref.bf16(rng.standard_normal((3, N, 2, D)).astype(np.float32)) for _ in range(2))
    _close(c, q, k, v, n_nodes, _tree_mask(rng, 3, N, n_nodes), 2.0 ** -16)
    _close(c, q, k, v, n_nodes, None, 2.0 ** -16)


@pytest.mark.parametrize("N,G,D", [(1, 4, 128), (20, 1, 64), (45, 1, 128)])
@pytest.mark.parametrize("n", [2, 3, 9, 70])
def test_probabilities_of_cached_rows(oil, N, G, D, n):  # noqa: F811
    """Few cached rows, so that roundings do not average: probabilities in binary16 (2^-11)."""
    rng = np.random.default_rng(100 * N + n)
    c = Both(oil, 2, 2, D, 80)
    k, v = (ref.bf16(rng.standard_normal((2, n, 2, D)).astype(np.float32)) for _ in range(2))
    c.append(k, v)
    q = ref.bf16(rng.standard_normal((2, N, 2 * G, D)).astype(np.float32))
    _close(c, q, None, None, None, None, 2.0 ** -11)


@pytest.mark.parametrize("n", [1, 5, 32, 300])
@pytest.mark.parametrize("G", [4, 20, 40])
def test_values_that_cancel_their_zero_points(oil, n, G):  # noqa: F811
    """Equal value rows under any weights: the output is the row, to the weights' 2^-11, half a
    spacing of bf16 and 2^-14 of s c, which may be far larger than the value."""
    rng = np.random.default_rng(n + G)
    B, D = 60, 128
    c = oil.KvCache(B, 1, D, n)
    v = np.broadcast_to(_rows(rng, B, 1, 1, D), (B, n, 1, D)).copy()
    c.append(_cu(_rows(rng, B, n, 1, D), torch.bfloat16), _cu(v, torch.bfloat16))
    out, _ = c.attend(_cu(_rows(rng, B, 1, G, D), torch.bfloat16))
    torch.cuda.synchronize()
    out = out.float().cpu().numpy().astype(np.float64)[:, 0]
    codes, s, z = (x.astype(np.float64) for x in ref.quantise(v[:, :1, 0]))
    want = z + s * codes
    off = (2.0 ** -11 + 2.0 ** -16) * np.abs(want) + 2.0 ** -14 * s * codes
    assert (np.abs(out - want) <= off + _half_spacing(np.abs(want) + off)).all()


# ------------------------------------------------------------------ strides
def test_last_rows_of_long_projections(oil):  # noqa: F811
    """The last token's heads out of a fused projection of 2,800 rows a request: requests
    lie more than 2^24 elements apart."""
    rng = np.random.default_rng(15)
    fused = torch.zeros((2, 2800, 48, 128), dtype=torch.bfloat16, device="cuda")
    assert fused.stride(0) > 1 << 24
    x = _rows(rng, 2, 1, 48, 128)
    fused[:, -1:] = _cu(x, torch.bfloat16)
    last = fused[:, -1:]
    q, k, v = last[:, :, :32], last[:, :, 32:40], last[:, :, 40:]
    c = Both(oil, 2, 8, 128, 64)
    c.fill(rng, [11, 40])
    _, lse = c.attend(x[:, :, :32], x[:, :, 32:40], x[:, :, 40:], tensors=[q, k, v])
    lse = lse.astype(np.float32)
    c.own.weigh(q, _cu(lse))
    c.ref.weigh(x[:, :, :32], lse, scale=128 ** -0.5)
    _check_weights(c, None, x[:, :, :32], lse, 128 ** -0.5)
    c.own.append(k, v)
    c.ref.append(x[:, :, 32:40], x[:, :, 40:])
    c.same(weights=False)


def test_strides_past_64_bits_are_refused(oil):  # noqa: F811
    c = oil.KvCache(4, 2, 64, 40)
    x = torch.zeros((1 << 16,), dtype=torch.bfloat16, device="cuda")
    p, L = x.data_ptr(), oil.lib()
    for ld in (1 << 60, (1 << 57) + 8, 1 << 62):
        assert L.oil_kv_append(c.handle, None, 4, p, p, 1, ld, 2, None, None, None, None) == -1
        assert L.oil_kv_attend(c.handle, None, 4, p, ld, 2, None, None, 0, None, None, 2, 1.0, p, 1 << 16, p, p, None) == -1
        assert L.oil_kv_attend(c.handle, None, 4, p, 128, 2, p, p, ld, None, None, 2, 1.0, p, 1 << 16, p, p, None) == -1
        assert L.oil_kv_weigh(c.handle, None, 4, p, ld, 2, p, 2, None, None, 1.0, None) == -1


# ------------------------------------------------------------------ exact inputs
@pytest.mark.parametrize("N,G", [(1, 4), (9, 2), (20, 1), (45, 1)])
@pytest.mark.parametrize("n", [33, 700])
def test_one_position_takes_all(oil, N, G, n):  # noqa: F811
    """Large scores that are exact: keys of whole numbers 0 .. 15 that 4 bits hold as they
    are, queries of one large power of two.  Each row's winner leads by at least 64, so that
    the output is the winner's held value row and lse its score."""
    rng = np.random.default_rng(n + N)
    D = 64
    k = np.zeros((2, n, 1, D), np.float32)
    k[:, :, 0, 1] = 15.0                               # s = 1, z = 0 in every row
    for d in range(2, 34):
        k[:, d - 2, 0, d] = 9 + (d % 5)                # row d - 2 alone has column d
    v = _rows(rng, 2, n, 1, D)
    c = Both(oil, 2, 1, D, n)
    c.append(k, v)
    q = np.zeros((2, N, G, D), np.float32)
    winner = rng.integers(0, 32, (2, N, G))
    for b, i, a in np.ndindex(*winner.shape):
        q[b, i, a, 2 + winner[b, i, a]] = 64.0
    out, lse = c.own.attend(_cu(q, torch.bfloat16), scale=1.0)
    torch.cuda.synchronize()
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    for b, i, a in np.ndindex(*winner.shape):
        w = winner[b, i, a]
        score = 64.0 * (9 + ((w + 2) % 5))         # rounded factors and sums: 16 u of it, 64 u of the sum
        assert abs(lse[b, i, a] - score) <= (16 * (1 + score) + 64) * U
        want = c.ref.v[b][0, w]
        off = 2.0 ** -10 * np.abs(want).max()      # the probability's rounding to binary16, twice over
        assert (np.abs(out[b, i, a] - want) <= off + _half_spacing(np.abs(want) + off)).all()


# ------------------------------------------------------------------ eviction
def test_evict_of_many_requests(oil):  # noqa: F811
    """Which rows of more than 64 requests stay, at weights given with the rows."""
    rng = np.random.default_rng(16)
    B, n = 130, 70
    c = Both(oil, B, 2, 64, n)
    w = np.stack([rng.permutation(2 * n).reshape(2, n) for _ in range(B)]).astype(np.float32)
    c.append(_rows(rng, B, n, 2, 64), _rows(rng, B, n, 2, 64), count=rng.integers(0, n + 1, B), weight=w)
    c.own.evict(40, 8)
    c.ref.evict(40, 8)
    c.same()
    slots = rng.permutation(B)[:100]
    c.own.evict(17, 3, slots=Both._i32(slots))
    c.ref.evict(17, 3, slots=slots)
    c.same()


@pytest.mark.parametrize("D", [8, 128])
@pytest.mark.parametrize("keep,n", [(4130, 4300), (4128, 4300), (4101, 4600)])
def test_evict_by_one_wave_a_tile(oil, D, keep, n):  # noqa: F811
    """More than 8,192 destination tiles, budgets that end inside a tile and at its edge."""
    rng = np.random.default_rng(keep + D)
    B, H = 8, 8
    c = Both(oil, B, H, D, n)
    w = rng.random((B, H, n)).astype(np.float32)
    rows = [_rows(rng, B, n, H, D) for _ in range(2)]
    c.append(*rows, weight=w)
    c.own.evict(keep, 100)
    c.ref.evict(keep, 100)
    c.same()
