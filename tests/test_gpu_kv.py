"""GPU parity of the 4-bit key/value cache against plain numpy (tests/_kv_ref.py).

Codes, positions, moves and lengths are exact.  Bounds of what is computed, u =
2^-24 (binary32), per row with A its largest sum of |scale q k|:
  scores  at most D + 8 roundings of sums no larger than A, and the same for
          the zero point, whose two parts may each exceed the score by the ratio
          |z| sum |q|, covered by A of the unreduced sums: dS = 4 (D + 8) u A'
          with A' = A + |S|; the tests take A' from sums over z and s c apart.
  lse     dS, the sum's own roundings (n / 64 + 64) u, and 8 u (1 + |lse|).
  out     half an ulp of bf16 (2^-8 of the value covers its neighbours), and of
          sum p |v|: 2^-8 for probabilities rounded to bf16 and 2 dS + 2^-16.
  weights relative 2 dS + 2^-18.
"""
import numpy as np
import pytest
import torch

from tests import _kv_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def oil():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_03839_amd as m
    m.lib()
    return m


def _cu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _rows(rng, *shape, offset=True):
    x = rng.standard_normal(shape).astype(np.float32)
    if offset:
        x = x * np.exp(0.3 * rng.standard_normal((*shape[:-1], 1))) + 1.5 * rng.standard_normal(shape[-1])
    return ref.bf16(x.astype(np.float32))


class Both:
    """A cache and its reference, driven together."""

    def __init__(self, oil, n_slots, H, D, cap):
        self.oil = oil
        self.own, self.ref = oil.KvCache(n_slots, H, D, cap), ref.Cache(n_slots, H, D, cap)
        self.n_slots, self.H, self.D, self.cap = n_slots, H, D, cap

    @staticmethod
    def _i32(x):
        return None if x is None else _cu(np.asarray(x, np.int32))

    def append(self, k, v, dtype=torch.bfloat16, nodes=None, count=None, weight=None, slots=None):
        self.own.append(_cu(k, dtype), _cu(v, dtype), self._i32(nodes), self._i32(count),
                        None if weight is None else _cu(weight.astype(np.float32)), self._i32(slots))
        self.ref.append(k, v, nodes, count, weight, slots)

    def fill(self, rng, lens, weights=False):
        """lens[s] rows in every slot."""
        for s, n in enumerate(lens):
            if n:
                w = np.exp(rng.standard_normal((1, self.H, n))).astype(np.float32) if weights else None
                self.append(_rows(rng, 1, n, self.H, self.D), _rows(rng, 1, n, self.H, self.D), weight=w, slots=[s])

    def same(self, weights=True):
        torch.cuda.synchronize()
        k, v = (x.cpu().numpy() for x in self.own.read(0, self.cap, dtype=torch.float32))
        pos, w, st = (x.cpu().numpy() for x in (self.own.positions, self.own.weights, self.own.state))
        for s in range(self.n_slots):
            n = self.ref.k[s].shape[1]
            assert st[s, 0] == n and st[s, 1] == self.ref.next[s] and st[s, 2] == 0
            assert np.array_equal(k[s, :, :n], self.ref.k[s].astype(np.float32), equal_nan=True)
            assert np.array_equal(v[s, :, :n], self.ref.v[s].astype(np.float32), equal_nan=True)
            assert not k[s, :, n:].any() and not v[s, :, n:].any()
            assert np.array_equal(pos[s, :, :n], self.ref.pos[s]) and (pos[s, :, n:] == -1).all()
            if weights:
                assert np.array_equal(w[s, :, :n], self.ref.w[s].astype(np.float32), equal_nan=True)
            assert not w[s, :, n:].any()

    def attend(self, q, k=None, v=None, n_nodes=None, mask=None, scale=None, slots=None, tensors=None):
        scale = self.D ** -0.5 if scale is None else scale
        B, N, Hq, D = q.shape
        if tensors is None:
            tensors = [None if x is None else _cu(x, torch.bfloat16) for x in (q, k, v)]
        m = None if mask is None else _cu(mask.view(np.int32))
        out, lse = self.own.attend(*tensors, self._i32(n_nodes), m, scale, self._i32(slots))
        torch.cuda.synchronize()
        out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        eo, el, size, spread = self.ref.attend(q, k, v, n_nodes, mask, scale, slots)
        ds = 4 * (D + 8) * U * (size + self._zero_size(q, scale, slots))
        n = self.cap + N
        fine = np.isfinite(el)
        assert np.array_equal(np.isnan(lse), np.isnan(el))
        assert np.array_equal(lse[~fine & ~np.isnan(el)], el[~fine & ~np.isnan(el)])
        bound = ds + (n / 64 + 64) * U + 8 * U * (1 + np.abs(np.where(fine, el, 0)))
        assert (np.abs(lse - el)[fine] <= bound[fine]).all(), np.abs(lse - el)[fine].max()
        bad = np.isnan(eo)
        assert np.array_equal(np.isnan(out), bad)
        okay = np.isfinite(eo)
        assert np.array_equal(out[~okay & ~bad], eo[~okay & ~bad])
        bound = 2.0 ** -8 * np.abs(eo) + (2.0 ** -8 + 2.0 ** -16 + 2 * ds[..., None]) * spread + 1e-37
        far = np.abs(out - eo)[okay] - bound[okay]
        assert (far <= 0).all(), far.max()
        return out, lse

    def _zero_size(self, q, scale, slots):
        """|scale| max |z| sum |q| of each row: the zero points' part of the scores, which s c may cancel."""
        B, N, Hq, D = q.shape
        size = np.zeros((B, N, Hq))
        for b, s in self.ref.named(slots, B):
            if self.ref.k[s].shape[1]:
                z = np.nanmax(np.abs(self.ref.k[s]), initial=0.0)
                size[b] = abs(scale) * z * np.abs(q[b].astype(np.float64)).sum(-1)
        return np.nan_to_num(size)


def _tree_mask(rng, B, N, n_nodes):
    mask = np.zeros((B, N, (N + 31) // 32), np.uint32)
    for b in range(B):
        for i in range(min(N, int(n_nodes[b]))):
            if i:
                mask[b, i] = mask[b, rng.integers(max(0, i - 6), i)]
            mask[b, i, i // 32] |= np.uint32(1 << (i % 32))
    return mask


# ------------------------------------------------------------------ append, read, reset
@pytest.mark.parametrize("D", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_and_read_exact(oil, D, dtype):
    rng = np.random.default_rng(D)
    c = Both(oil, 3, 2, D, 200)
    for n in (1, 30, 1, 33, 64, 5):          # tiles begun, ended and passed
        k, v = (rng.standard_normal((3, n, 2, D)).astype(np.float32) * 3 + 1 for _ in range(2))
        if dtype == torch.bfloat16:
            k, v = ref.bf16(k), ref.bf16(v)
        w = rng.random((3, 2, n)).astype(np.float32)
        c.append(k, v, dtype, weight=w, count=[n, n - 1, n // 2])
        c.same()
    c.own.reset(_cu(np.array([1], np.int32)))
    c.ref.reset([1])
    c.same()
    k = ref.bf16(rng.standard_normal((3, 7, 2, D)))
    c.append(k, -k, dtype)
    c.same()
    c.own.reset()
    c.ref.reset()
    c.same()


def test_read_range_and_bf16(oil):
    rng = np.random.default_rng(5)
    c = Both(oil, 2, 3, 96, 150)
    c.fill(rng, [101, 40])
    for first, n in ((0, 1), (31, 2), (33, 90), (149, 1), (64, 64)):
        k, v = c.own.read(first, n)
        k32, v32 = c.own.read(first, n, dtype=torch.float32)
        assert torch.equal(k, k32.to(torch.bfloat16)) and torch.equal(v, v32.to(torch.bfloat16))
        for s, m in enumerate((101, 40)):
            got = min(max(m - first, 0), n)
            assert np.array_equal(k32[s, :, :got].cpu().numpy(), c.ref.k[s][:, first:first + got].astype(np.float32))
            assert not k32[s, :, got:].any()
    k, _ = c.own.read(0, 40, slots=_cu(np.array([1, 7], np.int32)), dtype=torch.float32)
    assert np.array_equal(k[0].cpu().numpy(), c.ref.k[1].astype(np.float32)) and not k[1].any()


def test_append_extremes(oil):
    """Constant rows, tiny and huge ranges, offsets far from zero, rows that are not finite."""
    rng = np.random.default_rng(6)
    D = 64
    rows = [np.zeros(D), np.full(D, -0.0), np.full(D, 3.25), np.full(D, -1e-30), rng.standard_normal(D) * 1e-38,
            rng.standard_normal(D) * 1e-41, rng.standard_normal(D) * 1e30, 1000 + rng.standard_normal(D),
            -1000 + 1e-3 * rng.standard_normal(D), np.where(np.arange(D) == 5, np.nan, 1.0),
            np.where(np.arange(D) == 9, np.inf, 1.0), np.where(np.arange(D) == 9, -np.inf, 1.0),
            np.where(np.arange(D) % 2, 3.3e38, -3.3e38), np.where(np.arange(D) == 63, 1e6, 0.0)]
    x = np.array(rows, np.float32)[None, :, None, :]
    c = Both(oil, 1, 1, D, 64)
    c.append(x, x[:, ::-1].copy(), torch.float32)
    c.same()


def test_append_committed_path(oil):
    rng = np.random.default_rng(7)
    B, N, H, D = 4, 37, 2, 64
    c = Both(oil, 6, H, D, 120)
    nodes = np.full((B, N), -1, np.int32)
    count = np.array([0, 5, 36, -3], np.int32)
    for b in range(B):
        ids = np.sort(rng.permutation(np.arange(1, N))[:max(0, count[b])])
        nodes[b, :len(ids)] = ids
    for step in range(3):
        k, v = _rows(rng, B, N, H, D), _rows(rng, B, N, H, D)
        c.append(k, v, nodes=nodes, count=count, slots=[5, 0, 3, 2])
        c.same()
    nodes[1, 2] = 99                      # an id out of range ends the path
    nodes[2, 0] = -7
    c.append(_rows(rng, B, N, H, D), _rows(rng, B, N, H, D), nodes=nodes, count=count, slots=[5, 0, -1, 99])
    c.same()


def test_append_past_capacity(oil):
    rng = np.random.default_rng(8)
    c = Both(oil, 2, 2, 64, 45)
    for n in (40, 4, 9, 1):
        c.append(_rows(rng, 2, n, 2, 64), _rows(rng, 2, n, 2, 64), count=[n, min(n, 3)])
        c.same()


def test_strided_rows(oil):
    """k and v as slices of a fused projection's output, one and several rows."""
    rng = np.random.default_rng(9)
    for B, N in ((3, 9), (3, 1), (1, 5), (1, 1)):
        H, Hq, D = 2, 6, 80
        x = _rows(rng, B, N, Hq + 2 * H, D)
        t = _cu(x, torch.bfloat16)
        q, k, v = t[:, :, :Hq], t[:, :, Hq:Hq + H], t[:, :, Hq + H:]
        c = Both(oil, B, H, D, 64)
        c.fill(rng, [11] * B)
        c.attend(x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], tensors=[q, k, v])
        c.own.append(k, v)
        c.ref.append(x[:, :, Hq:Hq + H], x[:, :, Hq + H:])
        c.same()


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("D", [8, 64, 104, 128])
@pytest.mark.parametrize("G", [1, 4, 7])
def test_decode_lengths(oil, D, G):
    """Single tokens: slots from empty to several tiles, at every edge of one."""
    rng = np.random.default_rng(100 * D + G)
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 64, 100, 127, 128, 129, 300]
    H = 2
    c = Both(oil, len(lens), H, D, 300)
    c.fill(rng, lens)
    B = len(lens)
    q = _rows(rng, B, 1, H * G, D)
    k, v = _rows(rng, B, 1, H, D), _rows(rng, B, 1, H, D)
    c.attend(q, k, v)
    c.attend(q)                                  # the cache alone: an empty slot gives zeros and -inf
    out, lse = c.attend(q, slots=[13, -1, 3, 99, 0] + list(range(4, 13)))
    assert not out[1].any() and (lse[3] == -np.inf).all()


@pytest.mark.parametrize("N,G,H,D", [(2, 4, 2, 128), (5, 3, 1, 64), (17, 1, 3, 128), (33, 5, 1, 80), (61, 4, 2, 128),
                                     (65, 2, 2, 64), (100, 8, 1, 128)])
def test_trees(oil, N, G, H, D):
    rng = np.random.default_rng(N)
    lens = [0, 1, 45, 200, 513]
    B = len(lens)
    c = Both(oil, B, H, D, 520)
    c.fill(rng, lens)
    n_nodes = np.array([N, N - 1, max(1, N // 2), 0, N + 9], np.int32)
    mask = _tree_mask(rng, B, N, n_nodes)
    q, k, v = _rows(rng, B, N, H * G, D), _rows(rng, B, N, H, D), _rows(rng, B, N, H, D)
    c.attend(q, k, v, n_nodes, mask)
    c.attend(q, k, v, n_nodes)                   # causal


@pytest.mark.parametrize("N,G,D", [(200, 4, 128), (256, 1, 64), (256, 8, 128)])
def test_chunks(oil, N, G, D):
    rng = np.random.default_rng(N + G)
    c = Both(oil, 1, 1, D, 700)
    c.fill(rng, [641])
    c.attend(_rows(rng, 1, N, G, D), _rows(rng, 1, N, 1, D), _rows(rng, 1, N, 1, D))


def test_group_of_64(oil):
    rng = np.random.default_rng(64)
    c = Both(oil, 1, 2, 64, 90)
    c.fill(rng, [77])
    c.attend(_rows(rng, 1, 3, 128, 64), _rows(rng, 1, 3, 2, 64), _rows(rng, 1, 3, 2, 64))


def test_long_slots_in_parts(oil):
    """Lengths past what one workgroup takes, beside short ones."""
    rng = np.random.default_rng(65)
    lens = [5000, 1, 2999, 0]
    c = Both(oil, 4, 1, 128, 5000)
    c.fill(rng, lens)
    for N in (1, 7):
        q, k, v = _rows(rng, 4, N, 4, 128), _rows(rng, 4, N, 1, 128), _rows(rng, 4, N, 1, 128)
        c.attend(q, k, v)
        c.attend(q)


def test_masked_rows_do_not_reach(oil):
    """NaN and infinities in nodes past n_nodes, in nodes that no row sees, in
    nodes that some rows see (those alone are NaN), and in queries."""
    rng = np.random.default_rng(66)
    B, N, H, G, D = 2, 40, 2, 3, 128
    c = Both(oil, B, H, D, 100)
    c.fill(rng, [70, 0])
    n_nodes = np.array([33, 20], np.int32)
    mask = _tree_mask(rng, B, N, n_nodes)
    mask[:, :, 0] &= ~np.uint32(1 << 7)          # node 7 is seen by nobody, itself neither
    mask[1, 12] = 0                              # a row that sees nothing in an empty slot
    mask[:, :, 1] |= np.uint32(0xFE)             # bits past n_nodes
    q, k, v = _rows(rng, B, N, H * G, D), _rows(rng, B, N, H, D), _rows(rng, B, N, H, D)
    clean = c.attend(q, k, v, n_nodes, mask)
    for b in range(B):
        for bad, i in ((np.nan, 7), (np.inf, 7), (-np.inf, n_nodes[b]), (np.nan, N - 1)):
            k[b, i, :, ::3] = bad
            v[b, i, :, 1::3] = bad
        q[b, n_nodes[b]:] = np.nan
    again = c.attend(q, k, v, n_nodes, mask)
    assert np.array_equal(clean[0], again[0]) and np.array_equal(clean[1], again[1])
    v[0, 9, 0, 5] = np.nan                       # column 5 of the rows that see node 9
    v[0, 9, 0, 6] = np.inf
    v[1, 3, 1] = -np.inf
    q[0, 4, 2] = np.nan
    c.attend(q, k, v, n_nodes, mask)
    k[0, 11, 1, 0] = np.nan
    c.attend(q, k, v, n_nodes, mask)


def test_cached_row_not_finite(oil):
    rng = np.random.default_rng(67)
    c = Both(oil, 2, 2, 64, 100)
    c.fill(rng, [40, 40])
    k, v = _rows(rng, 1, 1, 2, 64), _rows(rng, 1, 1, 2, 64)
    k[0, 0, 0, 3], v[0, 0, 1, 9] = np.nan, np.inf
    c.append(k, v, slots=[1])
    c.attend(_rows(rng, 2, 3, 4, 64), _rows(rng, 2, 3, 2, 64), _rows(rng, 2, 3, 2, 64))


def test_stale_slots_do_not_reach(oil):
    """What a slot held before (NaN among it) is not seen after a reset."""
    rng = np.random.default_rng(68)
    c = Both(oil, 1, 1, 128, 70)
    bad = np.full((1, 70, 1, 128), np.nan, np.float32)
    c.append(bad, bad)
    c.own.reset()
    c.ref.reset()
    for n in (1, 4, 30):
        c.append(_rows(rng, 1, n, 1, 128), _rows(rng, 1, n, 1, 128))
        c.attend(_rows(rng, 1, 2, 4, 128), _rows(rng, 1, 2, 1, 128), _rows(rng, 1, 2, 1, 128))


@pytest.mark.parametrize("size", [1e-20, 1e-3, 30.0, 1e4])
def test_score_ranges(oil, size):
    """Queries so small that every score is 0, and so large that one position takes all."""
    rng = np.random.default_rng(69)
    c = Both(oil, 2, 1, 128, 600)
    c.fill(rng, [600, 37])
    q = ref.bf16(_rows(rng, 2, 5, 4, 128) * np.float32(size))
    k, v = _rows(rng, 2, 5, 1, 128), _rows(rng, 2, 5, 1, 128)
    c.attend(q, k, v)
    c.attend(q, k, v, scale=-0.3)
    c.attend(q, k, v, scale=0.0)


def test_value_ranges(oil):
    """Values of very unequal rows (scales of 1e-30 to 1e30) and constant rows; mixed magnitudes in a query."""
    rng = np.random.default_rng(70)
    c = Both(oil, 1, 1, 64, 300)
    k = _rows(rng, 1, 300, 1, 64)
    v = ref.bf16(rng.standard_normal((1, 300, 1, 64)).astype(np.float32)
                 * (10.0 ** rng.integers(-30, 30, (1, 300, 1, 1))).astype(np.float32))
    v[0, 50:60] = np.float32(2.5)
    c.append(k, v)
    q = ref.bf16(rng.standard_normal((1, 4, 3, 64)).astype(np.float32)
                 * (10.0 ** rng.integers(-12, 1, (1, 4, 3, 64))).astype(np.float32))
    c.attend(q, _rows(rng, 1, 4, 1, 64), _rows(rng, 1, 4, 1, 64))


def test_sink_and_many_light_positions(oil):
    """One heavy position beside thousands of light ones whose weights add up."""
    rng = np.random.default_rng(71)
    c = Both(oil, 1, 1, 64, 8000)
    k = np.zeros((1, 8000, 1, 64), np.float32)
    k[0, 17, 0, 0] = 64.0
    v = _rows(rng, 1, 8000, 1, 64) + 2
    c.append(k, ref.bf16(v))
    q = np.zeros((1, 1, 2, 64), np.float32)
    q[..., 0] = [0.1875, 0.25]
    c.attend(q, scale=1.0)


# ------------------------------------------------------------------ weights and eviction
def _check_weights(c, before, q, lse, scale):
    torch.cuda.synchronize()
    w = c.own.weights.cpu().numpy().astype(np.float64)
    for s in range(c.n_slots):
        n = c.ref.k[s].shape[1]
        if not n:
            continue
        a = abs(scale) * 2 * np.nanmax(np.abs(c.ref.k[s])) * np.abs(q.astype(np.float64)).sum(-1).max()
        ds = 4 * (c.D + 8) * U * a + 8 * U * np.abs(lse[np.isfinite(lse)]).max(initial=0.0)
        assert (np.abs(w[s, :, :n] - c.ref.w[s]) <= (2 * ds + 2.0 ** -18) * np.abs(c.ref.w[s])).all()
        assert not w[s, :, n:].any()


@pytest.mark.parametrize("N,G,H,D,commit", [(1, 4, 2, 128, 0), (1, 1, 3, 64, 0), (1, 7, 1, 40, 0), (40, 4, 2, 128, 6),
                                            (61, 8, 1, 128, 2), (256, 2, 1, 64, 255)])
def test_weigh(oil, N, G, H, D, commit):
    rng = np.random.default_rng(N + G)
    lens = [300, 0, 1, 33, 260]
    B = len(lens)
    c = Both(oil, B, H, D, 300)
    c.fill(rng, lens, weights=True)
    q = _rows(rng, B, N, H * G, D)
    scale = D ** -0.5
    lse = c.ref.attend(q, scale=scale)[1].astype(np.float32)
    nodes = np.full((B, N), -1, np.int32)
    count = np.minimum(rng.integers(0, commit + 1, B), N - 1).astype(np.int32)
    count[0] = commit
    for b in range(B):
        nodes[b, :count[b]] = np.sort(rng.permutation(np.arange(1, N))[:count[b]])
    for kw in (dict(nodes=nodes, count=count), dict(), dict(count=np.minimum(count + 1, N))):
        if N > 100 and not kw:
            continue
        c.own.weigh(_cu(q, torch.bfloat16), _cu(lse), *(Both._i32(kw.get(x)) for x in ("nodes", "count")), scale)
        c.ref.weigh(q, lse, kw.get("nodes"), kw.get("count"), scale)
        _check_weights(c, None, q, lse, scale)


def test_weigh_slots_and_empty_rows(oil):
    """Slots in another order; a row whose lse is -inf (it saw nothing) adds nothing, NaN queries of rows not committed neither."""
    rng = np.random.default_rng(73)
    c = Both(oil, 5, 2, 128, 64)
    c.fill(rng, [64, 40, 10, 64, 3])
    q = _rows(rng, 3, 6, 8, 128)
    lse = np.full((3, 6, 8), 3.0, np.float32)
    lse[1] = -np.inf
    q[:, 4:] = np.nan
    count = np.array([3, 3, 2], np.int32)
    c.own.weigh(_cu(q, torch.bfloat16), _cu(lse), None, _cu(count), 0.1, _cu(np.array([4, 0, 2], np.int32)))
    c.ref.weigh(q, lse, None, count, 0.1, [4, 0, 2])
    _check_weights(c, None, q[:, :4], lse, 0.1)


def test_weights_add_up(oil):
    """Over the cache alone, each head's weights grow by one a committed row."""
    rng = np.random.default_rng(74)
    c = Both(oil, 2, 2, 128, 500)
    c.fill(rng, [500, 123])
    q = _cu(_rows(rng, 2, 3, 8, 128), torch.bfloat16)
    _, lse = c.own.attend(q)
    c.own.weigh(q, lse)
    torch.cuda.synchronize()
    assert np.allclose(c.own.weights.double().sum(-1).cpu().numpy(), 12.0, rtol=1e-4)


@pytest.mark.parametrize("keep,recent", [(1, 0), (31, 5), (32, 32), (33, 0), (64, 10), (200, 64), (299, 1), (299, 299)])
def test_evict_exact(oil, keep, recent):
    rng = np.random.default_rng(keep)
    c = Both(oil, 4, 3, 64, 300)
    c.fill(rng, [300, keep, 0, min(300, keep + 1)], weights=True)
    c.own.evict(keep, recent)
    c.ref.evict(keep, recent)
    c.same()
    n = 300 - keep
    c.append(_rows(rng, 4, n, 3, 64), _rows(rng, 4, n, 3, 64), count=[n, n // 2, n, 0],
             weight=rng.random((4, 3, n)).astype(np.float32))
    c.own.evict(keep, min(recent, keep), slots=_cu(np.array([3, 1, 0], np.int32)))
    c.ref.evict(keep, recent, slots=[3, 1, 0])
    c.same()


def test_evict_ties_and_nan(oil):
    """Equal weights go by row, zeros of either sign are equal, NaN ranks lowest, infinities highest."""
    rng = np.random.default_rng(75)
    n = 2500
    c = Both(oil, 1, 4, 128, n)
    w = rng.integers(0, 4, (1, 4, n)).astype(np.float32)
    w[0, 1] = 0.0
    w[0, 1, ::2] = -0.0
    w[0, 2, rng.random(n) < 0.4] = np.nan
    w[0, 3, rng.random(n) < 0.1] = np.inf
    w[0, 3, rng.random(n) < 0.1] = -1.5
    c.append(_rows(rng, 1, n, 4, 128), _rows(rng, 1, n, 4, 128), weight=w)
    for keep, recent in ((2301, 100), (1100, 0), (1023, 700), (40, 3)):
        c.own.evict(keep, recent)
        c.ref.evict(keep, recent)
        c.same()


def test_evict_every_row_young_or_all_nan(oil):
    rng = np.random.default_rng(76)
    c = Both(oil, 2, 1, 64, 128)
    w = np.full((2, 1, 128), np.nan, np.float32)
    c.append(_rows(rng, 2, 128, 1, 64), _rows(rng, 2, 128, 1, 64), weight=w)
    c.own.evict(50, 50)
    c.ref.evict(50, 50)
    c.same()
    c.own.evict(20, 0)
    c.ref.evict(20, 0)
    c.same()


def test_attention_after_eviction(oil):
    rng = np.random.default_rng(77)
    c = Both(oil, 2, 2, 128, 400)
    c.fill(rng, [400, 390], weights=True)
    c.own.evict(150, 20)
    c.ref.evict(150, 20)
    c.attend(_rows(rng, 2, 9, 8, 128), _rows(rng, 2, 9, 2, 128), _rows(rng, 2, 9, 2, 128))


# ------------------------------------------------------------------ large offsets, streams, graphs
def test_offsets_past_32_bits(oil):
    """A slot that begins past 2^32 bytes of the buffer."""
    rng = np.random.default_rng(78)
    cap, H, D = 1 << 20, 8, 128
    own = oil.KvCache(5, H, D, cap)
    small = Both(oil, 1, H, D, 256)
    k, v = _rows(rng, 1, 200, H, D), _rows(rng, 1, 200, H, D)
    w = rng.random((1, H, 200)).astype(np.float32)
    slot = _cu(np.array([4], np.int32))
    own.append(_cu(k, torch.bfloat16), _cu(v, torch.bfloat16), weight=_cu(w), slots=slot)
    small.append(k, v, weight=w)
    q = _cu(_rows(rng, 1, 3, 32, D), torch.bfloat16)
    for _ in range(2):
        got, want = own.attend(q, slots=slot), small.own.attend(q)
        torch.cuda.synchronize()
        assert torch.allclose(got[1], want[1], rtol=0, atol=1e-5)
        assert torch.allclose(got[0].float(), want[0].float(), rtol=2 ** -7, atol=2 ** -7)
        for a, b in zip(own.read(0, 200, slots=slot), small.own.read(0, 200)):
            assert torch.equal(a, b)
        own.evict(90, 10, slots=slot)
        small.own.evict(90, 10)
    assert torch.equal(own.positions[4, :, :90], small.own.positions[0, :, :90])


def test_one_head_past_32_bits(oil):
    """One head's rows pass 2^31 bytes: 2^25 + 37 positions of width 8."""
    n, D = (1 << 25) + 37, 8
    own = oil.KvCache(1, 1, D, n)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    k = torch.randn((1, n, 1, D), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((1, n, 1, D), generator=g, device="cuda").to(torch.bfloat16)
    own.append(k, v)
    tail_k, tail_v = own.read(n - 40, 40, dtype=torch.float32)
    for got, x in ((tail_k, k), (tail_v, v)):
        want = ref.held(x[0, n - 40:, 0].float().cpu().numpy())
        assert np.array_equal(got[0, 0].cpu().numpy(), want.astype(np.float32))
    q = torch.zeros((1, 1, 2, D), device="cuda", dtype=torch.bfloat16)
    # a query along the last row, strong enough that rows like it decide
    q[0, 0, 0] = 6 * k[0, -1, 0]
    q[0, 0, 1] = 1.0
    out, lse = own.attend(q, scale=1.0)
    K, V = (x[0, 0] for x in own.read(0, n, dtype=torch.float32))
    for a in range(2):
        S = (K.double() * q[0, 0, a].double()).sum(1)   # no library product: one over 2^25 rows is wrong here
        want = torch.logsumexp(S, 0)
        p = torch.exp(S - want)
        assert abs(float(lse[0, 0, a]) - float(want)) <= 2e-4     # 2^25 terms: (n / 64) u at most 3e-2, 2e-4 as partial sums
        o, spread = ((p[:, None] * x).sum(0) for x in (V.double(), V.double().abs()))
        assert (out[0, 0, a].double() - o).abs().max() <= 2 ** -7 * spread.max()


def test_side_stream(oil):
    rng = np.random.default_rng(79)
    c = Both(oil, 2, 2, 64, 100)
    side = torch.cuda.Stream()
    k, v, q = (_cu(_rows(rng, 2, 50, h, 64), torch.bfloat16) for h in (2, 2, 4))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.own.append(k, v)
        out, lse = c.own.attend(q[:, :5].contiguous())
        c.own.weigh(q[:, :5].contiguous(), lse)
        c.own.evict(20, 3)
    side.synchronize()
    d = oil.KvCache(2, 2, 64, 100)
    d.append(k, v)
    out2, lse2 = d.attend(q[:, :5].contiguous())
    d.weigh(q[:, :5].contiguous(), lse2)
    d.evict(20, 3)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert torch.equal(c.own.positions, d.positions) and torch.equal(c.own.weights, d.weights)


def test_graph_replays(oil):
    """A step (attend, weigh, append of the committed path, evict) captured once and
    replayed, against the same steps run eagerly."""
    rng = np.random.default_rng(80)
    B, N, H, Hq, D, keep = 3, 13, 2, 8, 128, 60

    def start():
        cache = oil.KvCache(B, H, D, 80)
        r = np.random.default_rng(81)
        x = _rows(r, B, 57, H, D)
        cache.append(_cu(x, torch.bfloat16), _cu(-x, torch.bfloat16))
        return cache

    q, k, v = (torch.zeros((B, N, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    nodes = torch.zeros((B, N), dtype=torch.int32, device="cuda")
    count = torch.zeros((B,), dtype=torch.int32, device="cuda")
    out = (torch.empty((B, N, Hq, D), dtype=torch.bfloat16, device="cuda"),
           torch.empty((B, N, Hq), dtype=torch.float32, device="cuda"))

    def step(cache):
        o, lse = cache.attend(q, k, v, out=out)
        cache.weigh(q, lse, nodes, count)
        cache.append(k, v, nodes, count)
        cache.evict(keep, 8)

    def inputs(i):
        r = np.random.default_rng(200 + i)
        for t, h in ((q, Hq), (k, H), (v, H)):
            t.copy_(_cu(_rows(r, B, N, h, D), torch.bfloat16))
        n = np.full((B, N), -1, np.int32)
        cnt = r.integers(0, 6, B).astype(np.int32)
        for b in range(B):
            n[b, :cnt[b]] = np.sort(r.permutation(np.arange(1, N))[:cnt[b]])
        nodes.copy_(_cu(n))
        count.copy_(_cu(cnt))

    captured, eager = start(), start()
    warm = start()
    inputs(0)
    step(warm)                                   # kernels loaded before the capture
    for ws_key in warm._ws:                      # workspaces too
        captured._ws[ws_key] = torch.empty_like(warm._ws[ws_key])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for i in range(6):
        inputs(i)
        step(eager)
        want = [x.clone() for x in (*out, eager.positions, eager.weights, eager.state)]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*out, captured.positions, captured.weights, captured.state), want):
            assert torch.equal(a, b), i


def test_same_inputs_same_bits(oil):
    rng = np.random.default_rng(82)
    c = Both(oil, 2, 2, 128, 3000)
    c.fill(rng, [3000, 1500])
    q, k, v = (_cu(_rows(rng, 2, 9, h, 128), torch.bfloat16) for h in (8, 2, 2))
    first = [x.clone() for x in c.own.attend(q, k, v)]
    for _ in range(5):
        for a, b in zip(first, c.own.attend(q, k, v)):
            assert torch.equal(a, b)
