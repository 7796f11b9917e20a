"""Packed prompts at the ends of binary32: scores up to its range and past it."""
import math

import pytest
import torch

from tests import _prompt_ref as ref

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def oil():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_03839_amd as m
    m.lib()
    return m


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(shape, seed=5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)


def _f32(x):
    return torch.tensor(x, dtype=torch.float32).item()


def _one_column(n, Hq, H, D, product, keys):
    """q, k whose products are product * keys[j], exactly: one column of each is not zero.  q is a power
    of two, about the square root of the product."""
    q = torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda")
    a = 2.0 ** (math.frexp(abs(product))[1] // 2)
    q[..., 1] = a
    k[..., 1] = (product / a * keys).to(torch.bfloat16)[:, None]
    assert (k[:, 0, 1].double() == product / a * keys.double()).all()
    return q, k


def _exact(q, k, v, scale):
    """out, lse, sum of weights times |v|, in 64 bits, of one causal sequence."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, size = (torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.zeros((T, Hq), dtype=torch.float64, device="cuda")
    unseen = torch.ones((T, T), dtype=torch.bool, device="cuda").triu(1)
    for head in range(Hq):
        s = (scale * (q[:, head].double() @ k[:, head // G].double().T)).masked_fill(unseen, -INF)
        m = s.amax(1, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(1, keepdim=True)
        lse[:, head] = (m + total.log())[:, 0]
        out[:, head] = p / total @ v[:, head // G].double()
        size[:, head] = p / total @ v[:, head // G].double().abs()
    return out, lse, size


# (rows, query heads, heads, columns): one tile and several, two waves and four, both widths
SIZES = [(1, 1, 1, 8), (150, 4, 2, 8), (150, 2, 1, 72), (2100, 16, 16, 8), (1100, 32, 4, 128)]
# q . k of the keys that count most
PRODUCTS = [2.0 ** 13, -2.0 ** 20, 2.0 ** 24, 7516192768.0, 3221225472.0, -2.0 ** 31, 2.0 ** 40, -2.0 ** 60, 2.0 ** 60,
            2.0 ** 126, -1.75 * 2.0 ** 127, 1.75 * 2.0 ** 127]


@pytest.mark.parametrize("n,Hq,H,D", SIZES)
@pytest.mark.parametrize("scale", [1.0, _f32(128 ** -0.5), -0.75])
def test_large_scores(oil, n, Hq, H, D, scale):
    """Every key at one score, or one in ten a quarter nearer to zero: differences of 2^11 times the scale at
    least, so that keys weigh the same or nothing."""
    v = _normal((n, H, D))
    for product in PRODUCTS:
        for keys in (torch.ones(n), torch.where(torch.arange(n) % 10 == 3, 0.75, 1.0)):
            q, k = _one_column(n, Hq, H, D, product, keys.cuda())
            out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=scale)
            w_out, w_lse, size = _exact(q, k, v, scale)
            # weights alike, rounded to bf16 alike; sums of n values and of n weights, the quotient, bf16
            far = 2 * 2.0 ** -8 * w_out.abs() + (n + 8) * 2.0 ** -23 * size
            assert ((out.double() - w_out).abs() <= far).all(), (product, keys[3:4])
            # the score, the logarithm and their sum
            far = 2.0 ** -23 * (w_lse.abs() + 1) + 2.0 ** -22 * math.log(n + 1)
            assert ((lse.double() - w_lse).abs() <= far).all(), (product, keys[3:4])


@pytest.mark.parametrize("at", [0, 5, 100, 2000])
@pytest.mark.parametrize("D", [16, 104])
def test_one_large_score(oil, at, D):
    """A key whose score leaves the others' far behind, in the first tile or a later one, before it and
    after it ordinary rows; the other head's rows are ordinary throughout."""
    n = 2100
    q, k, v = _normal((n, 2, D), 1), _normal((n, 2, D), 2), _normal((n, 2, D), 3)
    clean_out, clean_lse = oil.prompt_attend(q, k, v, _int([0, n]))
    scale = 1 / math.sqrt(D)
    for size in (2.0 ** 10, 2.0 ** 32, 2.0 ** 60):
        qq, kk = q.clone(), k.clone()
        qq[:, 1, 0] = size
        kk[:, 1, 0] = 0.0
        kk[at, 1, 0] = size
        out, lse = oil.prompt_attend(qq, kk, v, _int([0, n]))
        assert torch.equal(out[:, 0], clean_out[:, 0]) and torch.equal(lse[:, 0], clean_lse[:, 0])
        w_out, w_lse, far_out, far_lse = ref.attend(qq[:at, 1:], kk[:at, 1:], v[:at, 1:], [0, at], scale)
        assert ((out[:at, 1:].double() - w_out).abs() <= far_out).all()
        # one weight and out, to bf16; where the row is made of it alone, nothing is rounded
        assert ((out[at:, 1].double() - v[at, 1].double()).abs() <= 2.01 * 2.0 ** -8 * v[at, 1].double().abs()).all()
        if size > 2.0 ** 30:
            assert (out[at:, 1] == v[at, 1]).all()
        score = scale * size * size + scale * (qq[at:, 1, 1:].double() @ kk[at, 1, 1:].double())
        # D products and sums, scaled
        assert ((lse[at:, 1].double() - score).abs() <= (D + 4) * 2.0 ** -23 * score).all()


@pytest.mark.parametrize("n,Hq,H,D", SIZES)
def test_scores_past_the_range(oil, n, Hq, H, D):
    """Above it the row is NaN, below it the score is -inf."""
    v = _normal((n, H, D))
    for at in sorted({0, n // 2, n - 1}):
        keys = torch.zeros(n, device="cuda")
        keys[at] = 1.0
        q, k = _one_column(n, Hq, H, D, 2.0 ** 127, keys)
        out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=4.0)
        assert torch.isnan(out[at:]).all() and torch.isnan(lse[at:]).all()
        assert torch.isfinite(out[:at]).all() and torch.isfinite(lse[:at]).all()
        weight = oil.prompt_weigh(q, k, lse, _int([0, n]), scale=4.0)
        assert torch.isnan(weight).all()
        # that key alone weighs nothing
        out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=-4.0)
        seen = torch.ones((n, n), dtype=torch.float64, device="cuda").tril()
        seen[:, at] = 0.0
        count = seen.sum(1)
        values = v.double().repeat_interleave(Hq // H, 1).flatten(1)
        want = (seen @ values / count.clamp(min=1.0)[:, None]).view(n, Hq, D)
        size = (seen @ values.abs() / count.clamp(min=1.0)[:, None]).view(n, Hq, D)
        far = 2 * 2.0 ** -8 * want.abs() + (n + 8) * 2.0 ** -23 * size
        assert ((out.double() - want).abs() <= far).all()
        w_lse = count.log()[:, None].expand(n, Hq)
        assert torch.equal(lse == -INF, w_lse == -INF)
        some = w_lse > -INF
        assert ((lse.double() - w_lse)[some].abs() <= 2.0 ** -22 * (1 + w_lse[some])).all()


def _weigh(q, k, lse, last, scale):
    """weight (H, T) of one sequence and its bound, in 64 bits from the lse given."""
    T, Hq, D = q.shape
    H = k.shape[1]
    weight, far = (torch.zeros((H, T), dtype=torch.float64, device="cuda") for _ in range(2))
    seen = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
    seen[:max(0, T - last)] = False
    for head in range(Hq):
        h, size = head // (Hq // H), lse[:, head, None].double()
        s = scale * (q[:, head].double() @ k[:, h].double().T)
        x = s - size
        p = torch.where(seen, torch.exp(x), 0.0)
        # the difference, its product with log2 e, the exponential; below 2^12 both sides' products as well
        e = (x.abs() + 1) * 2.0 ** -22 + torch.where(size.abs() < 4096, (s.abs() + size.abs()) * 2.0 ** -22, 0.0)
        weight[h] += p.sum(0)
        far[h] += torch.where(seen, p * e, 0.0).sum(0)
    return weight, far + weight * (T * (Hq // H) + 8) * 2.0 ** -24 + 2.0 ** -126


@pytest.mark.parametrize("n,Hq,H,D", SIZES)
@pytest.mark.parametrize("scale", [1.0, _f32(128 ** -0.5), -0.75])
def test_weights_of_large_scores(oil, n, Hq, H, D, scale):
    """lse as it rounds to binary32, and as attention gives it."""
    v = _normal((n, H, D))
    for product in PRODUCTS:
        for keys in (torch.ones(n), torch.where(torch.arange(n) % 10 == 3, 0.75, 1.0)):
            q, k = _one_column(n, Hq, H, D, product, keys.cuda())
            for lse in (_exact(q, k, v, scale)[1].float(), oil.prompt_attend(q, k, v, _int([0, n]), scale=scale)[1]):
                for last in (n, 70):
                    got = oil.prompt_weigh(q, k, lse, _int([0, n]), last=last, scale=scale)
                    want, far = _weigh(q, k, lse, last, scale)
                    # beside lse's last place a score may be past all exponentials: infinities have no difference
                    near = ((got.double() - want).abs() <= far) | (got == want.float())
                    assert near.all(), (product, last, keys[3:4])


@pytest.mark.parametrize("D", [16, 104])
def test_weights_beside_large_scores(oil, D):
    """One head of a group asks with scores past 2^12, the other with ordinary ones.  Whole numbers, so
    that every score is exact."""
    n = 700
    q, k, v = (_normal((n, h, D), i).float().mul(1.5).round().to(torch.bfloat16) for i, h in ((1, 4), (2, 2), (3, 2)))
    q[:, 1] *= 2048.0
    lse = _exact(q, k, v, 0.25)[1].float()
    assert (lse[200:, 1] > 4096).all() and (lse[:, 0] < 4096).all()
    for last in (n, 130):
        got = oil.prompt_weigh(q, k, lse, _int([0, n]), last=last, scale=0.25)
        want, far = _weigh(q, k, lse, last, 0.25)
        assert ((got.double() - want).abs() <= far).all()


@pytest.mark.parametrize("n,Hq,H,D", SIZES)
def test_scale_zero(oil, n, Hq, H, D):
    """Finite rows' scores are 0, their products in binary32's range or not; others' are NaN."""
    q, k, v = (_normal((n, h, D), i) for i, h in ((1, Hq), (2, H), (3, H)))
    q[..., 3], k[..., 3] = 2.0 ** 70, 2.0 ** 70
    k[n // 2, :, 3] = -2.0 ** 70
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=0.0)
    count = torch.arange(1, n + 1, dtype=torch.float64, device="cuda")[:, None]
    # the logarithm is right to a unit, 2^-23 of it; ln 2, the product and its sum with the score to half of one each
    assert ((lse.double() - count.log()).abs() <= (2.0 ** -23 + 3 * 2.0 ** -24) * count.log()).all()
    for last in (n, 17):
        weight = oil.prompt_weigh(q, k, lse, _int([0, n]), last=last, scale=0.0)
        rows = torch.where(torch.arange(n, device="cuda") >= n - last, 1 / count[:, 0], 0.0) * (Hq // H)
        want = rows.flip(0).cumsum(0).flip(0)
        # lse, its product with log2 e, the exponential, sums
        far = want * ((math.log(n) + 2) * 2.0 ** -22 + (n * (Hq // H) + 8) * 2.0 ** -24)
        assert ((weight.double() - want).abs() <= far).all()
    if n > 1:
        k[1, 0, 2] = INF
        got, size = oil.prompt_attend(q, k, v, _int([0, n]), scale=0.0)
        assert torch.isnan(size[1:, :Hq // H]).all() and torch.equal(size[:, Hq // H:], lse[:, Hq // H:])
        weight = oil.prompt_weigh(q, k, lse, _int([0, n]), scale=0.0)
        assert torch.isnan(weight[0, 1]) and torch.isfinite(weight[0, 2:]).all() and torch.isfinite(weight[1:]).all()


@pytest.mark.parametrize("Hq,H,D", [(4, 2, 64), (2, 2, 128), (3, 1, 24)])
@pytest.mark.parametrize("at", [0, 3, 70, 200])
def test_values_that_are_not_finite_without_weight(oil, Hq, H, D, at):
    """Under a weight that is 0 in binary32 they count, under a score of -inf they do not; alike for a
    sequence alone, in tiles of 64 rows, and packed, in tiles of 128."""
    n, G = 300, Hq // H
    more = 128 * 256 // Hq + 1
    q, k, v = (_normal((n + more, h, D), i) for i, h in ((1, Hq), (2, H), (3, H)))
    q[..., 0], k[..., 0] = 32.0, 0.0
    v[at, 0, 5], v[at, 0, 6], v[at, 0, 7] = INF, -INF, math.nan
    for low in (-300.0, -INF):
        k[at, 0, 0] = low                              # below the others by some 9,600, or without a score
        alone = oil.prompt_attend(q[:n], k[:n], v[:n], _int([0, n]), scale=1.0)
        packed = oil.prompt_attend(q, k, v, _int([0, n, n + more]), scale=1.0)
        for a, b in zip(alone, packed):
            assert ((a == b[:n]) | (a.isnan() & b[:n].isnan())).all()
        out, lse = alone
        clean = oil.prompt_attend(q[:n], k[:n], torch.where(v[:n].isfinite(), v[:n], 0.0), _int([0, n]), scale=1.0)
        assert torch.equal(lse, clean[1])
        same = torch.ones_like(out, dtype=torch.bool)
        same[at:, :G, 5:8] = False
        assert torch.equal(out[same], clean[0][same])
        if low != -INF:
            assert (out[at:, :G, 5] == INF).all() and (out[at:, :G, 6] == -INF).all()
            assert torch.isnan(out[at:, :G, 7]).all()
        else:
            # made in another way, with weights rounded to bf16 and out rounded in both
            size = oil.prompt_attend(q[:n], k[:n], torch.where(v[:n].isfinite(), v[:n].abs(), 0.0), _int([0, n]),
                                     scale=1.0)[0].double() * (1 + 2.0 ** -6)
            off = (out.double() - clean[0].double()).abs()
            assert (off <= 2 * 2.0 ** -8 * (size + clean[0].double().abs()) * (1 + 2.0 ** -7)).all()
            if at == 0:                                # a row of this key alone
                assert (out[0, :G] == 0).all() and (lse[0, :G] == -INF).all()


@pytest.mark.parametrize("n,Hq,H,D", [(90, 2, 1, 64), (2100, 16, 16, 128)])
def test_rows_without_scores(oil, n, Hq, H, D):
    """Scores of -inf alone give zeros, whatever the values are."""
    q, k, v = (_normal((n, h, D), i) for i, h in ((1, Hq), (2, H), (3, H)))
    q[..., 1], k[..., 1] = 2.0, -INF
    v[::5], v[1::5], v[2::5] = INF, -INF, math.nan
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]))
    assert (out == 0).all() and (lse == -INF).all()


def _finite_and_near(out, want, far):
    assert torch.isfinite(out).all()
    off = (out.double() - want).abs()
    assert (off <= far).all(), (off / far).max().item()


@pytest.mark.parametrize("n,Hq,H,D", [(1, 1, 1, 8), (300, 4, 2, 24), (300, 2, 2, 128), (2100, 16, 16, 64), (1500, 32, 8, 128)])
def test_large_values(oil, n, Hq, H, D):
    """Values up to the largest of bf16: a mean of them is no larger, whatever their weighted sum is."""
    q, k = _normal((n, Hq, D), 1), _normal((n, H, D), 2)
    scale = 1 / math.sqrt(D)
    largest = torch.finfo(torch.bfloat16).max
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    signs = torch.randint(2, (n, H, D), generator=g, device="cuda") * 2.0 - 1
    # a few scores: the largest far from the first tile's, where weights are above 1
    wide = q * 3
    for v in (torch.full((n, H, D), largest), torch.full((n, H, D), -2.0 ** 127), signs * largest,
              _normal((n, H, D), 3).float() * 2.0 ** 122):
        v = v.to(device="cuda", dtype=torch.bfloat16)
        for asks in (q, wide, q * 0):
            out, lse = oil.prompt_attend(asks, k, v, _int([0, n]), scale=scale)
            w_out, w_lse, far_out, far_lse = ref.attend(asks, k, v, [0, n], scale)
            _finite_and_near(out, w_out, far_out)
            assert ((lse.double() - w_lse).abs() <= far_lse).all()
        if (v == v[:1]).all():  # equal weights of equal values
            assert (out == v[0].repeat_interleave(Hq // H, 0)).all()


@pytest.mark.parametrize("at", [70, 1000, 2000])
@pytest.mark.parametrize("D", [8, 128])
def test_large_values_of_a_later_key(oil, at, D):
    """A key nearly 8 powers of two above the first tile's weighs 200 times the others' ones."""
    n = 2100
    q = torch.zeros((n, 2, D), dtype=torch.bfloat16, device="cuda")
    k, v = torch.zeros_like(q), _normal((n, 2, D), 3)
    q[..., 0] = 1.0
    k[at, :, 0] = 5.25
    v[at] = 2.0 ** 121
    v[at, 1] = -2.0 ** 127
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=1.0)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [0, n], 1.0)
    _finite_and_near(out, w_out, far_out)
    assert ((lse.double() - w_lse).abs() <= far_lse).all()


@pytest.mark.parametrize("Hq,H,D", [(8, 2, 128), (12, 12, 64), (5, 1, 40)])
def test_results_made_again_depend_on_what_they_see(oil, Hq, H, D):
    """Rows whose scores or values leave the ordinary pass: alone and packed, as part of a longer sequence and
    beside rows that hold anything, bit by bit."""
    lens = [300, 1, 1900, 64]
    at = [0, 300, 301, 2201, 2265]
    q, k, v = (_normal((at[-1], h, D), i) for i, h in ((1, Hq), (2, H), (3, H)))
    q[::3, :, 0] = 2.0 ** 40
    k[::7, :, 0] = 2.0 ** 30
    v[..., 1] = 2.0 ** 127
    v[::5, :, 1] *= -1.0
    v[3::50, 0, 2] = INF
    q[1::3, 0] *= 2.0 ** -100
    same = lambda a, b: ((a == b) | (a.isnan() & b.isnan())).all()  # noqa: E731
    out, lse = oil.prompt_attend(q, k, v, _int(at))
    assert torch.isfinite(out[..., 1]).all() and torch.isfinite(out[..., 3:]).all()
    for a, z in zip(at, at[1:]):
        alone = oil.prompt_attend(q[a:z], k[a:z], v[a:z], _int([0, z - a]))
        assert same(alone[0], out[a:z]) and torch.equal(alone[1], lse[a:z])
        half = a + (z - a + 1) // 2
        begun = oil.prompt_attend(q[a:half], k[a:half], v[a:half], _int([0, half - a]))
        assert same(begun[0], out[a:half]) and torch.equal(begun[1], lse[a:half])
    wild = q.clone()
    wild[2::3] = math.nan
    got = oil.prompt_attend(wild, k, v, _int(at))
    kept = torch.arange(at[-1], device="cuda") % 3 != 2
    assert same(got[0][kept], out[kept]) and torch.equal(got[1][kept], lse[kept])
    assert torch.isnan(got[0][~kept]).all()


@pytest.mark.parametrize("n,Hq,H,D", SIZES)
@pytest.mark.parametrize("scale", [1.5 * 2.0 ** 127, -2.0 ** 127, 2.0 ** -126, 2.0 ** -140])
def test_scales_at_the_ends(oil, n, Hq, H, D, scale):
    """Scales up to binary32's largest and down to subnormal ones, with products that bring the scores back as
    far as binary32 holds them."""
    q, k, v = (_normal((n, h, D), i) for i, h in ((1, Hq), (2, H), (3, H)))
    # products by 2^(e - 1), half of it in each; 128 of up to 2^4.5 each add up to less than 2^(e + 11)
    e = min(-math.frexp(scale)[1], 117)
    q, k = q * 2.0 ** (e // 2), k * 2.0 ** (e - e // 2 - 1)
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=scale)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [0, n], scale)
    # a subnormal scale times log2 e is rounded by 2^-150 at most
    lost = 2.0 ** (e + 11 - 150) if abs(scale) < 2.0 ** -125 else 0.0
    assert ((out.double() - w_out).abs() <= far_out + 2 * lost * v.double().abs().max()).all()
    assert ((lse.double() - w_lse).abs() <= far_lse + lost).all()
    for last in (n, 17):
        weight = oil.prompt_weigh(q, k, lse, _int([0, n]), last=last, scale=scale)
        want, far = ref.weigh(q, k, lse, [0, n], last, scale)
        assert ((weight.double() - want).abs() <= far + 2 * lost * want).all()
