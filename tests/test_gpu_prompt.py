"""Attention of packed prompts and the weight it leaves, against 64 bits; what rows do not
see; strides, streams, graphs; the packed append against the padded one."""
import math

import pytest
import torch

from tests import _prompt_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oil():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_03839_amd as m
    m.lib()
    return m


def _starts(lens, before=0):
    at = [before]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _rows(T, Hq, H, D, seed=1, pad=0, k_size=1.0):
    """q, k, v as slices of one buffer whose other columns are NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.full((T, (Hq + 2 * H) * D + pad), math.nan, dtype=torch.bfloat16, device="cuda")
    y = torch.randn((T, Hq + 2 * H, D), generator=g, device="cuda")
    y[:, Hq:Hq + H] *= k_size
    x[:, :(Hq + 2 * H) * D] = y.reshape(T, -1)
    cut = lambda a, n: x[:, a * D:(a + n) * D].unflatten(1, (n, D))  # noqa: E731
    return cut(0, Hq), cut(Hq, H), cut(Hq + H, H)


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _near(got, want, far, name):
    assert not torch.isnan(got).any(), name
    off = (got.double() - want).abs()
    assert (off <= far).all(), (name, (off / far).max().item())


SHAPES = [
    ([1], 1, 1, 8),
    ([2, 1, 0, 5], 4, 2, 64),
    ([0, 0, 33], 3, 3, 16),
    ([63, 64, 65, 1, 0, 130], 8, 2, 128),
    ([257], 10, 2, 40),
    ([300, 5], 7, 1, 96),
    ([31, 200], 64, 1, 64),                   # the largest group
    ([129, 64, 500], 12, 12, 128),
    ([2049, 700, 1, 0, 1500], 32, 4, 128),    # tiles of 256 rows
    ([4200], 32, 8, 72),
    ([1, 2, 3] * 100 + [700], 16, 4, 64),     # many short sequences
]


@pytest.mark.parametrize("lens,Hq,H,D", SHAPES)
def test_attend_and_weigh(oil, lens, Hq, H, D):
    starts = _starts(lens)
    q, k, v = _rows(starts[-1], Hq, H, D, pad=8)
    scale = 1.3 / math.sqrt(D)
    out, lse = oil.prompt_attend(q, k, v, _int(starts), scale=scale)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, starts, scale)
    _near(out, w_out, far_out, "out")
    _near(lse, w_lse, far_lse, "lse")
    for last in (None, 1, 17, 64):
        got = oil.prompt_weigh(q, k, lse, _int(starts), last=last, scale=scale)
        want, far = ref.weigh(q, k, lse, starts, starts[-1] if last is None else last, scale)
        _near(got, want, far, f"weight, last {last}")


def test_rows_outside_stay(oil):
    starts, T = [3, 40, 40, 101], 120
    q, k, v = _rows(T, 8, 2, 64)
    for x in (q, k, v):
        x[:3] = math.nan
        x[101:] = math.inf
    out = torch.full((T, 8, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, 8), 6.0, device="cuda")
    oil.prompt_attend(q, k, v, _int(starts), out=(out, lse))
    weight = torch.full((2, T), 7.0, device="cuda")
    oil.prompt_weigh(q, k, lse, _int(starts), last=9, out=weight)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, starts, 1 / 8)
    s = slice(3, 101)
    _near(out[s], w_out[s], far_out[s], "out")
    _near(lse[s], w_lse[s], far_lse[s], "lse")
    want, far = ref.weigh(q, k, lse, starts, 9, 1 / 8)
    _near(weight[:, s], want[:, s], far[:, s], "weight")
    for r in (slice(0, 3), slice(101, T)):
        assert (out[r] == 5).all() and (lse[r] == 6).all() and (weight[:, r] == 7).all()
    # starts past the rows count as their bound: the same as up to 120 rows, all of which are read then
    for x in (q, k, v):
        x[101:] = 1.0
    a = oil.prompt_attend(q, k, v, _int([3, 40, 40, 120]))
    b = oil.prompt_attend(q, k, v, _int([3, 40, 40, 2 ** 31 - 1]))
    assert torch.equal(a[0][3:], b[0][3:]) and torch.equal(a[1][3:], b[1][3:])


@pytest.mark.parametrize("n,Hq,H,D", [(200, 8, 2, 128), (150, 2, 2, 64), (4200, 32, 8, 128)])
def test_unseen_rows_do_not_reach(oil, n, Hq, H, D):
    """Values and keys that are not finite reach the rows that see them, and no other."""
    q, k, v = _rows(n, Hq, H, D)
    starts = _int([0, n])
    clean_out, clean_lse = oil.prompt_attend(q, k, v, starts)
    at, odd = n - 37, [math.nan, math.inf, -math.inf]
    for i, x in enumerate(odd):
        vv = v.clone()
        vv[at, 0, 3 + i] = x
        vv[at + 20, 0, 3 + i] = math.inf
        out, lse = oil.prompt_attend(q, k.clone(), vv, starts)
        assert torch.equal(lse, clean_lse)
        same = torch.ones_like(out, dtype=torch.bool)
        same[at:, :Hq // H, 3 + i] = False
        assert torch.equal(out[same], clean_out[same])
        seen = out[at:at + 20, :Hq // H, 3 + i].float()
        assert (torch.isnan(seen) if i == 0 else seen == x).all()
        late = out[at + 20:, :Hq // H, 3 + i].float()
        assert (late == math.inf if i == 1 else torch.isnan(late)).all()
    kk = k.clone()
    kk[at, 0] = math.nan
    out, lse = oil.prompt_attend(q, kk, v.clone(), starts)
    assert torch.equal(out[:at], clean_out[:at]) and torch.equal(lse[:at], clean_lse[:at])
    assert torch.isnan(out[at:, :Hq // H].float()).all() and torch.isnan(lse[at:, :Hq // H]).all()
    if H > 1:
        assert torch.equal(out[:, Hq // H:], clean_out[:, Hq // H:])
    clean = oil.prompt_weigh(q, k, clean_lse, starts, last=50)
    weight = oil.prompt_weigh(q, kk, clean_lse, starts, last=50)
    assert torch.isnan(weight[0, at])
    weight[0, at] = clean[0, at]
    assert torch.equal(weight, clean)
    qq = q.clone()
    qq[at, 0] = math.nan
    weight = oil.prompt_weigh(qq, k.clone(), clean_lse, starts, last=50)
    assert torch.isnan(weight[0, :at + 1]).all() and torch.equal(weight[0, at + 1:], clean[0, at + 1:])
    gone = clean_lse.clone()
    gone[at, 0] = -math.inf          # a row that counts nowhere, whatever it holds
    weight = oil.prompt_weigh(qq, k.clone(), gone, starts, last=50)
    want, far = ref.weigh(torch.where(qq.isnan(), 0, qq), k, gone, [0, n], 50, 1 / math.sqrt(D))
    _near(weight, want, far, "weight")


def test_next_columns_do_not_reach(oil):
    """head_dim below the padded width beside columns that are NaN."""
    q, k, v = _rows(90, 2, 1, 24, pad=104)
    out, lse = oil.prompt_attend(q, k, v, _int([0, 90]))
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [0, 90], 1 / math.sqrt(24))
    _near(out, w_out, far_out, "out")
    _near(lse, w_lse, far_lse, "lse")


@pytest.mark.parametrize("scale", [-0.2, 0.0, 4.0])
def test_scales(oil, scale):
    starts = [0, 100, 230]
    q, k, v = _rows(230, 4, 2, 64)
    out, lse = oil.prompt_attend(q, k, v, _int(starts), scale=scale)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, starts, scale)
    _near(out, w_out, far_out, "out")
    _near(lse, w_lse, far_lse, "lse")
    got = oil.prompt_weigh(q, k, lse, _int(starts), scale=scale)
    want, far = ref.weigh(q, k, lse, starts, 230, scale)
    _near(got, want, far, "weight")


def test_rising_scores(oil):
    """Scores that rise from key to key and jump between tiles: the running maximum is moved again
    and again.  Whole numbers, so that every score is exact."""
    n, D = 700, 64
    q = torch.zeros((n, 2, D), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((n, 1, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 1.0, 64.0
    at = torch.arange(n, device="cuda")
    k[:, 0, 0], k[:, 0, 1] = (at % 64).to(torch.bfloat16), (at // 64).to(torch.bfloat16)
    v = _rows(n, 1, 1, D, seed=4)[2].contiguous()
    for scale in (1.0, 0.03125, -0.25):
        out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=scale)
        w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [0, n], scale)
        _near(out, w_out, far_out, "out")
        _near(lse, w_lse, far_lse, "lse")


def test_rows_without_weight(oil):
    """Scores of -inf alone give zeros and -inf; beside others they weigh nothing."""
    q, k, v = _rows(70, 2, 1, 64)
    q[..., 5] = 1.0
    k[:10, 0, 5] = -math.inf
    out, lse = oil.prompt_attend(q, k, v, _int([0, 70]))
    assert (out[:10] == 0).all() and (lse[:10] == -math.inf).all()
    w_out, w_lse, far_out, far_lse = (x[10:] for x in ref.attend(
        q, torch.where(k.isinf(), -1e4, k), v, [0, 70], 1 / 8))
    _near(out[10:], w_out, far_out, "out")
    _near(lse[10:], w_lse, far_lse, "lse")
    weight = oil.prompt_weigh(q, k, lse, _int([0, 70]))
    assert (weight[0, :10] == 0).all() and torch.isfinite(weight).all()


def test_streams_graphs_and_calls_at_once(oil):
    lens = [64, 129, 1, 300]
    starts, T = _int(_starts(lens)), sum(lens)
    q, k, v = _rows(T, 8, 2, 128)
    want = oil.prompt_attend(q, k, v, starts)
    weight = oil.prompt_weigh(q, k, want[1], starts, last=20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = oil.prompt_attend(q, k, v, starts, stream=side)
    again = oil.prompt_attend(q, k, v, starts)
    side.synchronize()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = oil.prompt_attend(q, k, v, starts)
        w = oil.prompt_weigh(q, k, lse, starts, last=20)
    for turn in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(w, weight)
        out.fill_(1)
        w.fill_(1)
    # other lengths in the same buffers: the graph reads them on the device
    new = _int([0, 0, 400, 401, T])
    starts.copy_(new)
    graph.replay()
    torch.cuda.synchronize()
    eager = oil.prompt_attend(q, k, v, new)
    assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    assert torch.equal(w, oil.prompt_weigh(q, k, eager[1], new, last=20))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,lens", [(64, [1, 0, 33, 64, 200]), (128, [70, 31, 5, 0, 1])])
def test_packed_append_is_the_padded_one(oil, dtype, D, lens):
    B, H, cap = len(lens), 2, 230
    starts = _starts(lens, 4)
    T = starts[-1] + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    k, v = (torch.randn((T, H, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    weight = torch.rand((H, T), generator=g, device="cuda")
    slots = _int([4, 2, 0, 1, 3])
    a, b = (oil.KvCache(B, H, D, cap) for _ in range(2))
    for before in (17, 40):  # two appends: from an odd length on, the second past some slots' capacity
        x, y = (torch.randn((B, before, H, D), generator=g, device="cuda").to(dtype) for _ in range(2))
        for c in (a, b):
            c.append(x, y, slots=slots)
        a.append(k, v, starts=_int(starts), weight=weight, slots=slots)
        for i, (s, e) in enumerate(ref.spans(starts)):
            if e > s:
                b.append(k[None, s:e].contiguous(), v[None, s:e].contiguous(), slots=slots[i:i + 1],
                         weight=weight[None, :, s:e].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(a.state[:, :2], b.state[:, :2])
        assert torch.equal(a.positions, b.positions) and torch.equal(a.weights, b.weights)
        for p, r in zip(a.read(0, cap), b.read(0, cap)):
            assert torch.equal(p, r)


def test_prompt_to_answer(oil):
    """The calls as a server makes them: prompts attend, their rows' weights are counted, both enter
    the cache, the lightest rows leave, trees attend, logits become predictions and are accepted."""
    lens, Hq, H, D, V = [150, 7, 260], 8, 2, 64, 1000
    starts, T, B, N = _int(_starts(lens)), sum(lens), 3, 9
    q, k, v = _rows(T, Hq, H, D)
    out, lse = oil.prompt_attend(q, k, v, starts)
    weight = oil.prompt_weigh(q, k, lse, starts, last=32)
    cache = oil.KvCache(B, H, D, 300)
    cache.append(k, v, starts=starts, weight=weight)
    assert cache.lengths.tolist() == lens
    at = _starts(lens)
    for b, n in enumerate(lens):
        assert torch.equal(cache.weights[b, :, :n], weight[:, at[b]:at[b] + n])
    # the last token's row again, as a node over the rows before it: off by what 4 bits lose alone
    held = oil.KvCache(B, H, D, 300)
    held.append(k, v, starts=_int([a for a in at]))
    kept, _ = held.read(0, 300, dtype=torch.float32)
    for b, n in enumerate(lens):
        step = (k[at[b]:at[b] + n].float().amax(-1) - k[at[b]:at[b] + n].float().amin(-1)) / 15
        off = (kept[b, :, :n].transpose(0, 1) - k[at[b]:at[b] + n].float()).abs().amax(-1)
        assert (off <= step * 0.5 * (1 + 2.0 ** -6) + 0.02).all()
    cache.evict(100, 16)
    assert cache.lengths.tolist() == [100, 7, 100]
    heavy = weight[:, at[0]:at[0] + 134].topk(84, dim=1)  # beside the last 16
    for h in range(H):
        assert torch.isin(heavy.indices[h], cache.positions[0, h, :100].long()).all()
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 3, 4]] * B, dtype=torch.int32, device="cuda")
    token = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
    count = _int([9, 9, 4])
    mask = oil.tree_mask(parent, count)
    nq, nk, nv = (x.unflatten(0, (B, N)) for x in _rows(B * N, Hq, H, D, seed=9))
    o, _ = cache.attend(nq, nk, nv, n_nodes=count, mask=mask)
    assert torch.isfinite(o.float()).all()
    logits = torch.zeros((B, N, V), device="cuda")
    follow = [1, 3, 500, 6, 500, 500, 600, 500, 500]      # 0 -> 1 -> 3 -> 6, then 600
    logits[:, torch.arange(N), follow] = 9.0
    logprob, entropy, best, best_logprob = oil.token_logprobs(logits, token[..., None], top=1, n_rows=count)
    assert best[0, :, 0].tolist() == follow and best[2, :, 0].tolist() == follow[:4] + [-1] * 5
    length, nodes, bonus = oil.accept_walk(token, parent, count, best[..., 0].contiguous())
    assert length.tolist() == [3, 3, 2] and bonus.tolist() == [600, 600, 6]
    cache.append(nk, nv, nodes=nodes, count=length)
    assert cache.lengths.tolist() == [104, 11, 103]


def test_refusals(oil):
    q, k, v = _rows(20, 4, 2, 64)
    starts = _int([0, 20])
    _, lse = oil.prompt_attend(q, k, v, starts)
    for bad in (lambda: oil.prompt_attend(q.float(), k, v, starts), lambda: oil.prompt_attend(q, k[:19], v[:19], starts),
                lambda: oil.prompt_attend(q, k, v[..., :32], starts), lambda: oil.prompt_attend(q, k, v, starts.long()),
                lambda: oil.prompt_attend(q.cpu(), k, v, starts), lambda: oil.prompt_attend(q, k.cpu(), v.cpu(), starts),
                lambda: oil.prompt_attend(q, k, v, starts.cpu()), lambda: oil.prompt_attend(q.transpose(1, 2), k, v, starts),
                lambda: oil.prompt_attend(q, k, v, starts, out=(torch.empty_like(q).float(), lse)),
                lambda: oil.prompt_weigh(q, k, lse[:, :3], starts), lambda: oil.prompt_weigh(q, k, lse.double(), starts)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: oil.prompt_attend(q[:, :3], k, v, starts),       # heads that do not divide
                lambda: oil.prompt_attend(q, k, v, starts, scale=math.inf),
                lambda: oil.prompt_weigh(q, k, lse, starts, last=0)):
        with pytest.raises(oil.OilError):
            bad()
    c = oil.KvCache(2, 2, 64, 40)
    for bad in (lambda: c.append(k, v, starts=starts, count=_int([1])), lambda: c.append(k, v[:19], starts=starts),
                lambda: c.append(k, v, starts=starts, weight=torch.zeros((20, 2), device="cuda")),
                lambda: c.append(k, v, starts=starts, slots=_int([0, 1]))):
        with pytest.raises(ValueError):
            bad()
