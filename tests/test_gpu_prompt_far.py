"""Packed prompts whose rows lie far apart or far from the start, many sequences and chunks,
workspaces given and shared, and calls captured side by side."""
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


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(shape, seed=5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)


def _cut(x, Hq, H, D):
    return [x[:, a * D:(a + n) * D].unflatten(1, (n, D)) for a, n in ((0, Hq), (Hq, H), (Hq + H, H))]


def _near(got, want, far, name):
    assert not torch.isnan(got).any(), name
    off = (got.double() - want).abs()
    assert (off <= far).all(), (name, (off / far).max().item())


def test_many_rows(oil):
    """512 sequences whose outputs and inputs pass 2^32 bytes; the last ones against 64 bits."""
    Hq, H, D = 32, 8, 128
    lens = [2049 + (i % 3) for i in range(509)] + [1, 0, 700]
    at = _starts(lens)
    x = _normal((at[-1], (Hq + 2 * H) * D))
    assert x.numel() * 2 > 1 << 33 and at[-1] * Hq * D * 2 > 1 << 32
    q, k, v = _cut(x, Hq, H, D)
    starts, scale = _int(at), 1 / math.sqrt(D)
    out, lse = oil.prompt_attend(q, k, v, starts)
    weight = oil.prompt_weigh(q, k, lse, starts, last=40)
    for first, past in ((0, 1), (508, 512)):
        a, z = at[first], at[past]
        here = [s - a for s in at[first:past + 1]]
        w_out, w_lse, far_out, far_lse = ref.attend(q[a:z], k[a:z], v[a:z], here, scale)
        _near(out[a:z], w_out, far_out, "out")
        _near(lse[a:z], w_lse, far_lse, "lse")
        want, far = ref.weigh(q[a:z], k[a:z], lse[a:z], here, 40, scale)
        _near(weight[:, a:z], want, far, "weight")


@pytest.mark.parametrize("T,Hq,H,D,ld", [(40000, 2, 1, 64, 1 << 16),   # a sequence's keys pass 2^32 bytes
                                         (130, 1, 1, 56, 1 << 24),     # a tile's rows do
                                         (150, 3, 3, 120, 1 << 23)])
def test_rows_far_apart(oil, T, Hq, H, D, ld):
    """The same as of dense copies, bit by bit; what lies between the rows is NaN."""
    x = torch.full((T, ld), math.nan, dtype=torch.bfloat16, device="cuda")
    columns = (Hq + 2 * H) * D
    x[:, :columns] = _normal((T, columns))
    q, k, v = _cut(x, Hq, H, D)
    starts = _int([0, T])
    out, lse = oil.prompt_attend(q, k, v, starts)
    dense = [t.contiguous() for t in (q, k, v)]
    want = oil.prompt_attend(*dense, starts)
    assert torch.isfinite(out).all() and torch.equal(out, want[0]) and torch.equal(lse, want[1])
    for last in (1, 70, None):
        weight = oil.prompt_weigh(q, k, lse, starts, last=last)
        assert torch.isfinite(weight).all()
        assert torch.equal(weight, oil.prompt_weigh(dense[0], dense[1], lse, starts, last=last))


@pytest.mark.parametrize("lens,Hq,H,D", [([4200, 1, 900, 0, 3000], 16, 2, 128), ([600] * 12 + [1] * 20, 2, 2, 32)])
def test_weights_in_chunks(oil, lens, Hq, H, D):
    """Every row counts: sequences of many chunks, few and none beside each other."""
    at = _starts(lens)
    q, k, v = _cut(_normal((at[-1], (Hq + 2 * H) * D)), Hq, H, D)
    scale = 1 / math.sqrt(D)
    _, lse = oil.prompt_attend(q, k, v, _int(at))
    for last in (None, 333):
        weight = oil.prompt_weigh(q, k, lse, _int(at), last=last)
        want, far = ref.weigh(q, k, lse, at, at[-1] if last is None else last, scale)
        _near(weight, want, far, "weight")
        assert torch.equal(weight, oil.prompt_weigh(q, k, lse, _int(at), last=last))


def test_workspaces(oil):
    """One workspace for calls on one stream, as large as they ask for; a smaller one is refused."""
    lens, Hq, H, D = [500, 3, 0, 1200], 8, 2, 64
    at = _starts(lens)
    T, B, starts = at[-1], len(lens), _int(at)
    q, k, v = _cut(_normal((T, (Hq + 2 * H) * D)), Hq, H, D)
    want = oil.prompt_attend(q, k, v, starts)
    weight = oil.prompt_weigh(q, k, want[1], starts)
    need = oil.lib().oil_prompt_attend_workspace_bytes(B, T, Hq, H)
    more = oil.lib().oil_prompt_weigh_workspace_bytes(B, T, Hq, H, T)
    room = torch.full((max(need, more),), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        out, lse = oil.prompt_attend(q, k, v, starts, workspace=room)
        got = oil.prompt_weigh(q, k, lse, starts, workspace=room)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(got, weight)
    for bad in (lambda: oil.prompt_attend(q, k, v, starts, workspace=room[:need - 1]),
                lambda: oil.prompt_weigh(q, k, lse, starts, workspace=room[:more - 1]),
                lambda: oil.prompt_attend(q, k, v, starts, workspace=room[1:])):
        with pytest.raises(oil.OilError):
            bad()
    # without lse
    out = torch.empty_like(want[0])
    status = oil.lib().oil_prompt_attend(starts.data_ptr(), B, T, q.data_ptr(), q.stride(0), Hq, k.data_ptr(), v.data_ptr(),
                                         k.stride(0), H, D, 1 / math.sqrt(D), room.data_ptr(), room.numel(),
                                         out.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
    assert status == 0 and torch.equal(out, want[0])


def test_graphs_side_by_side(oil):
    """Two captured prompts, each with its packed append, replayed on two streams at once."""
    Hq, H, D, cap = 8, 2, 64, 4000
    made = []
    for seed, lens in ((1, [700, 1, 90]), (2, [64, 800, 0])):
        at = _starts(lens)
        q, k, v = _cut(_normal((at[-1], (Hq + 2 * H) * D), seed), Hq, H, D)
        starts, cache, side = _int(at), oil.KvCache(3, H, D, cap), torch.cuda.Stream()
        want = oil.prompt_attend(q, k, v, starts)
        weight = oil.prompt_weigh(q, k, want[1], starts, last=33)
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = oil.prompt_attend(q, k, v, starts)
            w = oil.prompt_weigh(q, k, lse, starts, last=33)
            cache.append(k, v, starts=starts, weight=w)
        made.append((graph, side, out, lse, w, want, weight, cache, lens, k, v, starts))
    for turn in range(4):
        for graph, side, *_ in made:
            with torch.cuda.stream(side):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, out, lse, w, want, weight, cache, lens, *_ in made:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(w, weight)
            assert cache.lengths.tolist() == [n * (turn + 1) for n in lens]
            out.fill_(3)
            w.fill_(3)
        torch.cuda.synchronize()
    for _, _, _, _, _, _, weight, cache, lens, k, v, starts in made:
        plain = oil.KvCache(3, H, D, cap)
        for _ in range(4):
            plain.append(k, v, starts=starts, weight=weight)
        assert torch.equal(cache.weights, plain.weights) and torch.equal(cache.positions, plain.positions)
        for a, b in zip(cache.read(0, cap), plain.read(0, cap)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("low", [-math.inf, -40.0])
@pytest.mark.parametrize("n", [500, 5000])
def test_first_keys_without_weight(oil, low, n):
    """The first 70 keys' scores are -inf, or so low that their weights are 0 beside the others':
    rows from 70 on are those of the sequence that begins there."""
    Hq, H, D, a = 8, 2, 64, 70
    q, k, v = (t.clone() for t in _cut(_normal((n, (Hq + 2 * H) * D)), Hq, H, D))
    q[..., 0] = 8.0                                  # 8 times the key's, beside which the others add 45 at most
    k[..., 0] = 0.0
    k[:a, :, 0] = low
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=1.0)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [a, n], 1.0)
    _near(out[a:], w_out[a:], far_out[a:], "out")
    _near(lse[a:], w_lse[a:], far_lse[a:], "lse")
    if low == -math.inf:
        assert (out[:a] == 0).all() and (lse[:a] == -math.inf).all()


@pytest.mark.parametrize("n", [500, 5000])
def test_first_keys_with_all_weight(oil, n):
    """The first keys' scores lie over 200 above the others', whose weights then are 0."""
    Hq, H, D, a = 8, 2, 64, 70
    q, k, v = (t.clone() for t in _cut(_normal((n, (Hq + 2 * H) * D)), Hq, H, D))
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[:a, :, 0] = 40.0
    out, lse = oil.prompt_attend(q, k, v, _int([0, n]), scale=1.0)
    w_out, w_lse, far_out, far_lse = ref.attend(q, k, v, [0, n], 1.0)
    _near(out, w_out, far_out, "out")
    _near(lse, w_lse, far_lse, "lse")


@pytest.mark.parametrize("Hq,H,D", [(8, 2, 128), (12, 12, 64), (5, 1, 40), (16, 4, 128)])
def test_rows_depend_on_what_they_see(oil, Hq, H, D):
    """A row's bits are the same whatever other rows ask for, and whatever its sequence is packed with."""
    lens = [300, 1, 1900, 64]
    at = _starts(lens)
    q, k, v = _cut(_normal((at[-1], (Hq + 2 * H) * D)), Hq, H, D)
    out, lse = oil.prompt_attend(q, k, v, _int(at))
    for a, z in zip(at, at[1:]):
        alone = oil.prompt_attend(q[a:z], k[a:z], v[a:z], _int([0, z - a]))
        assert torch.equal(alone[0], out[a:z]) and torch.equal(alone[1], lse[a:z])
    wild = q.clone()
    wild[::3] *= 40.0                                  # scores that leave their first tile's far behind
    wild[1::3, :, 0] = math.nan
    kept = torch.arange(at[-1], device="cuda") % 3 == 2
    got = oil.prompt_attend(wild, k.clone(), v.clone(), _int(at))
    assert torch.equal(got[0][kept], out[kept]) and torch.equal(got[1][kept], lse[kept])
    assert torch.isnan(got[0][1::3]).all() and torch.isfinite(got[0][::3]).all()
