"""Packed appends of starts that do not ascend, that lie past the rows, and of many requests."""
import pytest
import torch

pytestmark = pytest.mark.gpu

H, D = 2, 64


@pytest.fixture(scope="module")
def oil():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_03839_amd as m
    m.lib()
    return m


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rows(T, seed=3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (torch.randn((T, H, D), generator=g, device="cuda") for _ in range(2))
    return k, v, torch.rand((H, T), generator=g, device="cuda")


def _same(a, b, cap):
    assert torch.equal(a.state[:, :2], b.state[:, :2])
    assert torch.equal(a.positions, b.positions) and torch.equal(a.weights, b.weights)
    for x, y in zip(a.read(0, cap), b.read(0, cap)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("before", [0, 17, 96])
@pytest.mark.parametrize("starts", [
    [0, 1000, 0, 1000],
    [1000, 0, 1000, 0],
    [0, 990, 40, 1000],
    [500, 1000, 200, 700],
    [900, 1000, 0, 1000],
    [0, 33, 20, 90],
    [0, 600, 2 ** 31 - 1, -2 ** 31],
    [10, 5, 20, 30],
    [64, 64, 0, 1000],
])
def test_starts_that_do_not_ascend(oil, starts, before):
    """Every sequence's rows, or none and nothing changed: a slot never counts rows that were not written."""
    B, T, cap = len(starts) - 1, 1000, 2400
    k, v, weight = _rows(T)
    got, every, none = (oil.KvCache(B, H, D, cap) for _ in range(3))
    if before:
        x, y = (z.unflatten(0, (B, before)) for z in _rows(B * before, 4)[:2])
        for c in (got, every, none):
            c.append(x, y)
    lens = got.state[:, 0].tolist()
    got.append(k, v, starts=_int(starts), weight=weight)
    at = [min(max(s, 0), T) for s in starts]
    for b in range(B):
        a, z = at[b], max(at[b], at[b + 1])
        if z > a:
            every.append(k[None, a:z].contiguous(), v[None, a:z].contiguous(), slots=_int([b]),
                         weight=weight[None, :, a:z].contiguous())
    torch.cuda.synchronize()
    _same(got, none if got.state[:, 0].tolist() == lens else every, cap)
    # and what comes after is what it would have been
    tail = none if got.state[:, 0].tolist() == lens else every
    for c in (got, tail):
        c.append(k, v, starts=_int([0, 100, 100, 300]), weight=weight)
    torch.cuda.synchronize()
    _same(got, tail, cap)


def test_more_requests_than_a_workgroup_has_threads(oil):
    lens = [(7 * i) % 45 for i in range(700)]
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    k, v, weight = _rows(at[-1])
    a, b = (oil.KvCache(len(lens), H, D, 64) for _ in range(2))
    a.append(k, v, starts=_int(at), weight=weight)
    pad = max(lens)
    x, y = (torch.zeros((len(lens), pad, H, D), device="cuda") for _ in range(2))
    w = torch.zeros((len(lens), H, pad), device="cuda")
    for i, n in enumerate(lens):
        x[i, :n], y[i, :n], w[i, :, :n] = k[at[i]:at[i + 1]], v[at[i]:at[i + 1]], weight[:, at[i]:at[i + 1]]
    b.append(x, y, count=_int(lens), weight=w)
    torch.cuda.synchronize()
    assert a.state[:, 0].tolist() == lens
    _same(a, b, 64)
    swapped = list(at)
    swapped[300], swapped[301] = at[-1], 0
    a.append(k, v, starts=_int(swapped), weight=weight)
    torch.cuda.synchronize()
    _same(a, b, 64)
