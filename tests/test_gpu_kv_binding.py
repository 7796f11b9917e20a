"""The 4-bit cache's binding: the workspaces it keeps, by stream and bounded, and
the ones it is given."""
import pytest
import torch

from tests.test_gpu_kv import oil  # noqa: F401

pytestmark = pytest.mark.gpu


def _filled(oil, n_slots=8, heads=2, dim=64, n=300):  # noqa: F811
    c = oil.KvCache(n_slots, heads, dim, n)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    c.append(*(torch.randn((n_slots, n, heads, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)))
    return c


def _nodes(B, N, heads=2, group=4, dim=64, seed=2):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn((B, N, h, dim), generator=g, device="cuda").to(torch.bfloat16)
            for h in (heads * group, heads, heads)]


def test_kept_workspaces_do_not_grow_with_the_sizes_seen(oil):  # noqa: F811
    c = _filled(oil)
    sizes = [(B, N) for B in range(1, 9) for N in (1, 2, 5, 17, 33, 61, 65, 100, 200, 256)]
    keeps = list(range(250, 10, -7))
    need = max([c.attend_workspace_bytes(B, N, 8) for B, N in sizes] + [c.evict_workspace_bytes(8, k) for k in keeps])
    given = {s: _nodes(*s) for s in sizes}
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for s in sizes:
        c.attend(*given[s])
    for k in keeps:
        c.evict(k)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 4 * need + (1 << 20)


def test_streams_have_workspaces_of_their_own(oil):  # noqa: F811
    c = _filled(oil)
    q, k, v = _nodes(8, 17)
    side = torch.cuda.Stream()
    want = [x.clone() for x in c.attend(q, k, v)]
    torch.cuda.synchronize()
    here = c._ws["attend", (8, 17, 8)].data_ptr()
    with torch.cuda.stream(side):
        got = c.attend(q, k, v)
        there = c._ws["attend", (8, 17, 8)].data_ptr()
    side.synchronize()
    assert here != there
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = c.attend(q, k, v, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_given_workspace(oil):  # noqa: F811
    c, d = _filled(oil), _filled(oil)
    q, k, v = _nodes(8, 33)
    want = c.attend(q, k, v)
    need = max(d.attend_workspace_bytes(8, 33, 8), d.evict_workspace_bytes(8, 100))
    ws = torch.full((need // 4 + 1,), float("nan"), device="cuda")
    got = d.attend(q, k, v, workspace=ws)
    c.evict(100, 7)
    d.evict(100, 7, workspace=ws)
    torch.cuda.synchronize()
    assert not d._ws
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(c.positions, d.positions) and torch.equal(c.weights, d.weights)
    with pytest.raises(oil.OilError):
        d.attend(q, k, v, workspace=ws[:64])
    with pytest.raises(oil.OilError):
        d.evict(50, workspace=ws[:64])
    for bad in (ws[::2], ws.cpu()):
        with pytest.raises(ValueError):
            d.attend(q, k, v, workspace=bad)


def test_graph_keeps_its_workspace(oil):  # noqa: F811
    """A captured call's workspace stays while larger calls on the same stream follow."""
    c = _filled(oil)
    q, k, v = _nodes(2, 5)
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    want = [x.clone() for x in c.attend(q, k, v, slots=slots)]
    out = [torch.empty_like(x) for x in want]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c.attend(q, k, v, slots=slots, out=out)
    with torch.cuda.stream(side):
        for N in (17, 65, 256):
            c.attend(*_nodes(8, N))
    torch.cuda.synchronize()
    others = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
    for _ in range(3):
        for x in out:
            x.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(torch.isnan(x).all() for x in others)


def _stream_of(x):
    """The stream whose memory of torch's allocator x lies in."""
    at = x.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def test_memory_of_the_stream_given(oil):  # noqa: F811
    """With a stream given, what a call makes is allocated for that stream: what is free on the
    current one may still be in use there."""
    side = torch.cuda.Stream()
    c = _filled(oil)
    q, k, v = _nodes(8, 17)
    torch.cuda.synchronize()
    made = [*c.attend(q, k, v, stream=side), *c.read(3, 70, stream=side)]
    c.evict(90, stream=side)
    with torch.cuda.stream(side):
        made += list(c._ws.values())
    assert len(made) == 6
    d = oil.KvCache(3, 2, 64, 40, stream=side)
    made += [d.codes, d.positions, d.weights, d.state]
    side.synchronize()
    assert [_stream_of(x) for x in made] == [side.cuda_stream] * len(made)
    assert _stream_of(c.attend(q, k, v)[0]) == 0
    torch.cuda.synchronize()
