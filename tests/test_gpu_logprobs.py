"""Log probabilities, entropies and most likely tokens against 64 bits: vocabularies and
strides that 16 bytes do not divide, ties, masked tokens, rows without any, NaN."""
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


def _logits(B, N, V, dtype, seed=1, pad=0, spread=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.full((B, N, V + pad), math.nan, dtype=dtype, device="cuda")[..., :V]
    x.copy_(spread * torch.randn((B, N, V), generator=g, device="cuda"))
    return x, torch.randint(V, (B, N, 3), generator=g, device="cuda", dtype=torch.int32)


def _check(oil, x, tokens, top, n_rows=None):
    B, N, V = x.shape
    counts = [N] * B if n_rows is None else [max(0, min(N, n)) for n in n_rows]
    given = None if n_rows is None else torch.tensor(n_rows, dtype=torch.int32, device="cuda")
    logprob, entropy, ids, best = oil.token_logprobs(x, tokens, top=top, n_rows=given)
    for b, m in enumerate(counts):
        assert (logprob[b, m:] == -math.inf).all() and (entropy[b, m:] == 0).all()
        assert (ids[b, m:] == -1).all() and (best[b, m:] == -math.inf).all()
        if m == 0:
            continue
        y, want, order, far, far_entropy = ref.logprobs(x[b, :m], tokens[b, :m], top)
        assert torch.equal(ids[b, :m].long(), order)
        t = tokens[b, :m].long()
        inside = (t >= 0) & (t < V)
        w = torch.where(inside, y.gather(1, t.clamp(0, V - 1)), -math.inf)
        for got, w in ((logprob[b, :m], w), (best[b, :m], torch.where(order >= 0, y.gather(1, order.clamp(min=0)),
                                                                    -math.inf))):
            none = w == -math.inf
            assert torch.equal(none, got == -math.inf)
            off = (got.double() - w).abs()[~none]
            assert (off <= (far[:, None] + w.abs() * 2.0 ** -22)[~none]).all(), off.max()
        off = (entropy[b, :m].double() - want).abs()
        assert (off <= far_entropy).all(), (off / far_entropy).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,N,V,top,pad", [
    (1, 1, 1, 1, 0), (1, 1, 5, 8, 0), (2, 3, 63, 64, 1), (1, 2, 1000, 5, 3), (1, 1, 32003, 8, 0), (3, 7, 4099, 20, 5),
    (1, 61, 131072, 1, 0), (2, 5, 131073, 64, 7), (2, 1500, 1029, 2, 0), (1, 1, 262147, 64, 1), (4, 700, 333, 0, 0),
    (3, 40, 2050, 16, 0), (3, 300, 700, 17, 0), (2, 9, 5000, 33, 1), (2, 300, 900, 64, 0), (1, 5, 90000, 63, 3)])
def test_rows(oil, dtype, B, N, V, top, pad):
    x, tokens = _logits(B, N, V, dtype, pad=pad)
    tokens[0, 0, 0], tokens[-1, -1, 1] = -1, V
    _check(oil, x, tokens, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [3, 900])
def test_counts(oil, dtype, N):
    x, tokens = _logits(5, N, 999, dtype)
    for b, m in enumerate((N, 0, 1, N - 1, -4)):
        x[b, max(m, 0):] = math.nan          # not read
    _check(oil, x, tokens, 4, n_rows=[N + 7, 0, 1, N - 1, -4])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,N,V", [(1, 2, 20011), (2, 1100, 2050)])
def test_orders(oil, dtype, B, N, V):
    """Rows whose order is hard: all alike, rising, falling, few values, zeros of both signs."""
    at = torch.arange(V, device="cuda", dtype=torch.float32)
    _, tokens = _logits(B, N, V, dtype)
    for row in (torch.zeros(V, device="cuda"), at / 64, -at / 64, at % 3, (at % 2) * -0.0,
                torch.where(at % 7 == 3, -math.inf, at % 5)):
        x = row.to(dtype).expand(B, N, V).contiguous()
        if N > 100:
            x, t = x[:, ::100].contiguous(), tokens[:, ::100].contiguous()
            _check(oil, x, t, 64)
        x = row.to(dtype).expand(B, N, V).contiguous()
        got = oil.token_logprobs(x, top=64)[2]
        want = ref.logprobs(x[0, :1], None, 64)[2]
        assert (got.long() == want).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 50021])
def test_masked(oil, dtype, V):
    x, tokens = _logits(2, 3, V, dtype)
    x[0, 0] = -math.inf                       # nothing may follow
    x[0, 1, 3:] = -math.inf                   # three tokens may
    x[0, 2, :V - 1] = -math.inf               # one
    x[1, 0, ::2] = -math.inf
    x[1, 1, 17] = 1e30                        # certain
    x[1, 2] *= 1e30                           # far apart
    logprob, entropy, ids, best = oil.token_logprobs(x, tokens, top=5)
    assert (logprob[0, 0] == -math.inf).all() and entropy[0, 0] == 0
    assert (ids[0, 0] == -1).all() and (best[0, 0] == -math.inf).all()
    assert (ids[0, 1, 3:] == -1).all() and sorted(ids[0, 1, :3].tolist()) == [0, 1, 2]
    assert ids[0, 2].tolist() == [V - 1, -1, -1, -1, -1] and best[0, 2, 0] == 0 and entropy[0, 2] == 0
    assert ids[1, 1, 0] == 17 and best[1, 1, 0] == 0 and entropy[1, 1] == 0
    assert torch.isfinite(entropy).all()
    _check(oil, x[:, 1:2].contiguous(), tokens[:, 1:2].contiguous(), 5)


@pytest.mark.parametrize("V", [40, 50021])
def test_not_finite(oil, V):
    x, tokens = _logits(1, 4, V, torch.float32)
    x[0, 0, 7], x[0, 1, 9], x[0, 2, V - 1] = math.nan, math.inf, math.nan
    tokens[0, :, 0] = -1
    logprob, entropy, ids, best = oil.token_logprobs(x, tokens, top=3)
    assert torch.isnan(entropy[0, :3]).all() and torch.isfinite(entropy[0, 3])
    assert torch.isnan(logprob[0, :3, 1:]).all() and (logprob[0, :, 0] == -math.inf).all()
    assert torch.isnan(best[0, :3]).all() and torch.isfinite(best[0, 3]).all()
    assert torch.equal(ids.long(), ref.logprobs(x[0], None, 3)[2][None])
    assert ids[0, 1, 0] == 9


def test_sharp_rows(oil):
    """Rows nearly certain, and offsets that a plain sum of exponentials would not hold."""
    x, tokens = _logits(1, 6, 4096, torch.float32)
    for i, (peak, shift) in enumerate(((20, 0), (60, 0), (12, 3e4), (0, -2e5), (30, 900), (5, -900))):
        x[0, i, 77] += peak
        x[0, i] += shift
    tokens[..., 0] = 77
    _check(oil, x, tokens, 8)


def test_streams_graph_and_workspace(oil):
    x, tokens = _logits(2, 9, 40001, torch.bfloat16)
    count = torch.tensor([9, 4], dtype=torch.int32, device="cuda")
    want = oil.token_logprobs(x, tokens, top=8, n_rows=count)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = oil.token_logprobs(x, tokens, top=8, n_rows=count, stream=side)
    again = oil.token_logprobs(x, tokens, top=8, n_rows=count)
    side.synchronize()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    graphs = []
    for top in (8, 3):                        # two graphs, with workspaces of their own
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, oil.token_logprobs(x, tokens, top=top, n_rows=count), top))
    for turn in range(3):
        for g, out, top in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out, top in graphs:
            eager = oil.token_logprobs(x, tokens, top=top, n_rows=count)
            assert all(torch.equal(a, b) for a, b in zip(out, eager))
            out[0].zero_()
    need = oil.lib().oil_token_logprobs_workspace_bytes(2, 9, 40001, oil.OIL_BF16, 8)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    got = oil.token_logprobs(x, tokens, top=8, n_rows=count, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(oil.OilError):
        oil.token_logprobs(x, tokens, top=8, workspace=ws[:need - 1])


def test_refusals(oil):
    x, tokens = _logits(2, 3, 100, torch.float32)
    for bad in (lambda: oil.token_logprobs(x.half(), tokens), lambda: oil.token_logprobs(x[0], tokens),
                lambda: oil.token_logprobs(x.cpu(), tokens), lambda: oil.token_logprobs(x, tokens.cpu()),
                lambda: oil.token_logprobs(x, tokens.long()), lambda: oil.token_logprobs(x, tokens[:1]),
                lambda: oil.token_logprobs(x, tokens, top=65), lambda: oil.token_logprobs(x, tokens, top=-1),
                lambda: oil.token_logprobs(x.transpose(1, 2), tokens), lambda: oil.token_logprobs(x[:, ::2], tokens[:, ::2]),
                lambda: oil.token_logprobs(x, tokens, n_rows=torch.zeros((3,), dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
