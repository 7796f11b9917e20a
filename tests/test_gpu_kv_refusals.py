"""The 4-bit cache's refusals on a live handle: each returns its status before
anything is enqueued, and the cache is as it was."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oil():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_03839_amd as m
    m.lib()
    return m


def test_statuses(oil):
    L = oil.lib()
    c = oil.KvCache(600, 2, 64, 40)
    h = c.handle
    buf = torch.zeros((1 << 22,), dtype=torch.uint8, device="cuda")
    P = ctypes.c_void_p(buf.data_ptr())
    bad = ctypes.c_void_p(buf.data_ptr() + 8)
    n = 1 << 22
    before = c.state.clone()
    assert L.oil_kv_reset(h, None, 0, None) == -1
    assert L.oil_kv_reset(h, None, 601, None) == -1
    ap = lambda **k: L.oil_kv_append(h, None, k.get("B", 2), k.get("k", P), k.get("v", P), k.get("dt", 1),
                                     k.get("ld", 128), k.get("rows", 4), k.get("nodes"), k.get("count"), None, None)
    for kw in (dict(B=0), dict(B=601), dict(k=None), dict(v=None), dict(dt=2), dict(ld=120), dict(ld=132),
               dict(rows=0), dict(nodes=P), dict(k=bad), dict(v=bad)):
        assert ap(**kw) == -1, kw
    assert ap(nodes=P, count=P, rows=257) == -3
    rd = lambda first, m, dt=1, k=P: L.oil_kv_read(h, None, 2, first, m, k, P, dt, None)
    assert rd(-1, 4) == rd(0, 0) == rd(0, 41) == rd(38, 3) == rd(0, 4, 7) == rd(0, 4, 1, None) == rd(0, 4, 1, bad) == -1
    at = lambda **k: L.oil_kv_attend(h, None, k.get("B", 2), k.get("q", P), k.get("q_ld", 256), k.get("Hq", 4),
                                     k.get("k"), k.get("v"), k.get("ld", 128), None, k.get("mask"), k.get("N", 3),
                                     k.get("scale", 1.0), k.get("ws", P), k.get("nb", n), k.get("out", P), P, None)
    for kw in (dict(B=0), dict(B=601), dict(q=None), dict(q=bad), dict(q_ld=248), dict(q_ld=260), dict(Hq=3),
               dict(Hq=0), dict(k=P), dict(v=P), dict(k=P, v=P, ld=64), dict(k=P, v=bad), dict(mask=P), dict(N=0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None), dict(out=bad)):
        assert at(**kw) == -1, kw
    for kw in (dict(B=513), dict(N=257), dict(Hq=130, q_ld=130 * 64)):
        assert at(**kw) == -3, kw
    need = L.oil_kv_attend_workspace_bytes(h, 2, 3, 4)
    assert need > 0
    assert at(ws=None) == at(nb=need - 1) == at(ws=bad) == -5
    assert L.oil_kv_attend_workspace_bytes(h, 2, 257, 4) == 0
    we = lambda **k: L.oil_kv_weigh(h, None, k.get("B", 2), k.get("q", P), k.get("q_ld", 256), k.get("Hq", 4),
                                    k.get("lse", P), k.get("N", 3), k.get("nodes"), k.get("count"),
                                    k.get("scale", 1.0), None)
    for kw in (dict(q=None), dict(q=bad), dict(lse=None), dict(nodes=P), dict(q_ld=8), dict(scale=float("inf"))):
        assert we(**kw) == -1, kw
    assert we(N=257) == -3
    ev = lambda **k: L.oil_kv_evict(h, None, k.get("B", 2), k.get("keep", 10), k.get("recent", 0), k.get("ws", P),
                                    k.get("nb", n), None)
    for kw in (dict(B=0), dict(keep=0), dict(keep=41), dict(recent=-1), dict(recent=11)):
        assert ev(**kw) == -1, kw
    assert ev(B=513) == -3
    need = L.oil_kv_evict_workspace_bytes(h, 2, 10)
    assert need > 0 and ev(nb=need - 1) == ev(ws=None) == ev(ws=bad) == -5
    torch.cuda.synchronize()
    assert torch.equal(c.state, before)


def test_binding_checks(oil):
    c = oil.KvCache(3, 2, 64, 40)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((2, 4, 2, 64), **bf)
    with pytest.raises(ValueError):
        oil.KvCache(1, 2, 60, 40)
    with pytest.raises(ValueError):
        c.append(x, x[:, :3])
    with pytest.raises(ValueError):
        c.append(x.half(), x.half())
    with pytest.raises(ValueError):
        c.append(x.cpu(), x.cpu())
    with pytest.raises(ValueError):
        c.append(x.transpose(1, 2).contiguous().transpose(1, 2), x)          # heads of a row apart
    with pytest.raises(ValueError):
        c.append(x, x, count=torch.zeros((3,), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        c.append(x, x, slots=torch.zeros((2,), dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        c.append(x, x, weight=torch.zeros((2, 4, 2), device="cuda"))
    q = torch.zeros((2, 4, 4, 64), **bf)
    with pytest.raises(ValueError):
        c.attend(q, x)
    with pytest.raises(ValueError):
        c.attend(q.float())
    with pytest.raises(ValueError):
        c.attend(q, x, x, mask=torch.zeros((2, 4, 2), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        c.attend(torch.zeros((2, 4, 3, 64), **bf))
    with pytest.raises(ValueError):
        c.weigh(q, torch.zeros((2, 4, 2), device="cuda"))
    with pytest.raises(oil.OilError):
        c.evict(10, 11)
    with pytest.raises(ValueError):
        c.evict(41)
