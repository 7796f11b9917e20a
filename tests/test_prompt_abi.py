"""Refusals of the prompt calls, the packed append and the log probabilities, on the host:
no call here reaches a kernel.  And their reference against torch's own functions."""
import math

import pytest
import torch

from tests import _prompt_ref as ref
from tests.test_abi import _FakeBufs


@pytest.fixture(scope="module")
def L():
    import paper_2608_03839_amd as oil
    return oil.lib()


def test_prompt_statuses(L):
    f = _FakeBufs()
    P, bad = f.aligned, f.misaligned

    def attend(starts=P, B=2, total=10, q=P, q_ld=256, Hq=4, k=P, v=P, ld=128, H=2, D=64, scale=1.0, out=P, ws=P, nb=1 << 20):
        return L.oil_prompt_attend(starts, B, total, q, q_ld, Hq, k, v, ld, H, D, scale, ws, nb, out, None, None)

    def weigh(starts=P, B=2, total=10, q=P, q_ld=256, Hq=4, lse=P, k=P, ld=128, H=2, D=64, last=3, scale=1.0, weight=P,
              ws=P, nb=1 << 20):
        return L.oil_prompt_weigh(starts, B, total, q, q_ld, Hq, lse, k, ld, H, D, last, scale, ws, nb, weight, None)

    common = [dict(starts=None), dict(B=0), dict(total=0), dict(total=-5), dict(q=None), dict(q=bad), dict(k=None),
              dict(k=bad), dict(Hq=3), dict(Hq=0), dict(H=0), dict(D=0), dict(D=60), dict(q_ld=248), dict(q_ld=260),
              dict(ld=120), dict(ld=132), dict(scale=math.nan), dict(scale=math.inf)]
    for kw in common:
        assert attend(**kw) == -1 and weigh(**kw) == -1, kw
    for kw in (dict(v=None), dict(v=bad), dict(out=None), dict(out=bad)):
        assert attend(**kw) == -1, kw
    for kw in (dict(lse=None), dict(weight=None), dict(last=0), dict(last=-1)):
        assert weigh(**kw) == -1, kw
    for kw in (dict(B=513), dict(total=(1 << 28) + 1), dict(total=1 << 28, Hq=8), dict(H=257, Hq=257, q_ld=1 << 15,
                                                                                      ld=1 << 15),
               dict(D=136, q_ld=1024, ld=512), dict(Hq=130, q_ld=130 * 64), dict(q_ld=(1 << 24) + 8),
               dict(ld=(1 << 24) + 8)):
        assert attend(**kw) == -3 and weigh(**kw) == -3, kw
    need = L.oil_prompt_attend_workspace_bytes(2, 10, 4, 2)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=bad), dict(nb=need - 1)):
        assert attend(**kw) == -5, kw
    need = L.oil_prompt_weigh_workspace_bytes(2, 10, 4, 2, 3)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=bad), dict(nb=need - 1)):
        assert weigh(**kw) == -5, kw
    assert L.oil_prompt_attend_workspace_bytes(1, 10, 4, 2) == L.oil_prompt_weigh_workspace_bytes(1, 10, 4, 2, 3) == 256
    assert attend(B=1, ws=bad) == weigh(B=1, ws=bad) == -5
    for args in ((0, 10, 4, 2), (513, 10, 4, 2), (2, 0, 4, 2), (2, (1 << 28) + 1, 4, 2), (2, 1 << 28, 8, 2), (2, 10, 3, 2),
                 (2, 10, 0, 2), (2, 10, 4, 0), (2, 10, 130, 2), (2, 10, 257, 257)):
        assert L.oil_prompt_attend_workspace_bytes(*args) == L.oil_prompt_weigh_workspace_bytes(*args, 3) == 0, args
    assert L.oil_prompt_weigh_workspace_bytes(2, 10, 4, 2, 0) == 0


def test_append_packed_refuses_no_handle(L):
    P = _FakeBufs().aligned
    assert L.oil_kv_append_packed(None, None, 1, P, 4, P, P, 1, 64, None, None) == -1


def test_logprobs_statuses(L):
    f = _FakeBufs()
    P, bad = f.aligned, f.misaligned

    def call(B=2, N=3, n_rows=None, x=P, dt=1, V=100, ld=100, tokens=P, M=1, top=2, ws=P, nb=1 << 20, lp=P, ids=P, tl=P):
        return L.oil_token_logprobs(B, N, n_rows, x, dt, V, ld, tokens, M, top, ws, nb, lp, P, ids, tl, None)

    import ctypes
    odd = ctypes.c_void_p(P.value + 1)
    half = ctypes.c_void_p(P.value + 2)
    for kw in (dict(B=0), dict(N=0), dict(x=None), dict(x=odd), dict(dt=0, x=half), dict(dt=2), dict(V=0), dict(ld=99),
               dict(ld=1 << 60), dict(tokens=None), dict(M=-1), dict(top=-1), dict(lp=None), dict(ids=None),
               dict(tl=None)):
        assert call(**kw) == -1, kw
    for kw in (dict(top=65), dict(B=1 << 12, N=(1 << 11) + 1)):
        assert call(**kw) == -3, kw
    need = L.oil_token_logprobs_workspace_bytes(2, 3, 100, 1, 2)
    assert need > 0
    assert call(ws=bad) == call(nb=need - 1) == -5
    assert call(V=200000, ld=200000, ws=None) == -5
    for args in ((0, 3, 100, 1, 2), (2, 0, 100, 1, 2), (2, 3, 0, 1, 2), (2, 3, 100, 7, 2), (2, 3, 100, 1, 65),
                 (1 << 12, 1 << 12, 100, 1, 2)):
        assert L.oil_token_logprobs_workspace_bytes(*args) == 0, args


def test_reference():
    g = torch.Generator()
    g.manual_seed(1)
    q, k, v = (torch.randn((9, h, 8), generator=g) for h in (4, 2, 2))
    out, lse, _, _ = ref.attend(q, k, v, [1, 4, 4, 9], 0.5)
    assert torch.isnan(out[0]).all()
    for a, z in ((1, 4), (4, 9)):
        for i in range(a, z):
            for h in range(4):
                s = 0.5 * (k[a:i + 1, h // 2].double() @ q[i, h].double())
                assert torch.allclose(out[i, h], torch.softmax(s, 0) @ v[a:i + 1, h // 2].double())
                assert torch.allclose(lse[i, h], torch.logsumexp(s, 0))
    weight, _ = ref.weigh(q, k, lse, [1, 4, 4, 9], 100, 0.5)
    assert torch.allclose(weight[:, 1:].sum(), torch.tensor(8.0 * 4, dtype=torch.float64))   # each row and head gives 1
    weight, _ = ref.weigh(q, k, lse, [1, 4, 4, 9], 1, 0.5)
    assert torch.allclose(weight[:, 1:4].sum(1), torch.full((2,), 2.0, dtype=torch.float64))
    x = torch.tensor([[0.0, 2.0, 2.0, -math.inf]])
    y, entropy, ids, _, _ = ref.logprobs(x, None, 6)
    assert ids.tolist() == [[1, 2, 0, -1, -1, -1]]
    p = torch.tensor([1.0, math.e ** 2, math.e ** 2], dtype=torch.float64) / (1 + 2 * math.e ** 2)
    assert torch.allclose(entropy, -(p * p.log()).sum())
