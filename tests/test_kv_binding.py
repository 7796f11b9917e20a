"""The 4-bit cache's binding on the host: no call here reaches a kernel."""
import random

import pytest
import torch

import paper_2608_03839_amd as oil


def test_kept_workspaces_are_bounded():
    """Buffers of a stream, whatever sizes its calls had and in whatever order."""
    rng = random.Random(1)
    for order in ("random", "up", "down"):
        needs = [rng.randrange(1, 1 << 20) for _ in range(500)]
        needs = needs if order == "random" else sorted(needs, reverse=order == "down")
        kept = oil._Workspaces()
        for i, n in enumerate(needs):
            ws = kept.get(("attend", (i,)), n, "cpu")
            assert ws.numel() == n and kept.by_sizes["attend", (i,)] is ws
            held = [b.data_ptr() for b in kept.buffers]
            assert ws.data_ptr() in held      # whoever holds an address has its buffer kept
        assert sum(b.numel() for b in kept.buffers) <= 4 * max(needs)


def test_remembered_sizes_are_bounded():
    kept = oil._Workspaces()
    for i in range(2 * kept.SIZES + 5):
        kept.get(("evict", (i, 1)), 64, "cpu")
    assert len(kept.by_sizes) <= kept.SIZES and len(kept.buffers) == 1


# ------------------------------------------------------------------ devices
class _Tensor:
    """What the binding asks of a tensor: dense, of a device of its own."""

    def __init__(self, *shape, dtype=torch.bfloat16, index=1):
        self.shape, self.dtype, self.index, self.device = torch.Size(shape), dtype, index, torch.device("cuda", index)
        self.is_cuda = True

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 4096 * (1 + self.index)


class _Stream:
    def __init__(self, index):
        self.device, self.cuda_stream = torch.device("cuda", index), 77


@pytest.fixture
def cache(monkeypatch):
    """A cache on cuda:1 in a process whose current device is cuda:0; `cache.calls` holds each
    C call's name and the device that was current."""
    current, calls = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                calls.append((name, current[0]))
                return 0
            return call

    monkeypatch.setattr(oil, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 10 + index, raising=False)
    c = oil.KvCache.__new__(oil.KvCache)
    c.n_slots, c.n_heads, c.head_dim, c.capacity = 4, 2, 64, 40
    c.device, c._index, c.handle, c._kept, c.calls = torch.device("cuda", 1), 1, None, {}, calls
    return c


def _arguments(index=1, odd=None):
    """Tensors of every call; the one named `odd` on cuda:0."""
    at = lambda name: 0 if name == odd else index  # noqa: E731
    i32 = torch.int32
    t = dict(q=_Tensor(2, 3, 4, 64, index=at("q")), k=_Tensor(2, 3, 2, 64, index=at("k")),
             v=_Tensor(2, 3, 2, 64, index=at("v")), slots=_Tensor(2, dtype=i32, index=at("slots")),
             nodes=_Tensor(2, 3, dtype=i32, index=at("nodes")), count=_Tensor(2, dtype=i32, index=at("count")),
             mask=_Tensor(2, 3, 1, dtype=i32, index=at("mask")), out=_Tensor(2, 3, 4, 64, index=at("out")),
             lse=_Tensor(2, 3, 4, dtype=torch.float32, index=at("lse")),
             weight=_Tensor(2, 2, 3, dtype=torch.float32, index=at("weight")),
             ws=_Tensor(4096, dtype=torch.uint8, index=at("ws")),
             rows=_Tensor(2, 2, 5, 64, index=at("rows")))
    return t


def _calls(c, t, stream=None):
    return {
        "reset": lambda: c.reset(t["slots"], stream=stream),
        "append": lambda: c.append(t["k"], t["v"], t["nodes"], t["count"], t["weight"], t["slots"], stream),
        "read": lambda: c.read(0, 5, slots=t["slots"], out=(t["rows"], t["rows"]), stream=stream),
        "attend": lambda: c.attend(t["q"], t["k"], t["v"], t["count"], t["mask"], slots=t["slots"],
                                   out=(t["out"], t["lse"]), workspace=t["ws"], stream=stream),
        "weigh": lambda: c.weigh(t["q"], t["lse"], t["nodes"], t["count"], slots=t["slots"], stream=stream),
        "evict": lambda: c.evict(7, slots=t["slots"], workspace=t["ws"], stream=stream),
    }


def test_calls_go_to_the_cache_s_device(cache):
    for name, call in _calls(cache, _arguments()).items():
        del cache.calls[:]
        call()
        assert cache.calls == [("oil_kv_" + name, 1)]
    assert torch.cuda.current_device() == 0


def test_tensors_of_other_devices_are_refused(cache):
    takes = dict(q=("attend", "weigh"), k=("append", "attend"), v=("append", "attend"), mask=("attend",),
                 slots=("reset", "append", "read", "attend", "weigh", "evict"), nodes=("append", "weigh"),
                 count=("append", "attend", "weigh"), out=("attend",), lse=("attend", "weigh"), weight=("append",),
                 ws=("attend", "evict"), rows=("read",))
    for odd, names in takes.items():
        calls = _calls(cache, _arguments(odd=odd))
        for name in names:
            with pytest.raises(ValueError):
                calls[name]()
    assert not cache.calls


def test_streams_of_other_devices_are_refused(cache):
    for call in _calls(cache, _arguments(), _Stream(0)).values():
        with pytest.raises(ValueError):
            call()
    assert not cache.calls
    for call in _calls(cache, _arguments(), _Stream(1)).values():
        call()
    assert len(cache.calls) == 6
