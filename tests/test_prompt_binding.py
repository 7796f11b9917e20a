"""The binding of the calls on packed prompts and logits on the host: the device that a call
goes to, and what it refuses.  No call here reaches a kernel."""
import pytest
import torch

import paper_2608_03839_amd as oil

F32, I32, U8 = torch.float32, torch.int32, torch.uint8


class _Tensor:
    """What the binding asks of a tensor: dense, of a device of its own."""

    def __init__(self, *shape, dtype=torch.bfloat16, index=1):
        self.shape, self.dtype, self.index, self.device = torch.Size(shape), dtype, index, torch.device("cuda", index)
        self.is_cuda = True

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def stride(self):
        strides, n = [], 1
        for s in reversed(self.shape):
            strides.insert(0, n)
            n *= s
        return tuple(strides)

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
def calls(monkeypatch):
    """Each C call's name, the device that was current and its arguments, in a process whose
    current device is cuda:0."""
    current, made = [0], []

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
                if name.endswith("workspace_bytes"):
                    return 512
                made.append((name, current[0], args))
                return 0
            return call

    monkeypatch.setattr(oil, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 10 + index, raising=False)
    return made


def _tensors(odd=None):
    """Tensors of every call on cuda:1; the one named `odd` on cuda:0."""
    shapes = dict(q=(9, 4, 64), k=(9, 2, 64), v=(9, 2, 64), starts=((3,), I32), out=(9, 4, 64), lse=((9, 4), F32),
                  weight=((2, 9), F32), ws=((4096,), U8), logits=((2, 3, 50), F32), tokens=((2, 3, 1), I32),
                  n_rows=((2,), I32), logprob=((2, 3, 1), F32), entropy=((2, 3), F32), best=((2, 3, 4), I32),
                  best_logprob=((2, 3, 4), F32))
    made = {}
    for name, s in shapes.items():
        shape, dtype = s if isinstance(s[0], tuple) else (s, torch.bfloat16)
        made[name] = _Tensor(*shape, dtype=dtype, index=0 if name == odd else 1)
    return made


def _calls(t, stream=None):
    return {
        "prompt_attend": lambda: oil.prompt_attend(t["q"], t["k"], t["v"], t["starts"], out=(t["out"], t["lse"]),
                                                   workspace=t["ws"], stream=stream),
        "prompt_weigh": lambda: oil.prompt_weigh(t["q"], t["k"], t["lse"], t["starts"], out=t["weight"],
                                                 workspace=t["ws"], stream=stream),
        "token_logprobs": lambda: oil.token_logprobs(
            t["logits"], t["tokens"], 4, t["n_rows"], workspace=t["ws"], stream=stream,
            out=(t["logprob"], t["entropy"], t["best"], t["best_logprob"])),
    }


def test_calls_go_to_their_tensors_device(calls):
    for name, call in _calls(_tensors()).items():
        del calls[:]
        call()
        (made, device, args), = calls
        assert made == "oil_" + name and device == 1 and args[-1] == 11
    for name, call in _calls(_tensors(), _Stream(1)).items():
        call()
        assert calls[-1][2][-1] == 77


def test_other_devices_are_refused(calls):
    takes = dict(q=("prompt_attend", "prompt_weigh"), k=("prompt_attend", "prompt_weigh"), v=("prompt_attend",),
                 starts=("prompt_attend", "prompt_weigh"), out=("prompt_attend",), lse=("prompt_attend", "prompt_weigh"),
                 weight=("prompt_weigh",), ws=("prompt_attend", "prompt_weigh", "token_logprobs"),
                 logits=("token_logprobs",), tokens=("token_logprobs",), n_rows=("token_logprobs",),
                 logprob=("token_logprobs",), entropy=("token_logprobs",), best=("token_logprobs",),
                 best_logprob=("token_logprobs",))
    for odd, names in takes.items():
        every = _calls(_tensors(odd))
        for name in names:
            with pytest.raises(ValueError):
                every[name]()
    for name, call in _calls(_tensors(), _Stream(0)).items():
        with pytest.raises(ValueError):
            call()
    assert not calls


def test_host_tensors_are_refused():
    q, k = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    starts = torch.tensor([0, 5], dtype=I32)
    for call in (lambda: oil.prompt_attend(q, k, k, starts), lambda: oil.prompt_weigh(q, k, torch.zeros((5, 4)), starts),
                 lambda: oil.token_logprobs(torch.zeros((1, 2, 30)))):
        with pytest.raises(ValueError):
            call()


def test_shapes_and_types_are_refused(calls):
    def attend(**kw):
        t = _tensors()
        t.update(kw)
        return _calls(t)["prompt_attend"]()

    def logprobs(**kw):
        t = _tensors()
        t.update(kw)
        return _calls(t)["token_logprobs"]()

    for kw in (dict(q=_Tensor(9, 256)), dict(k=_Tensor(8, 2, 64)), dict(k=_Tensor(9, 2, 32)), dict(v=_Tensor(9, 1, 64)),
               dict(q=_Tensor(9, 4, 64, dtype=F32)), dict(v=_Tensor(9, 2, 64, dtype=torch.float16)),
               dict(starts=_Tensor(3, dtype=torch.int64)), dict(out=_Tensor(9, 4, 32)), dict(lse=_Tensor(9, 4))):
        with pytest.raises(ValueError):
            attend(**kw)
    for kw in (dict(logits=_Tensor(2, 150, dtype=F32)), dict(logits=_Tensor(2, 3, 50, dtype=torch.float16)),
               dict(tokens=_Tensor(2, 3, dtype=I32)), dict(tokens=_Tensor(2, 4, 1, dtype=I32)), dict(n_rows=_Tensor(3, dtype=I32)),
               dict(best=_Tensor(2, 3, 3, dtype=I32))):
        with pytest.raises(ValueError):
            logprobs(**kw)
    assert not calls
