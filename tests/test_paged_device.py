"""The paged-cache calls on a GPU that is not the current one. No GPU: tensors whose
`device` says cuda:1, a library that records with which device current it was
called, and the current device as a variable."""
import contextlib

import pytest
import torch

from paper_2608_23144_gb300 import _binding, _paged


class OnGpu1(torch.Tensor):
    device = property(lambda self: torch.device("cuda", 1))
    is_cuda = property(lambda self: True)


def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu1)


@pytest.fixture(params=[0, 1])
def gpus(request, monkeypatch):
    """{"current": device, "calls": [(function, device current then, stream)]}"""
    state = {"current": request.param, "calls": []}

    @contextlib.contextmanager
    def device(d):
        before, state["current"] = state["current"], torch.device(d).index
        yield
        state["current"] = before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                # the stream is the last argument, of awsrc_workspace_status the one before
                state["calls"].append((name, state["current"], args[1] if name == "awsrc_workspace_status" else args[-1]))
                return 0
            return call

    class Stream:
        def __init__(self, index):
            self.cuda_stream = 1000 + index

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(state["current"] if d is None else torch.device(d).index))
    monkeypatch.setattr(_paged, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(_paged, "_current_device", lambda: state["current"], raising=False)
    monkeypatch.setattr(_paged, "lib", Lib())
    monkeypatch.setattr(_binding, "lib", Lib())
    return state


def test_calls_run_with_the_device_of_the_cache_current(gpus, monkeypatch):
    before = gpus["current"]
    f8 = torch.float8_e4m3fn
    cache = _paged.awsrc_kv_cache(t(4, 2, 4, 16, 16, dtype=f8), t(4, 2, 1, 64, 16, dtype=f8), t(4, 2, dtype=torch.int8),
                                  t(4, 2, dtype=torch.int8))
    i32 = torch.int32
    batch = _paged.awsrc_kv_batch(t(2, dtype=i32), t(1, dtype=i32), t(1, 4, dtype=i32), 3, 3, 9)
    q, k = t(3, 4, 64), t(3, 2, 64)
    ws = t(1 << 10, dtype=torch.uint8)
    _paged.awsrc_kv_append(cache, batch, q, k, k, None, None, ws, q_out=q)
    _paged.awsrc_paged_attention(cache, batch, q, ws, out=t(3, 4, 64))
    _binding.awsrc_workspace_status(ws)
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", lambda *shape, dtype=None, device=None: t(*shape, dtype=dtype))
        _paged.awsrc_attention_workspace(cache, 4)
    calls = [c for c in gpus["calls"] if c[0] != "awsrc_attention_workspace_bytes"]  # asks for a size only
    assert [c[0] for c in calls] == ["awsrc_kv_append", "awsrc_paged_attention", "awsrc_workspace_status",
                                     "awsrc_attention_workspace_init"]
    assert all(current == 1 and stream == 1001 for _, current, stream in calls), calls
    assert gpus["current"] == before
