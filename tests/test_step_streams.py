"""What the serving-step calls allocate for a call on another stream than the current
one: it has to be made (and filled) with that stream current, or nothing orders the
fill, and the work that last used the memory, with the kernel. No GPU: a wrong order
would be a race, so tensors whose `device` says cuda:0 are made by functions that
record which stream was current."""
import contextlib

import pytest
import torch

from paper_2608_23144_gb300 import _binding, _paged, _step

I32 = torch.int32


class OnGpu(torch.Tensor):
    device = property(lambda self: torch.device("cuda", 0))
    is_cuda = property(lambda self: True)


class Stream:
    device = torch.device("cuda", 0)

    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, SIDE = Stream(1000), Stream(2000)
ZEROS, EMPTY = torch.zeros, torch.empty


def t(*shape, dtype=torch.float32):
    return ZEROS(*shape, dtype=dtype).as_subclass(OnGpu)


def matrix(rows, cols):
    blocks = -(-cols // 128)
    return _step.Fp8Matrix(rows, cols, t(blocks, -(-rows // 8) * 8, 128, dtype=torch.float8_e4m3fn),
                           t(-(-blocks // 4), -(-rows // 128), 32, 4, 4, dtype=torch.uint8))


@pytest.fixture
def record(monkeypatch):
    """{"made": streams current when something was allocated, "kept": streams that memory was recorded on, "calls": streams}"""
    state = {"now": CURRENT, "made": [], "kept": [], "calls": []}

    @contextlib.contextmanager
    def stream(s):
        before, state["now"] = state["now"], s
        yield
        state["now"] = before

    def maker(make):
        def f(*shape, dtype=torch.float32, device=None):
            state["made"].append(state["now"])
            return make(*shape, dtype=dtype).as_subclass(OnGpu)
        return f

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if not name.endswith("_bytes"):
                    state["calls"].append(args[-1])
                return 0
            return call

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: state["now"])
    monkeypatch.setattr(OnGpu, "record_stream", lambda self, s: state["kept"].append(s), raising=False)
    monkeypatch.setattr(_paged, "_raw_stream", lambda index: state["now"].cuda_stream)
    monkeypatch.setattr(_paged, "_current_device", lambda: 0)
    for module in (_step, _binding):
        monkeypatch.setattr(module, "lib", Lib())
    monkeypatch.setattr(torch, "empty", maker(EMPTY))
    monkeypatch.setattr(torch, "zeros", maker(ZEROS))
    return state


WS = t(256, dtype=torch.uint8)
CALLS = {
    "step_workspace": (1, lambda s: _step.awsrc_step_workspace("cuda", stream=s)),
    "kv_plan": (1, lambda s: _step.awsrc_kv_plan(_step.awsrc_kv_pool(t(3, 4, dtype=I32), t(3, dtype=I32), t(9, dtype=I32),
                                                                     t(1, dtype=I32), 16), None, t(3, dtype=I32), WS, n_tok=5,
                                                 stream=s)),
    "verify_drafts": (2, lambda s: _step.awsrc_verify_drafts(t(3, dtype=I32), t(5, dtype=I32), t(5, 11), None, t(5), t(2), WS,
                                                             max_draft=3, stream=s)),
    "fp8_quantize": (2, lambda s: _step.awsrc_fp8_quantize(t(6, 300), stream=s)),
    "fp8_gemm": (1, lambda s: _step.awsrc_fp8_gemm(matrix(6, 300), matrix(10, 300), WS, stream=s)),
    "fp8_linear": (1, lambda s: _step.awsrc_fp8_linear(t(6, 300), matrix(10, 300), matrix(6, 300), WS, stream=s)),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_is_made_on_its_stream(name, record):
    many, call = CALLS[name]
    call(SIDE)
    assert record["calls"] == [SIDE.cuda_stream] and record["now"] is CURRENT
    assert record["made"] == [SIDE] * many
    assert record["kept"] == [CURRENT] * many  # nor handed out again while the caller's stream may read it


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("stream", [None, CURRENT])
def test_calls_on_the_current_stream_allocate_there(name, stream, record):
    many, call = CALLS[name]
    call(stream)
    assert record["calls"] == [CURRENT.cuda_stream]
    assert record["made"] == [CURRENT] * many and not record["kept"]
