"""The serving-step calls on a GPU that is not the current one. No GPU: tensors whose
`device` says cuda:1, a library that records with which device current it was
called, and the current device as a variable."""
import contextlib

import pytest
import torch

from paper_2608_23144_gb300 import _paged, _step


class OnGpu1(torch.Tensor):
    device = property(lambda self: torch.device("cuda", 1))
    is_cuda = property(lambda self: True)


def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu1)


@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_with_the_device_of_their_tensors_current(current, monkeypatch):
    state, calls = {"current": current}, []

    @contextlib.contextmanager
    def device(d):
        before, state["current"] = state["current"], torch.device(d).index
        yield
        state["current"] = before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                calls.append((name, state["current"], args[-1]))
                return 0
            return call

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(_paged, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(_paged, "_current_device", lambda: state["current"])
    monkeypatch.setattr(_step, "lib", Lib())

    i32, ws = torch.int32, t(256, dtype=torch.uint8)
    pool = _step.awsrc_kv_pool(t(3, 4, dtype=i32), t(3, dtype=i32), t(9, dtype=i32), t(1, dtype=i32), 16)
    _step.awsrc_kv_plan(pool, t(3, dtype=i32), t(3, dtype=i32), ws, n_tok=5, q_start=t(4, dtype=i32), tok_pos=t(5, dtype=i32))
    _step.awsrc_verify_drafts(t(3, dtype=i32), t(5, dtype=i32), t(5, 11), t(5, 11, dtype=torch.bfloat16), t(5), t(2), ws,
                              kv_len=t(2, dtype=i32), accepted=t(2, dtype=i32), tokens=t(2, 4, dtype=i32), keep=t(2, dtype=i32))

    def matrix(rows, cols):
        blocks = -(-cols // 128)
        return _step.Fp8Matrix(rows, cols, t(blocks, -(-rows // 8) * 8, 128, dtype=torch.float8_e4m3fn),
                               t(-(-blocks // 4), -(-rows // 128), 32, 4, 4, dtype=torch.uint8))

    x8, w = matrix(6, 300), matrix(10, 300)
    _step.awsrc_fp8_quantize(t(6, 300), out=x8)
    _step.awsrc_fp8_gemm(x8, w, ws, out=t(6, 10))
    _step.awsrc_fp8_linear(t(6, 300), w, x8, ws, out=t(6, 10))
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", lambda *shape, dtype=None, device=None: t(*shape, dtype=dtype))
        _step.awsrc_step_workspace("cuda:1")
    calls = [c for c in calls if c[0] != "awsrc_step_workspace_bytes"]  # asks for a size only
    assert [c[0] for c in calls] == ["awsrc_kv_plan", "awsrc_verify_drafts", "awsrc_fp8_quantize", "awsrc_fp8_gemm",
                                     "awsrc_fp8_linear", "awsrc_step_workspace_init"]
    assert all(now == 1 and stream == 1001 for _, now, stream in calls), calls
    assert state["current"] == current
