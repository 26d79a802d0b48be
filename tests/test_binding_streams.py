"""What the other calls allocate for a call on another stream than the current one, as
tests/test_step_streams.py has it for the serving steps (whose recording tensors and
streams are used here). No GPU."""
import ctypes as ct

import pytest
import torch

from paper_2608_23144_gb300 import _binding, _paged
from test_step_streams import CURRENT, I32, SIDE, record, t  # noqa: F401

BF16, F8, U8 = torch.bfloat16, torch.float8_e4m3fn, torch.uint8
PRM = _binding.params(C=64, P=4, b=4, S=64)
ROWS, COLS = 8, 128
MODULE = {"W": t(ROWS, COLS, dtype=BF16), "W0": t(ROWS, COLS, dtype=BF16), "act": t(COLS), "fisher": None}
PACKED = {"codes": t(ROWS * COLS // 2, dtype=U8), "scales": t(ROWS * COLS // 128, dtype=torch.int16)}
CACHE = _paged.awsrc_kv_cache(t(4, 2, 4, 16, 16, dtype=F8), t(4, 2, 1, 64, 16, dtype=F8), t(4, 2, dtype=torch.int8),
                              t(4, 2, dtype=torch.int8))
BATCH = _paged.awsrc_kv_batch(t(2, dtype=I32), t(1, dtype=I32), t(1, 4, dtype=I32), 3, 3, 9)
Q, K, WS, BYTES = t(3, 4, 64), t(3, 2, 64), t(1 << 10, dtype=U8), t(256, dtype=U8)
SHAPES = [(ROWS, COLS)]

CALLS = {  # (allocations, call)
    "encode_tiles": (2, lambda s: _binding.awsrc_encode_tiles(PRM, [MODULE], stream=s)),
    "rtn_quantize": (3, lambda s: _binding.awsrc_rtn_quantize(MODULE["W"], stream=s)),
    "rtn_quantize_sdq": (5, lambda s: _binding.awsrc_rtn_quantize(MODULE["W"], sdq=True, stream=s)),
    "rtn_quantize_batch": (6, lambda s: _binding.awsrc_rtn_quantize_batch([MODULE["W"]] * 2, stream=s)),
    "sidecar_prepare": (1, lambda s: _binding.awsrc_sidecar_prepare(PRM, SHAPES, BYTES, stream=s)),
    "packed_gemv": (1, lambda s: _binding.awsrc_packed_gemv(PRM, SHAPES, 0, PACKED, t(1, COLS), stream=s)),
    "packed_gemv_batch": (1, lambda s: _binding.awsrc_packed_gemv_batch(PRM, SHAPES, [(0, PACKED, t(1, COLS))], stream=s)),
    "gen_basis": (1, lambda s: _binding.awsrc_gen_basis(PRM, stream=s)),
    "select_records": (4, lambda s: _binding.awsrc_select_records(PRM, [MODULE], t(16, 16, dtype=U8), [0.5], stream=s)),
    "decode_apply": (2, lambda s: _binding.awsrc_decode_apply(PRM, [MODULE], BYTES, 3, stream=s)),
    "verify_reciprocal": (1, lambda s: _binding.awsrc_verify_reciprocal(0, 1, stream=s)),
    "attention_workspace": (1, lambda s: _paged.awsrc_attention_workspace(CACHE, 4, stream=s)),
    "kv_append": (1, lambda s: _paged.awsrc_kv_append(CACHE, BATCH, Q, K, K, None, None, WS, stream=s)),
    "paged_attention": (1, lambda s: _paged.awsrc_paged_attention(CACHE, BATCH, Q, WS, stream=s)),
}


class Lib:
    """Answers sizes with 64 and records the stream of every other call."""

    def __init__(self, calls):
        self.calls = calls

    def __getattr__(self, name):
        def call(*args):
            if name.endswith(("_bytes", "_capacity")):
                ct.cast(args[-1], ct.POINTER(ct.c_size_t))[0] = 64
            else:
                self.calls.append(args[-1])
            return 0
        return call


@pytest.fixture
def world(record, monkeypatch):  # noqa: F811
    for module in (_binding, _paged):
        monkeypatch.setattr(module, "lib", Lib(record["calls"]))
    like, made = torch.empty_like, record["made"]

    def empty_like(x, dtype=None, device=None):
        made.append(record["now"])
        return like(x, dtype=dtype).as_subclass(type(x))

    monkeypatch.setattr(torch, "empty_like", empty_like)
    return record


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_is_made_on_its_stream(name, world):
    many, call = CALLS[name]
    call(SIDE)
    assert world["calls"] == [SIDE.cuda_stream] and world["now"] is CURRENT
    assert world["made"] == [SIDE] * many and world["kept"] == [CURRENT] * many


@pytest.mark.parametrize("name", CALLS)
def test_calls_without_a_stream_allocate_on_the_current_one(name, world):
    many, call = CALLS[name]
    call(None)
    assert world["calls"] == [CURRENT.cuda_stream]
    assert world["made"] == [CURRENT] * many and not world["kept"]


def test_rows_of_x_apart_are_put_together_on_the_products_stream(world, monkeypatch):
    """A packed product takes x as whole rows; a copy that it makes for that belongs to its stream as well."""
    seen, reshape = [], type(CACHE.k).reshape
    monkeypatch.setattr(type(CACHE.k), "reshape", lambda self, *s: (seen.append(world["now"]), reshape(self, *s))[1])
    x = t(2, 3, COLS).transpose(0, 1)  # its rows do not lie at one step
    assert not x.is_contiguous()
    _binding.awsrc_packed_gemv(PRM, SHAPES, 0, PACKED, x, stream=SIDE)
    assert seen == [SIDE]


def test_the_reciprocals_count_is_read_on_the_calls_stream(world, monkeypatch):
    seen, item = [], torch.Tensor.item
    monkeypatch.setattr(type(CACHE.k), "item", lambda self: (seen.append(world["now"]), item(self))[1], raising=False)
    _binding.awsrc_verify_reciprocal(0, 1, stream=SIDE)
    assert seen == [SIDE]
