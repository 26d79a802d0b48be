"""The example that serves an attention layer from packed weights and the paged
8-bit cache, against the same layer in 64 bits with nothing held in 8 bits.

The limit: an e4m3 code is within 2^-4 of a normal value, 2^-4 / sqrt(3) in the
mean square at most (0.036). The weighted sum of values keeps that ratio, and the
same ratio of scores of unit variance moves the weights by as much; in quadrature
0.051. The BF16 roundings (2^-9) vanish beside it. Twice that is the limit."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")


@pytest.mark.parametrize("kw", [dict(heads=16, kv_heads=2, dim=128, users=3, prompt=300, steps=9, page=64),
                                dict(heads=8, kv_heads=4, dim=64, users=8, prompt=5, steps=30, page=16),
                                dict(heads=4, kv_heads=4, dim=128, users=1, prompt=1, steps=3, page=128)])
def test_attention_layer_example(kw):
    spec = importlib.util.spec_from_file_location("attention_layer", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(**kw)
    assert 0 < got["prompt_error"] < 0.102 and 0 < got["step_error"] < 0.102
