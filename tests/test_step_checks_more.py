"""More of what the serving-step calls refuse before any launch (tests/test_step_checks.py
has the made-up addresses). No GPU: every call must stop at a check."""
import ctypes as ct

import pytest

import paper_2608_23144_gb300 as aw
from test_step_checks import INVALID, OK, P, mat


def linear(x8, w, rows=4):
    return aw.lib.awsrc_fp8_linear(P << 10, 0, 256, ct.byref(mat(rows=rows, **x8)), ct.byref(mat(**w)), P << 11, 0, 256, P << 12,
                                   1 << 30, None)


# 4 rows x 256: 2 x 8 x 128 bytes of codes, 512 of exponents; 200 rows: 2 x 200 x 128 and 1024
W = dict(rows=200, codes=P << 4, exps=P << 5)
C = 2 * 200 * 128


@pytest.mark.parametrize("x8", [
    dict(codes=(P << 4) + 128, exps=P), dict(codes=(P << 4) + C - 128, exps=P), dict(codes=(P << 4) - 1920, exps=P),  # codes
    dict(codes=P, exps=(P << 5) + 512), dict(codes=P, exps=(P << 5) - 496),                                           # exponents
    dict(codes=(P << 5) + 896, exps=P), dict(codes=P, exps=(P << 4) + 16),                                            # one in the other
])
def test_linear_refuses_codes_of_x_within_the_weights(x8):
    assert linear(x8, W) == INVALID


def test_codes_of_x_beside_the_weights_are_no_overlap():
    """Without rows nothing is launched, and nothing overlaps."""
    assert linear(dict(codes=(P << 4) + 128, exps=P), W, rows=0) == OK
