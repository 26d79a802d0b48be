"""The two 8-bit terms that the tiles kernel keeps a BF16 query in, over every bf16
value, restated on the CPU: an e4m3 term, then an e5m2 one of what it leaves, of a row
scaled by a power of two to a largest element in [2^7, 2^8). The header's limits: exact
from 2^-13 of the row's largest element on, below it within 2^-21 of that."""
import torch


def test_two_terms_hold_every_bf16_within_the_stated_limits():
    x = torch.arange(0x7F80, dtype=torch.int16).view(torch.bfloat16).double()
    x = x[x < 256]
    y = x.half()  # the kernel scales and splits in binary16
    hi = y.float().to(torch.float8_e4m3fn)
    lo = (y.float() - hi.float()).half().float().to(torch.float8_e5m2)
    err = (hi.double() + lo.double() - x).abs()
    assert (err[x >= 2.0 ** 8 * 2.0 ** -13 * 0.5] == 0).all()  # the largest element may be as small as 2^7
    assert err.max() <= 2.0 ** 7 * 2.0 ** -21
