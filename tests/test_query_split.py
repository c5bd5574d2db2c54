"""The queries of the 8-bit attention past 32 columns are sums of an e4m3 and an e5m2 number (attention_fp8.hip, Queries8):
how far such a sum is from the bf16 number, over all of them (CPU)."""
import numpy as np
import torch


def split(x):
    """hi + lo of x (float32, in units of the column's scale), 64 bits."""
    hi = x.to(torch.float8_e4m3fn)
    lo = (x - hi.float()).to(torch.float8_e5m2)
    return hi.double() + lo.double()


def bf16_up_to_448():
    x = torch.arange(1 << 15, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    return x[x <= 448]


def test_every_bf16_number_within_the_stated_bound():
    """Exact from 2^-13 of the column's largest value, which lies in (224, 448], and off by 2^-21 of it at most below."""
    x = bf16_up_to_448()
    assert x.numel() > 17000
    err = (split(x) - x.double()).abs()
    assert (err[x >= 2.0**-13 * 224] == 0).all() and (err[x >= 2.0**-6] == 0).all()
    assert err.max() <= 2.0**-21 * 224
    assert err.max() >= 2.0**-15                    # reached within a factor of two
    assert torch.equal(split(-x), -split(x))


def test_numbers_that_two_e4m3_parts_miss():
    """Two e4m3 numbers without a factor between them would be off by 2^-17.8 of the largest value."""
    x = bf16_up_to_448()
    hi = x.to(torch.float8_e4m3fn).float()
    two = hi.double() + (x - hi).to(torch.float8_e4m3fn).double()
    worst = (two - x.double()).abs().max().item()
    assert worst == 2.0**-10 and np.log2(worst / 225) > -17.82
