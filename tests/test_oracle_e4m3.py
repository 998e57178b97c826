"""The oracle of numbers in 8 bits against torch's conversions, and its scales against their definition."""
import numpy as np
import torch

from oracle import e4m3


def test_every_code_and_every_bf16_number():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    assert np.array_equal(e4m3.VALUES, codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    want = x.to(torch.float8_e4m3fn).double().numpy()
    got = e4m3.VALUES[e4m3.encode(x.numpy())]
    assert np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got), np.signbit(want) & ~np.isnan(want))


def test_scales():
    for x, s in ((0.0, 10), (448.0, 127), (448.1, 128), (447.0, 127), (224.0, 126), (3.3e38, 247), (2.0 ** -140, 10), (float("inf"), 10), (float("nan"), 10)):
        assert e4m3.least_scale([0.0, x]) == s, x
    assert e4m3.least_scale([1.0, float("nan"), float("-inf")]) == e4m3.least_scale([1.0]) == 119
