"""The 8-bit format as the tests' own definitions have it, against torch's (no GPU needed)."""
import numpy as np
import torch

import kvq_util as U


def test_code_values_are_e4m3fn():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(U.VALUES, want, equal_nan=True)
    assert np.nanmax(U.VALUES) == 448.0


def test_encode_rounds_to_nearest_even():
    rng = np.random.default_rng(1)
    between = (U._POSITIVE[1:] + U._POSITIVE[:-1]) / 2                         # ties
    x = np.concatenate([U._POSITIVE, between, np.nextafter(between, 0), np.nextafter(between, 500), rng.uniform(0, 448, 20000), np.exp(rng.uniform(-12, 6, 20000))])
    x = np.concatenate([x, -x])
    x32 = x.astype(np.float32)
    want = torch.from_numpy(x32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(U.encode(x32.astype(np.float64)), want)
    assert U.encode(np.inf) == U.NAN and U.encode(np.nan) & 0x7F == U.NAN


def test_smallest_scale():
    for most, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -120), (3.4e38, 120), (1e-45, -120)):
        s = U.smallest_scale([most, -most / 3, np.nan, -np.inf])
        assert s == 2.0 ** e, (most, s)
