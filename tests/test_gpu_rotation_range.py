"""Rotation at the ends of its range (ttkv_norm_rope): every position up to 2^53 with every frequency below 1e6.  Tolerances:
those of test_gpu_rotary.py."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2604_19769_amd.cache import Rotary
from test_gpu_rotary import DEV, check, rnd

pytestmark = pytest.mark.gpu

PI = Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59)   # 60 digits: angles of up to 1e22 to 1e-37


def rotated(x, pos, freq):
    """x [1][T][H][128], pos [T]: every angle's remainder in whole numbers."""
    x = x.double().cpu().numpy()
    y, size, half = x.copy(), np.abs(x), len(freq)
    for t, p in enumerate(pos):
        for i, f in enumerate(freq):
            angle = Fraction(int(p)) * Fraction(float(f))
            angle = float(angle - 2 * PI * round(angle / (2 * PI)))
            c, s = np.cos(angle), np.sin(angle)
            a, b = x[0, t, :, i], x[0, t, :, i + half]
            y[0, t, :, i], y[0, t, :, i + half] = a * c - b * s, b * c + a * s
            size[0, t, :, i] = size[0, t, :, i + half] = np.abs(a) + np.abs(b)
    return y, size


@pytest.mark.parametrize("freq", [999999.0, 1000.0, 31.4159, -123456.789, 1.0, 1e-3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions_of_all_frequencies(freq, dtype):
    freq = freq * (1.0 - np.arange(16, dtype=np.float64) / 37)
    pos = np.array([(1 << 53) - 1, -(1 << 53), (1 << 53) - 12345, 1 << 50, (1 << 47) + 1, 987654321987, -77, 0, 1], np.int64)
    x = rnd(1, 1, len(pos), 3, 128, dtype=dtype)
    r = Rotary(freq)
    y, _ = r.apply(x, positions=torch.from_numpy(pos)[None].to(DEV))
    check(y, rotated(x, pos, freq), f"{freq[0]}")
    r.close()
