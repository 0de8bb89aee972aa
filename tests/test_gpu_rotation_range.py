"""Rotation and norm at the ends of their ranges (ttkv_norm_rope): every position up to 2^53 with every frequency below 1e6, and rows
whose squares leave fp32's range.  Tolerances: those of test_gpu_rotary.py."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2604_19769_amd.cache import Rotary
from test_gpu_rotary import DEV, DT, check, rnd

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


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("by", [3e37, 1e25, 1e19, 1.0, 1e-7, 1e-19, 1e-22, 1e-35])
def test_norm_of_rows_of_all_sizes(dtype, eps, by):
    """The mean of the squares leaves fp32's range long before the row does."""
    if dtype == "f16" and not 1e-7 <= by <= 1.0:
        pytest.skip("not in fp16's range")
    x = rnd(2, 1, 6, 9, 128).clamp(-4, 4)
    x[0, 0, 0, 1:] = 0.0                                       # one channel alone
    x[0, 1, :, 64:] *= 1e-12                                   # large and small ones of a row
    x = (x * by).to(DT[dtype])
    x[0, 2, 3] = 0.0
    wq = rnd(3, 128).abs() + 0.5
    r = Rotary(Rotary.frequencies(0), norm=True, q_weight=wq, eps=eps)
    y, _ = r.apply(x, dtype=torch.float32)
    z = x.double()
    want = z / torch.sqrt((z * z).mean(-1, keepdim=True) + float(np.float32(eps))) * wq.double()
    if eps == 0.0:                                             # 0 / 0
        assert bool(y[0, 2, 3].isnan().all())
        y[0, 2, 3] = want[0, 2, 3] = 0.0
    err = (y.double() - want).abs()
    # the bound of test_gpu_rotary.py for a channel that does not turn; a result (or a factor of it) below 2^-126 is a multiple of 2^-149
    size = want.abs()
    assert bool((err <= (2.0 ** -24 + 2.0 ** -19) * size + 2.0 ** -148 * wq.double().amax()).all()), float((err / size.clamp_min(1e-300)).max())
    r.close()
