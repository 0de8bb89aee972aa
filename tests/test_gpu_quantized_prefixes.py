"""Long prefixes in quantized tiers (ttkv_shared_attn) against a plain 64-bit implementation on the stored values: waves that
take many steps of 32 tokens each, over the ends of blocks, around the ring and through a block table.

Tolerance: that of test_gpu_shared_prefix.py, 1e-5 of the result in the 2-norm.  The sums are fp32 (u = 2^-24).  Steps of random
values add up like sqrt(n), and so do n independent roundings, each of at most the running sum and half a step's 32 values; of int4,
whose 16 codes with their zero point stand for 16 s (1 + n / 16) + (z - 16 s), a step's sum is some 32 * 24 s / 2 before its
zero points are in, against sqrt(32) * 4.6 s for its result: 15 u per rounding, sqrt(6) of them, 2e-6.  The sum of the weights (all
positive, n / 2 additions per lane) is off by sqrt(n / 2) u / 2 at n tokens per wave, 1e-6 at 2048."""
import numpy as np
import pytest
import torch

from paper_2604_19769_amd.cache import TierConfig
from test_gpu_rotary import DEV, rnd
from test_gpu_shared_prefix import QUANT, check, make_prefix, reference, stored_values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k_fmt,v_fmt", QUANT)
@pytest.mark.parametrize("n_seq,Hq,Hkv,n,bt,paged,by", [
    (2, 8, 2, 32001, 64, 3, 1.0),                             # 256 tokens per item: one step per wave, every second one in a block of its own
    (4, 28, 4, 130001, 1024, None, 1.0),                      # 256 tokens per wave
    (64, 32, 8, 16321, 64, 5, 1.0),                           # 512, eight blocks of rows
    (64, 64, 4, 32700, 256, 7, 1.0),                          # 2048
    (64, 64, 4, 32700, 128, 7, 0.25),                         # flat maps: the average of all values
    (33, 4, 4, 9000, 128, 6, 8.0)])                           # peaked ones: references that move
def test_many_steps_per_wave(k_fmt, v_fmt, n_seq, Hq, Hkv, n, bt, paged, by):
    ring = -(-n // bt) + 1
    c, _, _ = make_prefix(Hq, Hkv, "f16", 0, tiers=[TierConfig(k_fmt, v_fmt, 10 ** 9, bt, ring, paged_seed=paged)], poison=False)
    c.pool[0].random_(0, 255)                                  # what is not live is anything
    c.start[0][:] = ring // 2 * bt                             # the ring's end inside the run
    loud = torch.ones(128, device=DEV)
    loud[::50] = 8.0
    k, v = (rnd(1, Hkv, n, 128) * loud * by).half(), rnd(2, Hkv, n, 128, dtype="f16")
    c.append(0, k, v, seq=0)
    q = rnd(7, n_seq, Hq, 128, dtype="f16")
    kv = stored_values(c, 0)
    out, lse = c.attend_shared(q)
    some = sorted({0, n_seq // 2, n_seq - 1})
    check(out[some], lse[some], [reference(q[i], [kv], c.c.softmax_scale) for i in some])
    c.close()


@pytest.mark.parametrize("k_fmt,v_fmt", QUANT)
def test_scores_that_grow_along_the_prefix(k_fmt, v_fmt):
    """Every step's scores are above the ones before: outputs and zero points are rescaled together, many times."""
    n, bt = 8000, 64
    c, _, _ = make_prefix(8, 8, "f16", 0, tiers=[TierConfig(k_fmt, v_fmt, 10 ** 9, bt, n // bt + 1, paged_seed=4)], poison=False)
    k, v = rnd(1, 8, n, 128) * 0.3, rnd(2, 8, n, 128, dtype="f16")
    ramp = torch.arange(n, device=DEV) / n
    k[:, :, 5] = 60.0 * ramp
    c.append(0, k.half(), v, seq=0)
    q = rnd(7, 300, 8, 128, dtype="f16")
    q[:, :, 5] = 16.0                                          # from 0 to 122 powers of two
    kv = stored_values(c, 0)
    out, lse = c.attend_shared(q)
    some = [0, 150, 299]
    check(out[some], lse[some], [reference(q[i], [kv], c.c.softmax_scale) for i in some])
    c.close()
