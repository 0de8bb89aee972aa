"""Weights of a shared prefix that lie far below the largest one, and values near their type's largest.

A weight over fp16 values is an fp16 number and its remainder, together within half of fp16's smallest step, 2^-25, when the largest weight
carries 2^unit or more; that is 2^-(25 + unit) of the largest one, and 22 bits of the weight above it.  With unit = 14 a weight 2^-20 of the largest is
good to 2^-19 at most and, as a rounding error, to 2^-19 / sqrt(3) = 1.1e-6 on average: under the 1e-5 of the
2-norm that test_gpu_shared_prefix.py holds results to.  (Its element-wise bound knows nothing of small values beside a large weight.)"""
import numpy as np
import pytest
import torch

from test_gpu_rotary import DEV, DT, rnd
from test_gpu_shared_prefix import check, make_prefix, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(2, 256, 256), (5, 32, 8), (33, 256, 64), (200, 8, 8), (40, 64, 8)])
@pytest.mark.parametrize("octaves", [8, 14, 17, 20])
def test_a_large_weight_on_values_of_zero(dtype, n_seq, Hq, Hkv, octaves):
    """Every 32nd token takes nearly all the weight and has values of zero (what models do with a prompt's first token): the result is
    what the others leave, 2^-octaves of it each in the root mean square."""
    n = 512
    c, _, _ = make_prefix(Hq, Hkv, dtype, 0, extra=6)
    k, v = rnd(1, Hkv, n, 128, dtype=dtype), rnd(2, Hkv, n, 128, dtype=dtype)
    q = rnd(3, n_seq, Hq, 128, dtype=dtype)
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[:, ::32] = 0.0
    k[:, ::32, 0] = (octaves + 1.44) * np.log(2.0) / 8.0 / c.c.softmax_scale   # e^x, x of deviation 1: 2^1.44 in the root mean square
    v[:, ::32] = 0.0
    c.append(0, k, v, seq=0)
    out, lse = c.attend_shared(q)
    some = sorted({0, n_seq // 2, n_seq - 1})
    check(out[some], lse[some], [reference(q[i], [(k, v)], c.c.softmax_scale) for i in some])
    c.close()


@pytest.mark.parametrize("n_seq,Hq,Hkv", [(2, 8, 2), (40, 8, 2)])
@pytest.mark.parametrize("top", [1e36, 3e38])
def test_values_near_the_largest_of_bf16(n_seq, Hq, Hkv, top):
    """An average of values is no larger than the largest, and nothing on the way to it may be: 300 values of random sign and of up to 1e36 with weights
    of up to 1 stay below 3.4e38, and so does one of 3e38 among small ones."""
    c, k, v = make_prefix(Hq, Hkv, "bf16", 300, poison=False)
    v = (v.float().clamp(-1, 1) * 1e36).to(DT["bf16"])
    if top > 1e36:
        v[:, 1:] = 0.0
        v[:, 0] = top
    c.len[0][:] = 0
    c.append(0, k, v, seq=0)
    q = rnd(5, n_seq, Hq, 128, dtype="bf16")
    out, lse = c.attend_shared(q)
    some = [0, n_seq - 1]
    check(out[some], lse[some], [reference(q[i], [(k, v)], c.c.softmax_scale) for i in some])
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(3, 8, 8), (300, 8, 8), (64, 32, 8)])
@pytest.mark.parametrize("n", [1500, 8000])
def test_scores_that_grow_along_the_prefix(dtype, n_seq, Hq, Hkv, n):
    """References that move every few steps, by up to 30 powers of two in all: outputs, sums and weights on their way are scaled together.  (A score's sum of up
    to 240 is rounded eight times to 2^-17 at most, 2^-17 sqrt(8 / 12) scale = 5e-7 of a weight on average: the usual bounds hold.)"""
    c, _, _ = make_prefix(Hq, Hkv, dtype, 0, bt=64, extra=-(-n // 64) + 1, paged=4)
    k, v = rnd(1, Hkv, n, 128) * 0.3, rnd(2, Hkv, n, 128, dtype=dtype)
    k[:, :, 5] = 60.0 * torch.arange(n, device=DEV) / n
    k = k.to(DT[dtype])
    c.append(0, k, v, seq=0)
    q = rnd(7, n_seq, Hq, 128, dtype=dtype)
    q[:, :, 5] = 4.0
    out, lse = c.attend_shared(q)
    some = [0, n_seq // 2, n_seq - 1]
    check(out[some], lse[some], [reference(q[i], [(k, v)], c.c.softmax_scale) for i in some])
    c.close()
