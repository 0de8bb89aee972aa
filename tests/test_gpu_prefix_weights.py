"""Values behind a shared prefix that lie near their type's largest."""
import pytest
import torch

from test_gpu_rotary import DT, rnd
from test_gpu_shared_prefix import check, make_prefix, reference

pytestmark = pytest.mark.gpu


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
