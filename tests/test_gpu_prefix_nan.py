"""Scores behind a shared prefix that are not numbers: the rows that meet one answer 0 with lse -inf, as in ttkv_decode_attn, and nobody else notices."""
import numpy as np
import pytest
import torch

from paper_2604_19769_amd.cache import TierConfig
from test_gpu_rotary import DEV, rnd
from test_gpu_shared_prefix import QUANT, check, make_prefix, reference, stored_values, window

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(2, 8, 2), (5, 32, 2), (70, 2, 2), (3, 128, 128)])
@pytest.mark.parametrize("n,where", [(700, 0), (700, 350), (700, 699), (33, 32), (1, 0), (65, 40)])
def test_a_key(dtype, n_seq, Hq, Hkv, n, where):
    p, k, v = make_prefix(Hq, Hkv, dtype, n, poison=False)
    q = rnd(1, n_seq, Hq, 128, dtype=dtype)
    out, lse = (x.clone() for x in p.attend_shared(q))
    k[1, where, 77] = float("nan")
    p.len[0][:] = 0
    p.append(0, k, v, seq=0)
    got, got_lse = p.attend_shared(q)
    G = Hq // Hkv
    bad = torch.zeros(Hq, dtype=torch.bool, device=DEV)
    bad[G:2 * G] = True
    assert bool((got[:, bad] == 0).all()) and bool((got_lse[:, bad] == -np.inf).all())
    assert torch.equal(got[:, ~bad], out[:, ~bad]) and torch.equal(got_lse[:, ~bad], lse[:, ~bad])
    one, one_lse = p.decode(q[:1].contiguous())
    assert torch.equal(one[0, bad], got[0, bad]) and torch.equal(one_lse[0, bad], got_lse[0, bad])
    p.close()


def check_but(bad, out, lse, refs):
    """0 and -inf in the bad rows; the others against 64 bits (bits may differ from those without a bad row: the 32 rows of a wave move their
    references together, and an exponent's rounding goes with its size)."""
    assert bool((out[bad] == 0).all()) and bool((lse[bad] == -np.inf).all())
    out, lse = out.double().cpu(), lse.double().cpu()
    for i, b in enumerate(bad.cpu()):
        out[i][b], lse[i][b] = refs[i][0][b], refs[i][1][b]
    check(out, lse, refs)


@pytest.mark.parametrize("k_fmt,v_fmt", QUANT + [("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("q_type", ["f16", "bf16"])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(3, 8, 2), (70, 4, 2)])
def test_a_query(k_fmt, v_fmt, q_type, n_seq, Hq, Hkv):
    if k_fmt == "bf16" and q_type == "f16":
        pytest.skip("bf16 keys take bf16 queries")
    p, _, _ = make_prefix(Hq, Hkv, "f16", 0, tiers=[TierConfig(k_fmt, v_fmt, 10 ** 9, 64, 12)], poison=False)
    src = k_fmt if k_fmt in ("f16", "bf16") else "f32"
    p.append(0, rnd(2, Hkv, 650, 128, dtype=src), rnd(3, Hkv, 650, 128, dtype=src), seq=0)
    q = rnd(1, n_seq, Hq, 128, dtype=q_type)
    q[1, 1, 5] = float("nan")
    q[2, Hq - 1] = -float("nan")
    bad = torch.zeros(n_seq, Hq, dtype=torch.bool, device=DEV)
    bad[1, 1] = bad[2, Hq - 1] = True
    out, lse = p.attend_shared(q)
    kv = stored_values(p, 0)
    check_but(bad, out, lse, [reference(x, [kv], p.c.softmax_scale) for x in torch.nan_to_num(q)])
    p.close()


def test_a_query_of_a_step():
    p, pk, pv = make_prefix(8, 2, "f16", 300)
    c, own = window(3, 8, 2, "f16", [10, 70, 5], p, [1, 1, 0])
    q = rnd(1, 3, 8, 128, dtype="bf16")
    q[1, 3, 100] = float("nan")
    bad = torch.zeros(3, 8, dtype=torch.bool, device=DEV)
    bad[1, 3] = True
    out, lse = c.decode(q)
    check_but(bad, out, lse, [reference(x, ([(pk, pv)] if b < 2 else []) + [own[b]], c.c.softmax_scale) for b, x in enumerate(torch.nan_to_num(q))])
    c.close(), p.close()
