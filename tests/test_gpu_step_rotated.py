"""Decode steps from the projections (TieredCache.step_rotated): refusals, evictions, caches without a prefix, positions that are given."""
import numpy as np
import pytest
import torch

from paper_2604_19769_amd import binding as B
from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache
from test_gpu_rotary import DEV, DT, rnd
from test_gpu_shared_prefix import check, make_prefix, reference, stored_values, window

pytestmark = pytest.mark.gpu


def projections(seed, Bn, Hq, Hkv, dtype):
    x = rnd(seed, Bn, 1, Hq + 2 * Hkv, 128, dtype=dtype)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def test_a_refused_step_leaves_the_cache_as_it_was():
    p, _, _ = make_prefix(8, 2, "f16", 100)
    other, _, _ = make_prefix(8, 2, "f16", 100, scale=0.1)                    # refused by the library
    bf, _, _ = make_prefix(8, 2, "bf16", 100)                                 # takes bf16 queries only
    a, _ = window(3, 8, 2, "f16", [10, 63, 5], p)
    b, _ = window(3, 8, 2, "f16", [10, 63, 5], p)
    r = Rotary(Rotary.frequencies(), norm=True)
    q, k, v = projections(1, 3, 8, 2, "f16")
    for bad in (other, bf):
        a.share(bad)
        for _ in range(2):
            with pytest.raises(B.TTKVError):
                a.step_rotated(r, q, k, v)
            assert a.len[0].tolist() == [10, 63, 5]
    a.share(p)
    two = torch.cat((q, q), 1), torch.cat((k, k), 1), torch.cat((v, v), 1)
    for wrong in (two, (q, two[1], two[2]), (two[0], k, v), (q[:2], k[:2], v[:2]), (q, k, v[:, :, :1])):
        with pytest.raises(AssertionError):
            a.step_rotated(r, *wrong)
        assert a.len[0].tolist() == [10, 63, 5]
    for i in range(3):                                                        # then as if nothing had been
        q, k, v = projections(10 + i, 3, 8, 2, "f16")
        got, want = a.step_rotated(r, q, k, v), b.step_rotated(r, q, k, v)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert a.len[0].tolist() == [13, 66, 8]
    for x in (a, b, p, other, bf, r):
        x.close()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("given", ["none", "first", "positions"])
@pytest.mark.parametrize("dtype,src", [("f16", "f16"), ("f16", "bf16"), ("bf16", "f32")])
def test_steps_over_evictions(dtype, src, shared, given):
    """Norm, rotation, append, attention and evictions in one call and in its parts: the same rows in every tier, the same results."""
    Bn, Hq, Hkv = 2, 8, 2
    tiers = [TierConfig(dtype, dtype, 128, 64, 4), TierConfig("i8", "i8", 128, 64, 5), TierConfig("i4", "i4", 10 ** 9, 64, 8, paged_seed=3)]
    p, pk, pv = make_prefix(Hq, Hkv, dtype, 150)
    a, _ = window(Bn, Hq, Hkv, dtype, [100, 127], p if shared else None, [0, 1] if shared else None, tiers=tiers)
    b, _ = window(Bn, Hq, Hkv, dtype, [100, 127], p if shared else None, [0, 1] if shared else None, tiers=tiers)
    r = Rotary(Rotary.frequencies(128, 10000.0), norm=True, q_weight=rnd(1, 128) + 1, k_weight=rnd(2, 128) + 1)
    start = np.array([100, 127]) + (np.array([0, 150]) if shared else 0)
    for i in range(210):
        q, k, v = projections(5 + i, Bn, Hq, Hkv, src)
        first = (start + i) if given == "none" else np.array([7 * i, 100000 - i])
        pos = torch.from_numpy(first)[:, None].contiguous().to(DEV)
        kw = {} if given == "none" else dict(first_pos=first) if given == "first" else dict(positions=pos)
        out, lse = (x.clone() for x in a.step_rotated(r, q, k, v, **kw))
        qr, kr = r.apply(q, k, first_pos=first, dtype=DT[dtype])
        want, want_lse = b.step(qr.view(Bn, Hq, 128), kr.view(Bn, Hkv, 1, 128), v.to(DT[dtype]).contiguous().view(Bn, Hkv, 1, 128))
        # two orders of the same fp32 sums
        assert float((out - want).norm()) <= 5e-6 * float(want.norm()) and float((lse - want_lse).abs().max()) <= 1e-5, i
    assert [x.tolist() for x in a.len] == [x.tolist() for x in b.len] and a.len[2].min() > 0
    for t in range(3):
        for s in range(Bn):
            x, y = a.dump_tier(t, s), b.dump_tier(t, s)
            assert all(np.array_equal(x[n], y[n]) for n in x if x[n] is not None), (t, s)
    if dtype == "f16":                                                        # and against the definition, on the stored values
        q = rnd(3, Bn, Hq, 128, dtype=dtype)
        out, lse = a.decode(q)
        c = [one_sequence(a, s) for s in range(Bn)]
        check(out, lse, [reference(q[s], ([(pk.float(), pv.float())] if shared and s else []) + c[s], a.c.softmax_scale) for s in range(Bn)])
    for x in (a, b, p, r):
        x.close()


def one_sequence(c, s):
    """Stored values of every tier of sequence s, newest tier first."""
    class View:
        cfg = c.cfg

        @staticmethod
        def dump_tier(t, _):
            return c.dump_tier(t, s)
    return [tuple(x.float() for x in stored_values(View, t)) for t in range(len(c.cfg))]
