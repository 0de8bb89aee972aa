"""Attention over a prefix that a batch shares (ttkv_shared_attn, ttkv_decode_step_shared) against a plain 64-bit
implementation on the stored values.

Tolerance.  Scores are fp32 sums of 128 exact products: at most 128 u (u = 2^-24) of sum |q_d k_d| off, typically sqrt(128) / 2 of it,
about 3e-7 of that sum; the exponential's argument and the power of two add 2 u of the score and 2^-23.  A weight is then off by
2^-17 sum |q k| scale + 2^-21 at the very most (it is split without loss beyond 2^-22).  The outputs are averages of values: off by
twice the weights' relative error times the largest |v| at most.  That is the element-wise bound; as independent errors they
average out, so the 2-norm of the difference is held to 1e-5 of the result's as well (a dropped remainder of the
weights gives 2e-4)."""
import numpy as np
import pytest
import torch

from paper_2604_19769_amd import binding as B
from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache
from test_gpu_rotary import DEV, DT, rnd

pytestmark = pytest.mark.gpu


def make_prefix(Hq, Hkv, dtype, n, bt=128, paged=None, extra=1, first_block=0, scale=None, seed=1, by=(1.0, 1.0), poison=True, tiers=None):
    """A cache of one sequence with n tokens; returns it with K, V [Hkv][n][128].  What is not live is NaN."""
    ring = -(-n // bt) + extra
    c = TieredCache(1, Hq, Hkv, tiers or [TierConfig(dtype, dtype, 10 ** 9, bt, ring, paged_seed=paged)], softmax_scale=scale)
    if poison:
        for p in c.pool:
            p.view(DT[dtype]).fill_(float("nan"))
    c.start[0][:] = first_block * bt
    k, v = rnd(seed, Hkv, n, 128, dtype=dtype, by=by[0]), rnd(seed + 1, Hkv, n, 128, dtype=dtype, by=by[1])
    if n:
        c.append(0, k, v, seq=0)
    return c, k, v


def reference(q, sets, scale):
    """q [Hq][128] of one sequence; sets: K, V [Hkv][n][128] to attend together.  out, lse and the element-wise bound, 64 bits."""
    k, v = (torch.cat([s[i].double() for s in sets], 1) for i in (0, 1))
    Hkv, G = k.shape[0], q.shape[0] // k.shape[0]
    q = q.double().view(Hkv, G, 128)
    if k.shape[1] == 0:
        return torch.zeros(Hkv * G, 128).double(), torch.full((Hkv * G,), -np.inf).double(), torch.zeros(Hkv * G, 1).double()
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    size = torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1) * scale
    out = torch.matmul(torch.softmax(s, -1), v)
    w = 2.0 ** -17 * size + 2.0 ** -21
    lim = 2 * w * v.abs().amax((1, 2)).view(-1, 1)
    return out.view(Hkv * G, 128).cpu(), torch.logsumexp(s, -1).view(-1).cpu(), lim.view(-1, 1).cpu()


def check(out, lse, refs, what=""):
    want, want_lse, lim = (torch.stack(x) for x in zip(*refs))
    out, lse = out.double().cpu(), lse.double().cpu()
    err = (out - want).abs()
    assert bool((err <= lim).all()), f"{what}: {float((err / lim.clamp_min(1e-300)).max()):.3g} times the bound"
    norm = float(want.norm())
    assert float((out - want).norm()) <= 1e-5 * norm, f"{what}: off by {float((out - want).norm()) / norm:.3g}"
    empty = torch.isinf(want_lse)
    assert torch.equal(lse[empty], want_lse[empty])
    d = (lse - want_lse)[~empty].abs()
    assert bool((d <= 1e-5 * want_lse[~empty].abs().clamp_min(1.0)).all()), what


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(1, 4, 4), (1, 8, 1), (3, 8, 2), (9, 28, 4), (33, 4, 4), (64, 8, 2), (65, 2, 2), (10, 64, 4), (129, 3, 1)])
@pytest.mark.parametrize("n", [1, 31, 33, 64, 65, 127, 129, 200, 1000])
def test_sizes(dtype, n_seq, Hq, Hkv, n):
    c, k, v = make_prefix(Hq, Hkv, dtype, n, bt=64, paged=5 if n % 2 else None, first_block=n % 3)
    q = rnd(7, n_seq, Hq, 128, dtype=dtype)
    out, lse = c.attend_shared(q)
    check(out, lse, [reference(x, [(k, v)], c.c.softmax_scale) for x in q])
    c.close()


@pytest.mark.parametrize("dtype,n_seq,Hq,Hkv,n,bt,paged", [("f16", 64, 32, 8, 9001, 128, 3), ("bf16", 24, 32, 32, 4100, 256, None), ("f16", 2, 8, 2, 30000, 64, 4),
                                                           ("bf16", 40, 8, 2, 20011, 1024, None), ("f16", 300, 8, 4, 3001, 128, None),
                                                           ("f16", 1500, 2, 2, 700, 64, 6), ("bf16", 2000, 4, 1, 321, 64, None)])
def test_long(dtype, n_seq, Hq, Hkv, n, bt, paged):
    c, k, v = make_prefix(Hq, Hkv, dtype, n, bt=bt, paged=paged, extra=2, first_block=1)
    q = rnd(8, n_seq, Hq, 128, dtype=dtype)
    out, lse = c.attend_shared(q)
    check(out, lse, [reference(x, [(k, v)], c.c.softmax_scale) for x in q])
    c.close()


@pytest.mark.parametrize("q_type,dtype", [("bf16", "f16"), ("f16", "f16")])
@pytest.mark.parametrize("scale,by", [(None, (8.0, 1.0)), (1.0, (1.0, 1.0)), (0.01, (0.1, 1e-3)), (4.0, (4.0, 100.0))])
def test_scores_of_all_sizes(q_type, dtype, scale, by):
    """Peaked and flat maps; a scale that the library takes as given."""
    c, k, v = make_prefix(8, 2, dtype, 777, scale=scale, by=by)
    q = rnd(9, 6, 8, 128, dtype=q_type)
    out, lse = c.attend_shared(q)
    s = c.c.softmax_scale
    refs = [reference(x, [(k, v)], s) for x in q]
    want = torch.stack([r[0] for r in refs])
    lim = torch.stack([r[2] for r in refs])
    assert bool(((out.double().cpu() - want).abs() <= lim).all())
    # scores grow with scale and keys, and their roundings with them: sqrt(128) / 2 roundings of |q| |k| scale
    rel = 2.0 ** -24 * 6 * float(torch.stack([x.double().norm(dim=-1).max() for x in q]).max() * k.double().norm(dim=-1).max()) * s
    assert float((out.double().cpu() - want).norm()) <= (2e-6 + 2 * rel) * float(want.norm())
    c.close()


def test_small_values_keep_their_digits():
    for dtype, by in (("f16", 2.0 ** -9), ("bf16", 1e-25), ("bf16", 1e25)):
        c, k, v = make_prefix(8, 2, dtype, 500, by=(1.0, by))
        q = rnd(10, 4, 8, 128, dtype=dtype)
        out, lse = c.attend_shared(q)
        check(out, lse, [reference(x, [(k, v)], c.c.softmax_scale) for x in q], f"{dtype} {by}")
        c.close()


def test_equal_and_extreme_scores():
    c, k, v = make_prefix(4, 2, "f16", 300)
    q = torch.zeros(3, 4, 128, dtype=torch.float16, device=DEV)            # every weight equal
    out, lse = c.attend_shared(q)
    mean = v.double().mean(1).repeat_interleave(2, 0).cpu()
    assert float((out.double().cpu() - mean).abs().max()) <= 2.0 ** -21
    assert float((lse.cpu() - np.log(300)).abs().max()) <= 2.0 ** -20
    c.close()
    c, k, v = make_prefix(4, 2, "f16", 300, by=(0.0, 1.0))
    k[:, 211] = 100.0
    c.len[0][:] = 0
    c.append(0, k, v, seq=0)
    q = torch.full((3, 4, 128), 100.0, dtype=torch.float16, device=DEV)    # one token takes everything (scores 0 and 113137)
    q[1] = -100.0                                                          # and one nothing
    out, lse = c.attend_shared(q)
    # its weight is 2^14 e^d, d the rounding of score x log2 e (up to 2^-8 at a score of 113137), so no round number: the two fp16
    # parts that multiply v hold it to 2^-22, the sum it is divided by to 2^-24, and product and quotient round once each
    want = v[:, 211].double().repeat_interleave(2, 0).cpu()
    for got in (out[0], out[2]):
        assert bool(((got.double().cpu() - want).abs() <= (2.0 ** -22 + 3 * 2.0 ** -24) * want.abs()).all())
    rest = (v.double().sum(1) - v[:, 211].double()).repeat_interleave(2, 0).cpu() / 299
    assert float((out[1].double().cpu() - rest).abs().max()) <= 2.0 ** -20
    c.close()


def test_a_value_that_is_not_a_number_reaches_its_head_only():
    c, k, v = make_prefix(4, 2, "bf16", 200, poison=False)
    v[1, 150, 5] = float("inf")
    c.len[0][:] = 0
    c.append(0, k, v, seq=0)
    out, lse = c.attend_shared(rnd(3, 2, 4, 128, dtype="bf16"))
    assert bool(torch.isfinite(out[:, :2]).all()) and bool(torch.isfinite(lse).all())
    bad = ~torch.isfinite(out[:, 2:])
    assert bool(bad[..., 5].all()) and int(bad.sum()) == 4
    c.close()


def test_empty_prefix_and_no_sequences():
    c, _, _ = make_prefix(4, 2, "f16", 0)
    out, lse = c.attend_shared(rnd(3, 5, 4, 128, dtype="f16"))
    assert bool((out == 0).all()) and bool((lse == -np.inf).all())
    out, lse = c.attend_shared(torch.empty(0, 4, 128, dtype=torch.float16, device=DEV))
    assert out.shape == (0, 4, 128)
    c.close()


def test_two_tiers_of_a_prefix():
    tiers = [TierConfig("f16", "f16", 10 ** 9, 64, 4), TierConfig("f16", "f16", 10 ** 9, 256, 4)]
    c, k, v = make_prefix(8, 2, "f16", 100, tiers=tiers)
    k1, v1 = rnd(5, 2, 700, 128, dtype="f16"), rnd(6, 2, 700, 128, dtype="f16")
    c.append(1, k1, v1, seq=0)
    q = rnd(7, 9, 8, 128, dtype="f16")
    out, lse = c.attend_shared(q)
    check(out, lse, [reference(x, [(k, v), (k1, v1)], c.c.softmax_scale) for x in q])
    c.close()


def stored_values(c, t):
    """K, V [Hkv][n][128] that tier t of a cache of one sequence stands for."""
    d, out = c.dump_tier(t, 0), []
    for name, fmt in (("k", c.cfg[t].k_fmt), ("v", c.cfg[t].v_fmt)):
        x = d[name]
        if fmt in ("f16", "bf16"):
            out.append(torch.from_numpy(x.view(np.int16).copy()).view(DT[fmt]).to(DEV))
            continue
        meta = d[name + "_meta"].view(np.float16).astype(np.float32)
        if fmt == "i8":
            v = x.view(np.int8).astype(np.float32) * np.repeat(meta, 32, -1)
        else:
            codes = np.stack((x & 15, x >> 4), -1).reshape(*x.shape[:-1], 128).astype(np.float32)
            v = codes * np.repeat(meta[..., 0::2], 64, -1) + np.repeat(meta[..., 1::2], 64, -1)
        out.append(torch.from_numpy(v).to(DEV))
    return tuple(out)


QUANT = [("i8", "i8"), ("i4", "i4"), ("i8", "i4")]


@pytest.mark.parametrize("k_fmt,v_fmt", QUANT)
@pytest.mark.parametrize("n_seq,Hq,Hkv,n,bt,paged,q_type", [
    (1, 4, 4, 1, 64, None, "f16"), (3, 8, 2, 31, 64, 3, "bf16"), (9, 28, 4, 65, 128, None, "f16"), (33, 4, 4, 200, 64, 5, "f16"),
    (64, 8, 2, 1000, 256, 6, "bf16"), (2, 8, 2, 20011, 128, 7, "f16"), (16, 32, 8, 4097, 1024, None, "f16"), (300, 2, 1, 700, 64, None, "f16")])
def test_quantized_tiers(k_fmt, v_fmt, n_seq, Hq, Hkv, n, bt, paged, q_type):
    c, _, _ = make_prefix(Hq, Hkv, "f16", 0, tiers=[TierConfig(k_fmt, v_fmt, 10 ** 9, bt, -(-n // bt) + 1, paged_seed=paged)], poison=False)
    c.pool[0].random_(0, 255)                                  # what is not live is anything
    c.start[0][:] = n % 3 * bt if -(-n // bt) >= 2 else bt
    loud = torch.ones(128, device=DEV)
    loud[::50] = 8.0
    k, v = (rnd(1, Hkv, n, 128) * loud).half(), rnd(2, Hkv, n, 128, dtype="f16")
    c.append(0, k, v, seq=0)
    q = rnd(7, n_seq, Hq, 128, dtype=q_type)
    kv = stored_values(c, 0)
    out, lse = c.attend_shared(q)
    check(out, lse, [reference(x, [kv], c.c.softmax_scale) for x in q])
    c.close()


@pytest.mark.parametrize("k_fmt,v_fmt", QUANT)
@pytest.mark.parametrize("by", [2.0 ** -9, 2.0 ** 9])
def test_quantized_values_of_all_sizes(k_fmt, v_fmt, by):
    c, _, _ = make_prefix(8, 2, "f16", 0, tiers=[TierConfig(k_fmt, v_fmt, 10 ** 9, 64, 8)], poison=False)
    k, v = rnd(1, 2, 400, 128, dtype="f16"), rnd(2, 2, 400, 128, dtype="f16", by=by)
    v[:, ::7] = 0.0                                            # scales of zero
    c.append(0, k, v, seq=0)
    q = rnd(7, 5, 8, 128, dtype="f16")
    out, lse = c.attend_shared(q)
    check(out, lse, [reference(x, [stored_values(c, 0)], c.c.softmax_scale) for x in q])
    c.close()


def test_a_tiered_prompt_as_prefix():
    """A prompt that went through fp16 -> int8 -> int4 evictions, shared by a batch with tiers of its own."""
    def tiers(ring):
        return [TierConfig("f16", "f16", 128, 64, 4), TierConfig("i8", "i8", 256, 64, 8), TierConfig("i4", "i4", 10 ** 9, 128, ring, paged_seed=3)]
    p, _, _ = make_prefix(8, 2, "f16", 0, tiers=tiers(12), poison=False)
    for i in range(9):
        p.append(0, rnd(3 * i, 2, 100, 128, dtype="f16"), rnd(3 * i + 1, 2, 100, 128, dtype="f16"), seq=0)
        p.demote()
    assert all(int(x[0]) > 0 for x in p.len) and sum(int(x[0]) for x in p.len) == 900
    prefix = [stored_values(p, t) for t in range(3)]
    sets = [(k.float(), v.float()) for k, v in prefix]
    c, own = window(5, 8, 2, "f16", [3, 0, 70, 64, 1], p, [1, 1, 1, 0, 1], tiers=tiers(2))
    for i in range(3):
        q, k, v = (rnd(60 + 3 * i + j, 5, h, 128, dtype="f16") for j, h in enumerate((8, 2, 2)))
        out, lse = c.step(q, k[:, :, None].contiguous(), v[:, :, None].contiguous())
        own = [[torch.cat((x[0], k[b, :, None]), 1), torch.cat((x[1], v[b, :, None]), 1)] for b, x in enumerate(own)]
        check(out, lse, [reference(q[b], (sets if b != 3 else []) + [own[b]], c.c.softmax_scale) for b in range(5)], f"step {i}")
    q = rnd(90, 64, 8, 128, dtype="f16")
    out, lse = p.attend_shared(q)
    check(out, lse, [reference(x, sets, p.c.softmax_scale) for x in q], "alone")
    c.close(), p.close()


def test_parts_of_several_calls_join():
    """As documented: m = lse, l = 1, acc = out."""
    a, ka, va = make_prefix(8, 2, "f16", 300, seed=1)
    b, kb, vb = make_prefix(8, 2, "f16", 45, seed=5)
    e, _, _ = make_prefix(8, 2, "f16", 0)
    q = rnd(7, 6, 8, 128, dtype="f16")
    parts = [[x.clone() for x in c.attend_shared(q)] for c in (a, e, b)]
    rows = 6 * 8
    acc = torch.stack([p[0].view(rows, 128) for p in parts], 1).contiguous()
    m = torch.stack([p[1].view(rows) for p in parts], 1).contiguous()
    out, lse = torch.empty(rows, 128, device=DEV), torch.empty(rows, device=DEV)
    B.ttkv_merge_partials(a.h, m, torch.ones_like(m), acc, 3, 3, None, rows, out, lse, a._compute())
    torch.cuda.synchronize()
    check(out.view(6, 8, 128), lse.view(6, 8), [reference(x, [(ka, va), (kb, vb)], a.c.softmax_scale) for x in q])
    for c in (a, b, e):
        c.close()


# ---------------------------------------------------------------- the decode step

def window(Bn, Hq, Hkv, dtype, held, prefix, members=None, tiers=None, seed=40):
    c = TieredCache(Bn, Hq, Hkv, tiers or [TierConfig(dtype, dtype, 10 ** 9, 64, max(held) // 64 + 2, paged_seed=9)], prefix=prefix, members=members)
    own = []
    for b, n in enumerate(held):
        k, v = rnd(seed + 2 * b, Hkv, n, 128, dtype=dtype), rnd(seed + 2 * b + 1, Hkv, n, 128, dtype=dtype)
        if n:
            c.append(0, k, v, seq=b)
        own.append([k, v])
    return c, own


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,held,n,members", [
    (8, 2, [0, 5, 64, 200], 300, None), (4, 4, [1, 0, 333], 129, [1, 0, 1]), (32, 8, [70] * 16, 2000, None), (8, 8, [3] * 33, 65, [b % 3 > 0 for b in range(33)]),
    (6, 2, [10, 20], 0, None), (8, 2, [100, 300, 50], 500, [0, 0, 0]), (8, 1, [900], 100, None), (16, 2, [1000, 1] * 20, 4097, [b != 7 for b in range(40)])])
def test_decode_step(dtype, Hq, Hkv, held, n, members):
    p, pk, pv = make_prefix(Hq, Hkv, dtype, n, bt=64, paged=2)
    Bn = len(held)
    c, own = window(Bn, Hq, Hkv, dtype, held, p, members)
    part = [True] * Bn if members is None else members
    for i in range(3):
        q, k, v = (rnd(60 + 3 * i + j, Bn, h, 128, dtype=dtype) for j, h in enumerate((Hq, Hkv, Hkv)))
        out, lse = c.step(q, k[:, :, None].contiguous(), v[:, :, None].contiguous())
        for b in range(Bn):
            own[b] = [torch.cat((own[b][0], k[b, :, None]), 1), torch.cat((own[b][1], v[b, :, None]), 1)]
        refs = [reference(q[b], ([(pk, pv)] if part[b] else []) + [own[b]], c.c.softmax_scale) for b in range(Bn)]
        check(out, lse, refs, f"step {i}")
        assert c.len[0].tolist() == [x + i + 1 for x in held]
    q = rnd(90, Bn, Hq, 128, dtype=dtype)                        # attend only
    out, lse = c.decode(q)
    check(out, lse, [reference(q[b], ([(pk, pv)] if part[b] else []) + [own[b]], c.c.softmax_scale) for b in range(Bn)], "attend")
    for b in range(Bn):                                          # the tokens are where they belong
        d = c.dump_tier(0, b)
        assert np.array_equal(d["k"].view(np.uint16), own[b][0].cpu().view(torch.int16).numpy().view(np.uint16))
        assert np.array_equal(d["v"].view(np.uint16), own[b][1].cpu().view(torch.int16).numpy().view(np.uint16))
    c.share(None)                                                # and alone again
    out, lse = c.decode(q)
    check(out, lse, [reference(q[b], [own[b]], c.c.softmax_scale) for b in range(Bn)], "alone")
    c.close(), p.close()


def test_sequences_without_own_tokens():
    p, pk, pv = make_prefix(8, 2, "f16", 200)
    c, _ = window(3, 8, 2, "f16", [0, 0, 0], p, [1, 0, 1])
    q = rnd(1, 3, 8, 128, dtype="f16")
    out, lse = c.decode(q)
    none = [pk[:, :0], pv[:, :0]]
    check(out, lse, [reference(q[b], [(pk, pv) if b != 1 else none], c.c.softmax_scale) for b in range(3)])
    c.close(), p.close()


def test_a_workspace_of_the_counted_parts_is_enough_and_steps_outgrow_it():
    """The parts are counted every 64 steps; a prefix that grows meanwhile makes the library ask for more."""
    p, _, _ = make_prefix(8, 2, "f16", 100, bt=64, extra=300)
    c, own = window(2, 8, 2, "f16", [10, 20], p)
    q, k, v = (rnd(60 + j, 2, h, 128, dtype="f16") for j, h in enumerate((8, 2, 2)))
    pk, pv = rnd(1, 2, 100, 128, dtype="f16"), rnd(2, 2, 100, 128, dtype="f16")
    for grow in (0, 15000, 3000):
        if grow:
            more = rnd(grow, 2, grow, 128, dtype="f16"), rnd(grow + 1, 2, grow, 128, dtype="f16")
            p.append(0, *more, seq=0)
            pk, pv = torch.cat((pk, more[0]), 1), torch.cat((pv, more[1]), 1)
        for _ in range(2):
            out, lse = c.step(q, k[:, :, None].contiguous(), v[:, :, None].contiguous())
            own = [[torch.cat((x[0], k[b, :, None]), 1), torch.cat((x[1], v[b, :, None]), 1)] for b, x in enumerate(own)]
        check(out, lse, [reference(q[b], [(pk, pv), own[b]], c.c.softmax_scale) for b in range(2)], f"grown by {grow}")
    c.close(), p.close()


def test_evicting_tiers_behind_a_prefix():
    """A prefix in front of fp16 -> int8 -> int4 tiers that evict: the step is the one without a prefix joined with the prefix."""
    tiers = [TierConfig("f16", "f16", 128, 64, 4), TierConfig("i8", "i8", 128, 64, 5), TierConfig("i4", "i4", 10 ** 9, 64, 8)]
    p, pk, pv = make_prefix(8, 2, "f16", 150)
    a, _ = window(2, 8, 2, "f16", [100, 127], p, tiers=tiers)
    b, _ = window(2, 8, 2, "f16", [100, 127], None, tiers=tiers)
    for i in range(200):
        q, k, v = (rnd(3 * i + j, 2, h, 128, dtype="f16") for j, h in enumerate((8, 2, 2)))
        args = k[:, :, None].contiguous(), v[:, :, None].contiguous()
        out, lse = a.step(q, *args)
        own, own_lse = b.step(q, *args)
        if i % 25 == 0 or i > 190:
            s, s_lse = p.attend_shared(q)
            w = torch.exp(own_lse - lse)[..., None].double(), torch.exp(s_lse - lse)[..., None].double()
            want = own.double() * w[0] + s.double() * w[1]
            assert float((out.double() - want).norm()) <= 5e-6 * float(want.norm()), i
    assert [x.tolist() for x in a.len] == [x.tolist() for x in b.len] and a.len[2].min() > 0
    for x in (a, b, p):
        x.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_from_the_projections(dtype):
    """Norm, rotation, append and attention behind a prefix that went the same way, over several steps: one layer's decode."""
    Bn, Hq, Hkv, n = 3, 8, 2, 333
    freq = Rotary.frequencies(128, 10000.0)
    wq, wk = rnd(1, 128) + 1, rnd(2, 128) + 1
    r = Rotary(freq, norm=True, q_weight=wq, k_weight=wk)
    p, _, _ = make_prefix(Hq, Hkv, dtype, 0, extra=4, paged=3)
    qkv = rnd(3, 1, n, Hq + 2 * Hkv, 128, dtype=dtype)
    p.append_rotated(r, qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:])
    c, _ = window(Bn, Hq, Hkv, dtype, [0] * Bn, p, [1, 1, 0], tiers=[TierConfig(dtype, dtype, 10 ** 9, 64, 3)])

    def turned(x, pos, w):                                     # [T][H][128] as the cache stores it
        x = x.double().cpu()
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.double().cpu()
        ang = torch.outer(pos.double(), torch.from_numpy(freq))[:, None]
        a, b = x[..., :64], x[..., 64:]
        return torch.cat((a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()), -1).to(DT[dtype])

    pk = turned(qkv[0, :, Hq:Hq + Hkv], torch.arange(n), wk).transpose(0, 1)
    pv = qkv[0, :, Hq + Hkv:].transpose(0, 1).cpu()
    own = [[torch.empty(Hkv, 0, 128, dtype=DT[dtype])] * 2 for _ in range(Bn)]
    for i in range(70):                                        # over a block's end
        x = rnd(100 + i, Bn, 1, Hq + 2 * Hkv, 128, dtype=dtype)
        out, lse = c.step_rotated(r, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:])
        refs = []
        for b in range(Bn):
            pos = torch.tensor([i + (n if b < 2 else 0)])
            own[b] = [torch.cat((own[b][0], turned(x[b, :, Hq:Hq + Hkv], pos, wk).transpose(0, 1)), 1),
                      torch.cat((own[b][1], x[b, :, Hq + Hkv:].transpose(0, 1).cpu()), 1)]
            refs.append(reference(turned(x[b, :, :Hq], pos, wq)[0], ([(pk, pv)] if b < 2 else []) + [own[b]], c.c.softmax_scale))
        if i % 23 == 0 or i > 66:
            # queries and keys are rounded to their type after fp32 arithmetic here and 64-bit arithmetic there: one in a few
            # thousand falls to the other side, one step (2 u) of one channel, which moves a score by 2 u |q_d k_d| scale
            want = torch.stack([z[0] for z in refs])
            u = torch.finfo(DT[dtype]).eps / 2
            assert float((out.double().cpu() - want).norm()) <= (1e-5 + u) * float(want.norm()), i
    c.close(), p.close(), r.close()


def test_captured_and_on_another_stream():
    c, k, v = make_prefix(8, 2, "f16", 3000)
    q = rnd(1, 12, 8, 128, dtype="f16")
    c.attend_shared(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = c.attend_shared(q)
    for i in range(4):
        q.copy_(rnd(30 + i, 12, 8, 128, dtype="f16"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        check(*got, [reference(x, [(k, v)], c.c.softmax_scale) for x in q], f"replay {i}")
        eager = c.attend_shared(q)
        assert torch.equal(eager[0], got[0]) and torch.equal(eager[1], got[1])        # the same sums in the same order
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [x.clone() for x in c.attend_shared(q)]
    side.synchronize()
    assert torch.equal(other[0], got[0])
    c.close()


def test_a_captured_step_and_two_caches_of_one_prefix_at_once():
    p, pk, pv = make_prefix(8, 2, "f16", 2500, paged=4)
    a, own_a = window(3, 8, 2, "f16", [100, 7, 333], p)
    b, own_b = window(40, 8, 2, "f16", [20 + i for i in range(40)], p, seed=200)
    qa, qb = rnd(1, 3, 8, 128, dtype="f16"), rnd(2, 40, 8, 128, dtype="f16")
    want = [[reference(q[i], [(pk, pv), own[i]], a.c.softmax_scale) for i in range(len(q))] for q, own in ((qa, own_a), (qb, own_b))]
    a.decode(qa), b.decode(qb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):                                     # both in flight, each with its own workspace
        with torch.cuda.stream(sa):
            ra = [x.clone() for x in a.decode(qa)]
        with torch.cuda.stream(sb):
            rb = [x.clone() for x in b.decode(qb)]
        torch.cuda.synchronize()
        check(*ra, want[0], "first"), check(*rb, want[1], "second")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = a.decode(qa)
    for i in range(4):
        qa.copy_(rnd(50 + i, 3, 8, 128, dtype="f16"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        check(*got, [reference(qa[i], [(pk, pv), own_a[i]], a.c.softmax_scale) for i in range(3)], f"replay {i}")
        eager = a.decode(qa)
        assert torch.equal(eager[0], got[0]) and torch.equal(eager[1], got[1])
    for c in (a, b, p):
        c.close()


def test_queries_in_front_of_the_batch_and_larger_batches_later():
    """The workspace grows with the number of sequences; results do not depend on what an earlier call left in it."""
    c, k, v = make_prefix(8, 4, "bf16", 900, bt=64)
    for n in (3, 70, 2, 200, 1):
        q = rnd(n, n, 8, 128, dtype="bf16")
        out, lse = c.attend_shared(q)
        check(out, lse, [reference(x, [(k, v)], c.c.softmax_scale) for x in q], f"{n} sequences")
    c.close()


def test_selection_is_refused_behind_a_prefix():
    p, _, _ = make_prefix(8, 2, "f16", 10)
    c, _ = window(2, 8, 2, "f16", [3, 3], p)
    q, k, v = (rnd(j, 2, h, 128, dtype="f16") for j, h in enumerate((8, 2, 2)))
    with pytest.raises(AssertionError):
        c.step(q, k[:, :, None].contiguous(), v[:, :, None].contiguous(), select_k=1)
    assert c.len[0].tolist() == [3, 3]
    c.close(), p.close()


def test_captured_calls_keep_buffers_of_their_own():
    """Two graphs of one cache at once, and after larger eager calls whose buffers replace the cache's (what was free in between is
    NaN now, and would not be if a graph still wrote there)."""
    p, k, v = make_prefix(8, 2, "f16", 1500)
    own, parts = window(3, 8, 2, "f16", [100, 7, 333], p)
    qa, qb = rnd(1, 4, 8, 128, dtype="f16"), rnd(2, 9, 8, 128, dtype="f16")
    qc = rnd(3, 3, 8, 128, dtype="f16")
    p.attend_shared(qa), own.decode(qc)
    torch.cuda.synchronize()
    graphs, results = [], []
    for run in (lambda: p.attend_shared(qa), lambda: p.attend_shared(qb), lambda: own.decode(qc)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = run()
            results.append((out * 1, lse * 1))
        graphs.append(graph)
        del out, lse
    p.attend_shared(rnd(5, 700, 8, 128, dtype="f16"))
    p.attend_shared(qa[:1].contiguous())
    own._workspace(4 * own.ws_parts)
    free = [torch.full((1 << s,), float("nan"), device="cuda") for s in range(8, 24) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in graphs]
    for i in range(4):
        for j, q in enumerate((qa, qb, qc)):
            q.copy_(rnd(10 * i + j + 7, *q.shape, dtype="f16"))
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for j, (q, got) in enumerate(zip((qa, qb), results)):
            check(*got, [reference(x, [(k, v)], p.c.softmax_scale) for x in q], f"graph {j}, replay {i}")
        check(*results[2], [reference(qc[b], [(k, v), parts[b]], own.c.softmax_scale) for b in range(3)], f"step, replay {i}")
    assert all(bool(x.isnan().all()) for x in free)
    for c in (own, p):
        c.close()


def test_a_prefix_has_no_prefix():
    p, _, _ = make_prefix(8, 2, "f16", 10)
    m, _, _ = make_prefix(8, 2, "f16", 20)
    c, _ = window(2, 8, 2, "f16", [3, 3], m)
    q = rnd(1, 2, 8, 128, dtype="f16")
    for bad in (m, p):
        with pytest.raises(AssertionError):
            bad.share(bad)
    m.share(p)
    for call in (lambda: c.share(m), lambda: c.decode(q), lambda: m.attend_shared(q)):
        with pytest.raises(AssertionError):
            call()
    m.share(None)
    c.decode(q), m.attend_shared(q)
    for x in (c, m, p):
        x.close()


@pytest.mark.parametrize("n_seq,Hq,Hkv", [(2, 8, 2), (5, 32, 2)])
def test_scores_that_are_not_numbers_answer_as_in_decode(n_seq, Hq, Hkv):
    """A NaN among a query's channels or in a live key: 0 and -inf for the rows that it meets, the others as they were."""
    p, k, v = make_prefix(Hq, Hkv, "f16", 700, poison=False)
    q = rnd(1, n_seq, Hq, 128, dtype="f16")
    q[1, Hq // 2] = float("nan")
    out, lse = (x.clone() for x in p.attend_shared(q))
    same_out, same_lse = [], []
    for x in q:
        one = [y.clone() for y in p.decode(x[None].contiguous())]
        same_out.append(one[0][0]), same_lse.append(one[1][0])
    bad = torch.zeros(n_seq, Hq, dtype=torch.bool, device="cuda")
    bad[1, Hq // 2] = True
    assert torch.equal(torch.stack(same_lse)[bad], lse[bad]) and torch.equal(torch.stack(same_out)[bad], out[bad])
    want = [reference(x, [(k, v)], p.c.softmax_scale) for x in torch.nan_to_num(q)]
    keep = ~bad.cpu()
    assert bool(((out.cpu().double() - torch.stack([w[0].view(Hq, 128) for w in want])).abs()[keep]
                 <= torch.stack([w[2].view(Hq, 1) for w in want])[keep]).all())
    p.close()
