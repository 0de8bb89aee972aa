"""Norm per head, position rotation and the rotated append (ttkv_norm_rope, ttkv_rope_append) against a plain 64-bit
implementation.

Tolerance.  The result is rounded once to its type: u = finfo.eps / 2 of the value (fp16: or half a subnormal, 2^-25).  Before that,
in fp32 (u32 = 2^-24): the mean of squares (at most 19 additions and a product), root, quotient and two products (x inv w) put at
most 10 + 1 + 1 + 1.5 + 1 + 1 < 16 u32 on a channel; sine and cosine 2^-22 at most (reduction rounded to fp32, 2 pi 2^-26; the
function 2 ulp), one product each and a sum: 16 + 4 + 2 < 24 u32 of |a| + |b| = 2^-19 (|a| + |b|)."""
import numpy as np
import pytest
import torch

from paper_2604_19769_amd import binding as B
from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda:0"
TWO_PI = 8 * np.arctan(np.longdouble(1))


def rnd(seed, *shape, dtype="f32", by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * by).to(DT[dtype]).to(DEV)


def reference(x, pos, freq, interleaved=False, norm=False, weight=None, eps=1e-6, magnitude=1.0):
    """x [B][T][H][128], pos [B][T] -> (y, |a| + |b|) in 64 bits, written pair by pair."""
    x = x.double().cpu().numpy()
    if norm:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight.double().cpu().numpy()
    y, size = x.copy(), np.abs(x)
    half = len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        # 64 bits lose 1e-4 of the angle at a position of 2^40: the product and the whole turns in the 64-bit mantissa of a long double
        angle = np.mod(pos.astype(np.longdouble) * np.longdouble(freq[i]), TWO_PI).astype(np.float64)[:, :, None]
        c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = abs(magnitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def check(got, ref, what=""):
    want, size = ref
    u = torch.finfo(got.dtype).eps / 2
    lim = u * np.abs(want) + (1 + u) * 2.0 ** -19 * size + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= lim), f"{what}: {(err / np.maximum(lim, 1e-300)).max():.3g} times the tolerance"


@pytest.mark.parametrize("src,dst", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rotary,interleaved,norm", [(128, False, True), (128, True, False), (64, False, True), (96, True, True), (16, False, False),
                                                     (112, False, True), (0, False, True)])
def test_norm_rope(src, dst, rotary, interleaved, norm):
    Bn, T, Hq, Hkv = 3, 5, 12, 3
    q, k = rnd(1, Bn, T, Hq, 128, dtype=src), rnd(2, Bn, T, Hkv, 128, dtype=src, by=4.0)
    wq, wk = rnd(3, 128).abs() + 0.5, rnd(4, 128)
    freq = Rotary.frequencies(rotary, 10000.0)
    r = Rotary(freq, interleaved=interleaved, norm=norm, q_weight=wq, k_weight=wk, magnitude=1.25)
    first = [0, 77, 1000003]
    qo, ko = r.apply(q, k, first_pos=first, dtype=DT[dst])
    pos = np.array(first)[:, None] + np.arange(T)
    check(qo, reference(q, pos, freq, interleaved, norm, wq, magnitude=1.25), "q")
    check(ko, reference(k, pos, freq, interleaved, norm, wk, magnitude=1.25), "k")
    if not norm:
        assert torch.equal(qo[..., rotary:], q[..., rotary:].to(DT[dst]))          # channels that pass keep their values
    r.close()


@pytest.mark.parametrize("Bn,T,Hq,Hkv", [(1, 1, 1, 1), (64, 1, 8, 2), (2, 0, 4, 4), (1, 2, 9, 1), (5, 333, 28, 4), (1, 3000, 17, 17)])
def test_sizes(Bn, T, Hq, Hkv):
    x = rnd(5, Bn, T, Hq + 2 * Hkv, 128, dtype="bf16")
    freq = Rotary.frequencies(128, 500000.0)
    r = Rotary(freq, norm=(True, False))
    qo, ko = r.apply(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv])          # where a packed projection leaves them
    pos = np.broadcast_to(np.arange(T), (Bn, T))
    check(qo, reference(x[:, :, :Hq], pos, freq, norm=True))
    check(ko, reference(x[:, :, Hq:Hq + Hkv], pos, freq))
    r.close()


def test_layouts_positions_and_inputs_as_outputs():
    freq = Rotary.frequencies(64, 10000.0)
    r = Rotary(freq, interleaved=True)
    g = np.random.Generator(np.random.Philox(1))
    pos = g.integers(-5, 1 << 40, (3, 7))
    dpos = torch.from_numpy(pos).to(DEV)
    heads_first = rnd(6, 3, 5, 7, 128, dtype="f16").transpose(1, 2)                # stored [B][H][T][128]
    y, none = r.apply(heads_first, positions=dpos)
    assert none is None
    check(y, reference(heads_first, pos, freq, True), "heads first")
    one = rnd(7, 1, 7, 5, 128, dtype="f16").expand(3, 7, 5, 128)                   # every sequence the same rows
    none, y = r.apply(k=one, positions=dpos)
    check(y, reference(one, pos, freq, True), "expanded")
    wide = rnd(8, 3, 7, 5, 256, dtype="f16")
    x = wide[..., 128:]
    want, kept = reference(x, pos, freq, True), wide[..., :128].clone()
    y, _ = r.apply(x, positions=dpos, q_out=x)                                     # in place, rows 256 apart
    assert y.data_ptr() == x.data_ptr()
    check(x, want, "in place")
    assert torch.equal(wide[..., :128], kept)
    out = torch.full((3, 9, 6, 128), 7.0, dtype=torch.float16, device=DEV)         # into the middle of a larger tensor
    r.apply(heads_first, positions=dpos, q_out=out[:, 1:8, :5])
    check(out[:, 1:8, :5], reference(heads_first, pos, freq, True), "view")
    assert bool((out[:, 0] == 7).all() and (out[:, 8] == 7).all() and (out[:, :, 5] == 7).all())
    for bad in (x[..., :64], rnd(9, 3, 7, 5, 256)[..., ::2], wide[..., 4:132].double()):
        with pytest.raises((AssertionError, KeyError)):
            r.apply(bad)
    with pytest.raises(B.TTKVError):
        r.apply(wide[..., 4:132])                                                  # rows at multiples of 8 bytes
    r.close()


def test_values_that_are_not_numbers_stay_in_their_head_or_channel():
    freq = Rotary.frequencies(64, 10000.0)
    x = rnd(10, 1, 2, 4, 128)
    x[0, 0, 1, 100] = float("inf")                 # a channel that passes
    x[0, 1, 2, 3] = float("nan")                   # one that turns, with 35
    r = Rotary(freq)
    y, _ = r.apply(x)
    assert y[0, 0, 1, 100] == float("inf")
    bad = ~torch.isfinite(y)
    bad[0, 0, 1, 100] = False
    assert bad.nonzero().tolist() == [[0, 1, 2, 3], [0, 1, 2, 35]]
    n = Rotary(freq, norm=True)
    y, _ = n.apply(x)
    rows = torch.isfinite(y).all(-1)[0]
    assert rows.tolist() == [[True, False, True, True], [True, True, False, True]]
    z, _ = n.apply(torch.zeros(1, 1, 1, 128, device=DEV))
    assert bool((z == 0).all())                    # eps keeps a row of zeros
    r.close(), n.close()


# ---------------------------------------------------------------- append

def window(Bn, Hkv, dtype, bt, ring, paged=None, start=None, held=None, tiers=None, Hq=None):
    c = TieredCache(Bn, Hq or 2 * Hkv, Hkv, tiers or [TierConfig(dtype, dtype, 10 ** 9, bt, ring, paged_seed=paged)])
    c.pool[0].view(torch.int16).random_(-30000, 30000)          # what lies there already
    if start is not None:
        c.start[0][:] = start
    if held is not None:
        c.len[0][:] = held
    return c


def rows_of(c, b, lo, n):
    """(record, row) of tokens lo .. lo + n - 1 of sequence b's live ones in tier 0."""
    bt, ring = c.cfg[0].block_tokens, c.cfg[0].ring_blocks
    o = int(c.start[0][b]) + np.arange(lo, lo + n)
    r = o // bt % ring
    return (c.table[0][b][r] if c.table[0] is not None else b * ring + r), o % bt


@pytest.mark.parametrize("src,dst,paged", [("bf16", "bf16", 3), ("f16", "f16", None), ("f32", "bf16", 4), ("f32", "f16", None), ("bf16", "f16", 5)])
@pytest.mark.parametrize("bt,ring,T,held", [(64, 4, 1, 63), (64, 3, 100, 0), (128, 3, 257, 100), (256, 2, 13, 256)])
def test_append(src, dst, paged, bt, ring, T, held):
    Bn, Hq, Hkv = 4, 6, 3
    x = rnd(11, Bn, T, Hq + 2 * Hkv, 128, dtype=src)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    wk = rnd(12, 128)
    freq = Rotary.frequencies(128, 10000.0)
    r = Rotary(freq, norm=(False, True), k_weight=wk)
    start = [(b % ring) * bt for b in range(Bn)]                 # rings that wrap at different places
    counts = [T, 0, max(1, T // 3), T - 1 if T > 1 else 1]
    c = window(Bn, Hkv, dst, bt, ring, paged, start, held, Hq=Hq)
    before = c.pool[0].view(DT[dst]).view(-1, Hkv, 2, bt, 128).clone()
    q_out = torch.full((Bn, T, Hq, 128), 9.0, dtype=DT[dst], device=DEV)
    c.append_rotated(r, k, v, q=q, q_out=q_out, counts=counts)
    pool = c.pool[0].view(DT[dst]).view(-1, Hkv, 2, bt, 128)
    pos = held + np.broadcast_to(np.arange(T), (Bn, T))
    kr, qr = reference(k, pos, freq, norm=True, weight=wk), reference(q, pos, freq)
    left = torch.ones(pool.shape[0], bt, dtype=torch.bool)
    for b, n in enumerate(counts):
        assert c.len[0][b] == held + n
        rec, row = rows_of(c, b, held, n)
        left[rec, row] = False
        check(pool[rec, :, 0, row], [z[b, :n] for z in kr], f"keys of {b}")
        assert torch.equal(pool[rec, :, 1, row], v[b, :n].to(DT[dst])), f"values of {b}"
        check(q_out[b, :n], [z[b, :n] for z in qr], f"queries of {b}")
        assert bool((q_out[b, n:] == 9).all())
    same = (pool == before) | (torch.isnan(pool) & torch.isnan(before))
    assert bool(same.permute(0, 3, 1, 2, 4)[left.to(DEV)].all())  # every other row as it was
    r.close(), c.close()


def test_append_to_one_sequence_and_to_a_deeper_tier():
    tiers = [TierConfig("f16", "f16", 256, 64, 6), TierConfig("f16", "f16", 10 ** 9, 64, 6)]
    c = window(3, 2, "f16", 64, 6, tiers=tiers, held=7)
    c.len[1][:] = [64, 0, 128]
    freq = Rotary.frequencies(32)
    r = Rotary(freq)
    k, v = rnd(13, 1, 50, 2, 128, dtype="f16"), rnd(14, 1, 50, 2, 128, dtype="f16")
    assert c.append_rotated(r, k, v, seq=2) is None
    assert [x.tolist() for x in c.len] == [[7, 7, 57], [64, 0, 128]]
    pool = c.pool[0].view(torch.float16).view(-1, 2, 2, 64, 128)
    rec, row = rows_of(c, 2, 7, 50)
    check(pool[rec, :, 0, row], [z[0] for z in reference(k, 135 + np.arange(50)[None], freq)])      # behind all tiers' tokens
    c.append_rotated(r, k, v, seq=0, tier=1, first_pos=[11])
    pool = c.pool[1].view(torch.float16).view(-1, 2, 2, 64, 128)
    check(pool[1, :, 0, :50].transpose(0, 1), [z[0] for z in reference(k, 11 + np.arange(50)[None], freq)])
    with pytest.raises(B.TTKVError):
        c.append_rotated(r, rnd(15, 3, 400, 2, 128, dtype="f16"), rnd(15, 3, 400, 2, 128, dtype="f16"))
    assert [x.tolist() for x in c.len] == [[7, 7, 57], [114, 0, 128]]
    r.close(), c.close()


def test_captured_and_on_another_stream():
    freq = Rotary.frequencies(128)
    r = Rotary(freq, norm=True)
    x = rnd(16, 2, 3, 4, 128, dtype="bf16")
    out = torch.zeros_like(x)
    pos = torch.zeros(2, 3, dtype=torch.int64, device=DEV)
    r.apply(x, positions=pos, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.apply(x, positions=pos, q_out=out)
    for i in range(4):                                       # positions and inputs change between replays
        p = np.arange(6).reshape(2, 3) * (i + 1) + 100 * i
        pos.copy_(torch.from_numpy(p))
        x.copy_(rnd(20 + i, 2, 3, 4, 128, dtype="bf16"))
        graph.replay()
        torch.cuda.synchronize()
        check(out, reference(x, p, freq, norm=True), f"replay {i}")
        eager, _ = r.apply(x, positions=pos)
        assert torch.equal(eager, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, _ = r.apply(x, positions=pos)
    side.synchronize()
    assert torch.equal(y, out)
    r.close()


@pytest.mark.parametrize("rotary,interleaved", [(96, False), (64, False), (16, False), (96, True), (128, False)])
@pytest.mark.parametrize("src,dst", [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16")])
def test_appended_rows_are_those_of_apply(rotary, interleaved, src, dst):
    """Whatever way a row takes to its place: the tier's rows, outputs of their own and inputs as outputs hold the same bits."""
    n, Hq, Hkv = 70, 18, 9                                   # batches of eight heads with two and one in the last
    r = Rotary(Rotary.frequencies(rotary), interleaved=interleaved, norm=True)
    q, k, v = rnd(21, 2, n, Hq, 128, dtype=src), rnd(22, 2, n, Hkv, 128, dtype=src), rnd(23, 2, n, Hkv, 128, dtype=src)
    c = window(2, Hkv, dst, 64, 3, 5, [0, 64], 30, Hq=Hq)
    got = c.append_rotated(r, k, v, q=q)
    qo, ko = r.apply(q, k, first_pos=[30, 30], dtype=DT[dst])
    assert torch.equal(got, qo)
    pool = c.pool[0].view(DT[dst]).view(-1, Hkv, 2, 64, 128)
    for b in range(2):
        rec, row = rows_of(c, b, 30, n)
        assert torch.equal(pool[rec, :, 0, row], ko[b]) and torch.equal(pool[rec, :, 1, row], v[b].to(DT[dst]))
    if src == dst:
        r.apply(q, k, first_pos=[30, 30], q_out=q, k_out=k)
        assert torch.equal(q, qo) and torch.equal(k, ko)
    r.close(), c.close()
