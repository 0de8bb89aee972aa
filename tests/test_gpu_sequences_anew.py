"""A sequence's place in a batch that another one takes: its tokens' weights begin at 0 in every tier, its positions at 0 or right behind
the prefix."""
import pytest
import torch

from chunk_testlib import check, rnd
from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache
from test_gpu_token_weights import check_added, start_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("appended_first", [False, True])
@pytest.mark.parametrize("tiers", [2, 3])
def test_weights_of_a_lower_tier(tiers, appended_first):
    """Tokens that come down the cascade into places whose sequence has ended begin at 0, as those of a new place do: the tier ends earlier
    than it did before.  Weights of the sequence beside it stay."""
    cfg = [TierConfig("f16", "f16", 128, 64, 12), TierConfig("i8", "i8", 10 ** 9, 64, 20, weights=True)]
    if tiers == 3:
        cfg = [cfg[0], TierConfig("f16", "f16", 128, 64, 8), TierConfig("i8", "i8", 10 ** 9, 64, 20, weights=True)]
    low = tiers - 1
    c = TieredCache(2, 8, 2, cfg)
    c.append(0, rnd(1, 2, 2, 500, 128), rnd(2, 2, 2, 500, 128))
    c.demote()
    q = rnd(3, 2, 8, 8, 128)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse, tier=low)
    held = int(c.len[low][1])
    assert held >= 256
    c.weights[low] += 1000.0                                      # what the sequence that ends here had
    k, v = rnd(4, 2, 330, 128), rnd(5, 2, 330, 128)
    if appended_first:                                            # its older tokens end between the new ones' append and the cascade
        c.append(0, k, v, seq=1)
        for t in range(1, tiers):
            c.len[t][1] = 0
    else:
        for t in range(tiers):
            c.len[t][1] = 0
        c.append(0, k, v, seq=1)
    c.demote()
    newer = sum(int(x[1]) for x in c.len[:low])
    fresh = newer + int(c.len[low][1])
    assert 64 <= c.len[low][1] < held                             # below where the tier ended before
    before = start_weights(c, low)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse, tier=low)
    check_added(c, before, q, lse, None, [0, fresh], t=low, part="f16")
    c.close()


def rotated(seed, n, T):
    return (rnd(seed + i, n, T, h, 128) for i, h in enumerate((8, 2, 2)))


@pytest.mark.parametrize("way", ["lengths", "call"])
@pytest.mark.parametrize("first", ["prefill", "step"])
def test_positions_behind_a_prefix(first, way):
    """A sequence whose tokens were thinned out ends; the next one in its place begins right behind the prefix, the one beside it goes on."""
    p = TieredCache(1, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 6)])
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 9, weights=True)], prefix=p)
    rotary = Rotary(Rotary.frequencies(128))
    p.prefill(rotary, *rotated(1, 1, 100))
    q, k, v = rotated(4, 2, 300)
    _, lse = c.prefill(rotary, q, k, v)
    c.add_weights(rotary.apply(q, first_pos=[100, 100])[0], lse)
    c.evict_light(100, 20)
    assert (c.len[0] == 108).all() and (c.evicted == 192).all()
    if way == "call":
        c.begin_anew(1)
        assert c.evicted.tolist() == [192, 0]
    else:
        c.len[0][1] = 0
    assert c.len[0].tolist() == [108, 0]
    if first == "step":
        q, k, v = rotated(7, 2, 1)
        turned, _ = rotary.apply(q, first_pos=[400, 100])
        out, lse = c.step_rotated(rotary, q, k, v)
        torch.cuda.synchronize()
        o, l = c.attend_chunk(turned)
        # log-sum-exps: fp32 scores of 128 products, 130 x 2^-24 x 10 each; outputs: a half step of the chunk's weights and one of its result, values below 6
        assert (lse - l.view(2, 8)).abs().max() < 1.6e-4 and (out - o.view(2, 8, 128)).abs().max() < 2.0 ** -10 * 6
        check(c, turned, o, l)
    q, k, v = rotated(10, 2, 40)
    turned, _ = rotary.apply(q, first_pos=[401, 101] if first == "step" else [400, 100])
    out, lse = c.prefill(rotary, q, k, v)
    torch.cuda.synchronize()
    check(c, turned, out, lse)
    assert c.evicted.tolist() == [192, 0]
    c.close()
    p.close()


def test_a_prefix_that_begins_anew():
    """Another prompt in a prefix that was thinned out: the sequences' tokens come right behind it."""
    p = TieredCache(1, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 6, weights=True)])
    rotary = Rotary(Rotary.frequencies(128))
    q, k, v = rotated(1, 1, 300)
    _, lse = p.prefill(rotary, q, k, v)
    p.add_weights(rotary.apply(q)[0], lse)
    p.evict_light(100, 20)
    assert p.evicted[0] == 192
    for again in ("call", "lengths"):
        if again == "call":
            p.begin_anew()
        else:
            p.evict_light(64, 20)
            assert p.evicted[0] > 0
            p.len[0][:] = 0
        _, k, v = rotated(20, 1, 150)
        _, lse = p.prefill(rotary, q[:, :150].contiguous(), k, v)
        p.add_weights(rotary.apply(q[:, :150].contiguous())[0], lse)
        c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 6)], prefix=p, members=[True, False])
        qn, kn, vn = rotated(30, 2, 9)
        turned, _ = rotary.apply(qn, first_pos=[150, 0])
        out, lse = c.prefill(rotary, qn, kn, vn)
        torch.cuda.synchronize()
        check(c, turned, out, lse)
        c.close()
    p.close()


def test_every_tier_begins_anew():
    """begin_anew ends a sequence in all tiers, or all sequences; what comes then is answered as in a cache of its own."""
    tiers = [TierConfig("f16", "f16", 128, 64, 12, weights=True), TierConfig("i8", "i8", 10 ** 9, 64, 20, weights=True)]
    c = TieredCache(2, 8, 2, tiers)
    c.append(0, rnd(1, 2, 2, 500, 128), rnd(2, 2, 2, 500, 128))
    c.demote()
    q = rnd(3, 2, 8, 8, 128)
    held = [x.copy() for x in c.len]
    c.begin_anew(0)
    assert [x.tolist() for x in c.len] == [[0, int(x[1])] for x in held]
    _, lse = c.attend_chunk(q)
    assert torch.isinf(lse[0]).all() and torch.isfinite(lse[1]).all()
    c.begin_anew()
    assert not any(x.any() for x in c.len)
    c.append(0, rnd(5, 2, 2, 90, 128), rnd(6, 2, 2, 90, 128))
    out, lse = c.attend_chunk(q)
    torch.cuda.synchronize()
    check(c, q, out, lse)
    before = start_weights(c)
    c.add_weights(q, lse)
    check_added(c, before, q, lse, None, [90, 90])
    for bad in (-2, 2):
        with pytest.raises(AssertionError):
            c.begin_anew(bad)
    c.close()
