"""A sequence's place in a batch that another one takes: its tokens' weights begin at 0 in every tier."""
import pytest
import torch

from chunk_testlib import rnd
from paper_2604_19769_amd.cache import TierConfig, TieredCache
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
