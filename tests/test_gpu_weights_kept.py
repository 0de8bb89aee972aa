"""What TieredCache knows of its tokens' weights: which have been weighed, and what a step adds to which."""
import pytest
import torch

from chunk_testlib import make_cache, rnd
from paper_2604_19769_amd import binding as B
from paper_2604_19769_amd.cache import TierConfig, TieredCache
from test_gpu_token_weights import check_added, evict_and_check, live, weights_of

pytestmark = pytest.mark.gpu


def refused(c, keep, recent, **kw):
    held = [x.copy() for x in c.len], [x.copy() for x in c.start], c.evicted.copy()
    with pytest.raises(B.TTKVError) as e:
        c.evict_light(keep, recent, **kw)
    assert e.value.status == B.ERR_INVALID_ARG
    assert all((a == b).all() for x, y in zip(held[:2], (c.len, c.start)) for a, b in zip(x, y)) and (held[2] == c.evicted).all()


@pytest.mark.parametrize("stale", [0.0, 1e6])
def test_tokens_that_were_never_weighed(stale):
    """Tokens behind the last that add_weights has seen have to be among the recent ones, where a sequence loses blocks."""
    c = make_cache(2, (8, 2), [("f16", [400, 100])], weights=True, spare=4)
    q = rnd(1, 2, 8, 8, 128)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse)
    rec = c.weights[0].clone()
    c.weights[0][torch.isnan(rec)] = stale                        # what the places of tokens to come hold
    c.append(0, rnd(2, 2, 50, 128), rnd(3, 2, 50, 128), seq=0)
    for swap in (False, True):
        refused(c, 200, 49, swap=swap)
        refused(c, 64, 0, swap=swap)
    c.evict_light(440, 0)                                         # no block goes: nothing is decided
    assert c.len[0].tolist() == [450, 100]
    c.len[0][0] -= 20                                             # taken back: 30 are left
    refused(c, 200, 29)
    evict_and_check(c, 200, 30)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse)
    evict_and_check(c, 64, 0)
    c.close()


def test_one_sequence_weighed():
    c = make_cache(2, (8, 2), [("f16", [300, 300])], weights=True)
    q = rnd(1, 1, 8, 8, 128)
    _, lse = c.attend_chunk(q, seq=0)
    c.add_weights(q, lse, seq=0)
    refused(c, 100, 20)
    _, lse = c.attend_chunk(q, seq=1)
    c.add_weights(q, lse, seq=1)
    evict_and_check(c, 100, 20)
    c.close()


def test_tokens_that_came_down():
    """The cascade's tokens in a lower tier that is weighed."""
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 128, 64, 12), TierConfig("i8", "i8", 10 ** 9, 64, 20, weights=True)])
    q = rnd(3, 2, 8, 8, 128)
    for n in (500, 200):
        c.append(0, rnd(n, 2, 2, n, 128), rnd(n + 1, 2, 2, n, 128))
        c.demote()
        if n == 500:
            _, lse = c.attend_chunk(q)
            c.add_weights(q, lse, tier=1)
    came = int(c.len[1][0]) - 384
    assert came > 0
    refused(c, 256, came - 1, tier=1)
    evict_and_check(c, 256, came, t=1)
    c.close()


def test_every_step_adds_its_own():
    """Decode steps whose window wraps around its ring and whose cascade fills the tier behind it: in both tiers each step adds what its queries
    give to what was there, and a token that came since the last call begins at 0 whatever its place holds.  (The rest of the log-sum-exp
    is the other tier's, so the weights of both make 1 per query.)"""
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 256, 64, 6, weights=True), TierConfig("i8", "i8", 10 ** 9, 64, 9, weights=True)])
    k, v = rnd(1, 2, 2, 250, 128), rnd(2, 2, 2, 250, 128)
    c.append(0, k, v)
    for w in c.weights:
        w.fill_(1e4)
    q = rnd(3, 2, 8, 8, 128)
    _, lse = c.attend_chunk(q)
    seen = [[int(c.start[t][b] + c.len[t][b]) for b in range(2)] for t in range(2)]

    def weigh(q, lse, fresh):
        for t in range(2):
            newer = [sum(int(c.len[i][b]) for i in range(t)) for b in range(2)]
            want = [f + n for f, n in zip(fresh[t], newer)]
            before = [weights_of(c, t, b) for b in range(2)]
            c.add_weights(q, lse, tier=t)
            check_added(c, before, q, lse, None, want, t=t, part="f16")
    weigh(q, lse, [[250, 250], [0, 0]])
    for step in range(150):
        q, kn, vn = rnd(10 + step, 2, 8, 128), rnd(600 + step, 2, 2, 1, 128), rnd(900 + step, 2, 2, 1, 128)
        _, lse = c.decode(q, new=(kn, vn))
        for b in range(2):                                        # (what was there of another token)
            rec, row = live(c, 0, b)
            c.weights[0][rec[-1], :, row[-1]] = 1e4
        fresh = [[int(c.start[t][b] + c.len[t][b]) - seen[t][b] for b in range(2)] for t in range(2)]
        assert fresh[0] == [1, 1] and fresh[1] in ([0, 0], [64, 64])
        total = sum(float(weights_of(c, t, b)[:, :-1 if t == 0 else None].double().sum()) for t in range(2) for b in range(2)) - \
            sum(float(weights_of(c, 1, b)[:, c.len[1][b] - fresh[1][b]:].double().sum()) for b in range(2))
        weigh(q.unsqueeze(1), lse.view(2, 1, 8), fresh)
        now = sum(float(weights_of(c, t, b).double().sum()) for t in range(2) for b in range(2))
        assert abs((now - total) / 16 - 1) < 1e-3                 # sums of some thousands, fp32 places
        seen = [[int(c.start[t][b] + c.len[t][b]) for b in range(2)] for t in range(2)]
        c.demote()
    assert c.start[0][0] + c.len[0][0] > 384 and c.len[1][0] >= 192
    c.close()
