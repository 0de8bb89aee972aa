"""Attention of a chunk of new tokens over the tiers that hold it, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from chunk_testlib import DEV, DT, all_tokens, check, make_cache, rnd
from paper_2604_19769_amd import binding as B

pytestmark = pytest.mark.gpu


def attend(c, q, counts=None, seq=-1, dtype=None):
    n, T, Hq = q.shape[:3]
    out = torch.full((n, T, Hq, 128), 7.0, dtype=dtype or q.dtype, device=DEV)
    lse = torch.full((n, T, Hq), 7.0, device=DEV)
    got = c.attend_chunk(q, counts=counts, out=out, lse=lse, seq=seq)
    assert got[0] is out and got[1] is lse
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2), (4, 2), (8, 2), (7, 1), (48, 3)])
@pytest.mark.parametrize("T,past", [(1, 0), (1, 31), (2, 62), (3, 700), (7, 57), (16, 0), (31, 1), (33, 64), (40, 2500), (65, 63), (130, 0), (130, 333)])
def test_sizes(T, past, heads, dtype):
    c = make_cache(2, heads, [(dtype, [past + T, past + T])], seed=T)
    q = rnd(past, 2, T, heads[0], 128, dtype=dtype)
    check(c, q, *attend(c, q))
    c.close()


@pytest.mark.parametrize("dtype,block,paged", [("f16", 64, True), ("bf16", 128, True), ("f16", 256, False)])
@pytest.mark.parametrize("T,past", [(600, 0), (300, 1900), (5, 6000)])
def test_longer(T, past, dtype, block, paged):
    c = make_cache(1, (8, 2), [(dtype, [past + T])], block=block, paged=paged, k_by=2.0)
    q = rnd(3, 1, T, 8, 128, dtype=dtype)
    check(c, q, *attend(c, q))
    c.close()


@pytest.mark.parametrize("dtype,heads", [("f16", (8, 2)), ("bf16", (28, 4))])
@pytest.mark.parametrize("T,counts,past", [(6, [6, 0, 1, 5], [100, 40, 0, 900]), (50, [0, 50, 13, 1], [700, 3, 64, 0]),
                                           (200, [1, 200, 199, 77], [2000, 0, 31, 5]), (4, [0, 0, 0, 0], [9, 9, 9, 9])])
def test_padded_batches(T, counts, past, dtype, heads):
    c = make_cache(4, heads, [(dtype, [p + n for p, n in zip(past, counts)])], paged=True)
    q = rnd(5, 4, T, heads[0], 128, dtype=dtype)
    q[torch.arange(T, device=DEV) >= torch.tensor(counts, device=DEV).view(4, 1)] = float("nan")     # what lies behind a count is not read
    check(c, q, *attend(c, q, counts), counts=counts, untouched=7.0)
    c.close()


@pytest.mark.parametrize("older", ["i8", "i4", "k8v4"])
@pytest.mark.parametrize("dtype,T,new,old", [("f16", 3, [3, 70], [500, 0]), ("bf16", 3, [40, 3], [64, 130]), ("f16", 40, [41, 40], [200, 1]),
                                             ("bf16", 90, [300, 90], [33, 1111]), ("f16", 90, [100, 20], [0, 100]), ("f16", 4, [2, 0], [100, 300])])
def test_quantized_tiers(older, dtype, T, new, old):
    """The chunk in the first tier, in both or in the quantized one alone; tiers that hold nothing."""
    c = make_cache(2, (8, 2), [(dtype, new), (older, old)], block=128)
    q = rnd(9, 2, T, 8, 128, dtype=dtype)
    counts = [min(T, a + b) for a, b in zip(new, old)]
    check(c, q, *attend(c, q, counts), counts=counts, untouched=7.0)
    c.close()


@pytest.mark.parametrize("fmt", ["i8", "i4", "k8v4"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantized_tiers_alone(fmt, dtype):
    c = make_cache(2, (16, 4), [(fmt, [333, 65])], paged=True)
    q = rnd(2, 2, 20, 16, 128, dtype=dtype)
    check(c, q, *attend(c, q), part=dtype)
    c.close()


def test_four_tiers():
    c = make_cache(2, (8, 2), [("f16", [70, 10]), ("i8", [128, 0]), ("k8v4", [64, 200]), ("i4", [300, 31])])
    q = rnd(2, 2, 200, 8, 128)
    check(c, q, *attend(c, q))
    c.close()


@pytest.mark.parametrize("T", [2, 30, 100])
@pytest.mark.parametrize("fmts", [("f16", "f16"), ("f16", "i8"), ("bf16", "bf16"), ("i4", "f16")])
def test_prefixes(T, fmts):
    dtype = "bf16" if fmts[0] == "bf16" else "f16"
    p = make_cache(1, (8, 2), [(fmts[0], [150]), (fmts[1], [333])], seed=40)
    for members in (None, [True, False, True]):
        c = make_cache(3, (8, 2), [(dtype, [T, T + 5, 2 * T])], prefix=p, members=members)
        q = rnd(8, 3, T, 8, 128, dtype=dtype)
        check(c, q, *attend(c, q))
        c.close()
    p.close()


@pytest.mark.parametrize("T", [5, 100])
def test_queries_in_front_of_everything_see_nothing(T):
    """More queries than tokens: those in front of the oldest token are 0 with a log-sum-exp of minus infinity."""
    c = make_cache(2, (8, 2), [("f16", [3, 0])])
    q = rnd(1, 2, T, 8, 128)
    out, lse = attend(c, q)
    assert not out[0, :T - 3].any() and (lse[0, :T - 3] == -np.inf).all() and not out[1].any() and (lse[1] == -np.inf).all()
    assert torch.isfinite(lse[0, T - 3:]).all()
    keys, values = all_tokens(c, 0)
    s = (q[0, T - 3:].double().view(3, 2, 4, 128) @ keys.transpose(1, 2).unsqueeze(0)) * float(c.c.softmax_scale)
    s = s.masked_fill(torch.arange(3, device=DEV) > torch.arange(3, device=DEV).view(3, 1, 1, 1), -np.inf)
    want = torch.softmax(s, -1) @ values.unsqueeze(0)
    # three tokens: a half step of the weights, one of the result, and fp32's far below both
    assert ((out[0, T - 3:].double().view(3, 2, 4, 128) - want).abs() <= 2.0 ** -11 * (torch.softmax(s, -1) @ values.abs().unsqueeze(0) + want.abs()) + 1e-4).all()
    c.close()


@pytest.mark.parametrize("T", [3, 40, 150])
def test_views_and_types(T):
    """Queries where a packed projection left them, results of another type into rows of a wider tensor."""
    c = make_cache(2, (8, 2), [("f16", [T + 90, T + 10])])
    packed = rnd(4, 2, T, 12, 128, dtype="bf16")
    wide = torch.full((2, T + 3, 20, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    q, out = packed[:, :, 2:10], wide[:, 1:1 + T, 4:12]
    o, lse = c.attend_chunk(q, out=out)
    torch.cuda.synchronize()
    check(c, q, o, lse)
    rest = torch.ones_like(wide, dtype=torch.bool)
    rest[:, 1:1 + T, 4:12] = False
    assert (wide[rest] == 3.0).all()
    o16, _ = c.attend_chunk(q, dtype=torch.float16)
    assert o16.dtype == torch.float16
    check(c, q, o16, lse)
    heads_first = rnd(4, 2, 8, T, 128).transpose(1, 2)
    o, lse = c.attend_chunk(heads_first)
    check(c, heads_first, o, lse)
    c.close()


def test_one_sequence_of_a_batch():
    c = make_cache(3, (8, 2), [("f16", [200, 77, 300])])
    q = rnd(4, 1, 50, 8, 128)
    for b in range(3):
        check(c, q, *attend(c, q, seq=b), seqs=[b])
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [3, 20, 70, 200])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_wild_values_of_tokens_that_a_query_does_not_see(value, T, dtype):
    """An infinite (or no) number in the newer tokens' keys and values: older queries' rows keep every bit, the newer ones get it in its channel."""
    n = T + 70
    c = make_cache(1, (8, 2), [(dtype, [n])], wrap=False)
    q = rnd(6, 1, T, 8, 128, dtype=dtype)
    clean = attend(c, q)
    row = n - (T + 1) // 2                                        # seen by the queries from T - (n - row) on
    pool = c.pool[0].view(DT[dtype]).view(-1, 2, 2, 64, 128)
    pool[row // 64, 0, 1, row % 64, 17] = value
    wild = attend(c, q)
    seen = T - (n - row)
    assert torch.equal(wild[0][:, :seen], clean[0][:, :seen]) and torch.equal(wild[1], clean[1])
    assert torch.isnan(wild[0][:, seen:, :4, 17]).all() or torch.isinf(wild[0][:, seen:, :4, 17]).any()
    assert not torch.isfinite(wild[0][:, seen:, :4, 17]).any()
    others = torch.arange(128, device=DEV) != 17
    assert torch.equal(wild[0][:, :, :, others], clean[0][:, :, :, others]) and torch.equal(wild[0][:, :, 4:], clean[0][:, :, 4:])
    pool[row // 64, 0, 1, row % 64, 17] = 0.0
    before = attend(c, q)
    pool[row // 64, 1, 0, row % 64, 5] = float("nan")             # a key: scores that are no numbers
    wild = attend(c, q)
    assert torch.equal(wild[0][:, :seen], before[0][:, :seen]) and torch.equal(wild[1][:, :seen], before[1][:, :seen])
    assert torch.isnan(wild[0][:, seen:, 4:]).all() and torch.isnan(wild[1][:, seen:, 4:]).all()
    assert torch.equal(wild[0][:, :, :4], before[0][:, :, :4])
    c.close()


def test_a_query_that_is_no_number_spoils_its_own_row_only():
    c = make_cache(1, (8, 2), [("f16", [300])])
    q = rnd(6, 1, 90, 8, 128)
    clean = attend(c, q)
    q[0, 40, 3, 9] = float("nan")
    wild = attend(c, q)
    mine = torch.zeros(1, 90, 8, dtype=torch.bool, device=DEV)
    mine[0, 40, 3] = True
    assert torch.isnan(wild[0][mine]).all() and torch.isnan(wild[1][mine]).all()
    assert torch.equal(wild[0][~mine], clean[0][~mine]) and torch.equal(wild[1][~mine], clean[1][~mine])
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [4, 100])
def test_score_ranges(T, dtype):
    """Scores of thousands and of nearly nothing; one token with all the weight."""
    c = make_cache(1, (8, 2), [(dtype, [T + 300])])
    for by in (1e-4, 40.0, 600.0):
        q = rnd(6, 1, T, 8, 128, dtype=dtype, by=by)
        check(c, q, *attend(c, q))
    c.close()


def test_calls_on_two_streams_and_growing_workspaces():
    c = make_cache(1, (8, 2), [("f16", [4000])])
    sizes = [[3, 9, 2, 30], [16, 4, 40, 5]]
    qs = [[rnd(10 * i + j, 1, s, 8, 128) for j, s in enumerate(x)] for i, x in enumerate(sizes)]
    want = [[c.attend_chunk(q) for q in x] for x in qs]
    torch.cuda.synchronize()
    check(c, qs[0][0], *want[0][0])
    streams = [torch.cuda.Stream() for _ in sizes]
    for _ in range(5):
        got = [[], []]
        for j in range(4):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    got[i].append(c.attend_chunk(qs[i][j]))
        torch.cuda.synchronize()
        for i in range(2):
            for j in range(4):
                assert torch.equal(got[i][j][0], want[i][j][0]) and torch.equal(got[i][j][1], want[i][j][1]), (i, j)
    c.close()


def test_captured_calls():
    c = make_cache(2, (8, 2), [("f16", [3000, 900])])
    a, b = rnd(1, 2, 4, 8, 128), rnd(2, 2, 30, 8, 128)
    want = [[x.clone() for x in c.attend_chunk(q)] for q in (a, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for q in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(c.attend_chunk(q))
        graphs.append(g)
    for i in range(4):
        for o, l in outs:
            o.fill_(0), l.fill_(0)
        for g in (graphs if i % 2 else graphs[::-1]):
            g.replay()
        c.attend_chunk(rnd(5, 2, 50, 8, 128))                     # eager work beside them
        torch.cuda.synchronize()
        for (o, l), (wo, wl) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(l, wl)
    c.close()


def test_another_current_stream_than_the_tensors_own():
    c = make_cache(1, (8, 2), [("f16", [2000])])
    q = rnd(1, 1, 6, 8, 128)
    want = c.attend_chunk(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.attend_chunk(q)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.close()


def test_a_refused_chunk_leaves_the_cache_as_it_was():
    from paper_2604_19769_amd.cache import Rotary
    c = make_cache(2, (8, 2), [("f16", [100, 50]), ("i8", [64, 0])], spare=2)
    rotary = Rotary(Rotary.frequencies(128))
    q, k, v = rnd(1, 2, 60, 8, 128), rnd(2, 2, 60, 2, 128), rnd(3, 2, 60, 2, 128)
    held = c.len[0].copy()
    with pytest.raises(B.TTKVError) as e:
        c.prefill(rotary, q, k, v, dtype=torch.float32)           # results are 16 bits wide
    assert e.value.status == B.ERR_UNSUPPORTED and (c.len[0] == held).all()
    c.close()


@pytest.mark.parametrize("T", [3, 30, 100])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_format_at_once(T, dtype):
    """All quantized formats in one call, some of them a prefix's."""
    p = make_cache(1, (8, 2), [("i4", [100]), ("k8v4", [65])], seed=40)
    c = make_cache(3, (8, 2), [(dtype, [T, 1, 70]), ("i8", [0, T, 300]), ("i4", [200, 0, 31])], prefix=p, members=[1, 0, 1], paged=True)
    q = rnd(4, 3, T, 8, 128, dtype=dtype)
    counts = [T, T, T - 1]
    check(c, q, *attend(c, q, counts), counts=counts, untouched=7.0)
    c.close()
    p.close()


def test_places_beyond_32_bits():
    """Rows of the pool, of the queries and of the results more than 4 GiB apart; a run that begins at the pool's end."""
    c = make_cache(1, (8, 8), [("f16", [300])], spare=20000)
    assert c.pool[0].numel() > 1 << 32
    far = torch.empty(2, 2 ** 31 + 1024, dtype=torch.float16, device=DEV)
    few, many = rnd(1, 1, 3, 8, 128), rnd(2, 1, 270, 8, 128)
    for q in (few, many):
        check(c, q, *attend(c, q))
    c.close()
    c = make_cache(2, (8, 2), [("f16", [300, 200])])
    for T in (3, 100):
        n = T * 8 * 128
        q, out = far[:, :n].view(2, T, 8, 128), far[:, n:2 * n].view(2, T, 8, 128)
        q.copy_(rnd(3, 2, T, 8, 128))
        o, lse = c.attend_chunk(q, out=out)
        check(c, q, o, lse)
    c.close()


def test_blocks_that_are_divided_by():
    """Rings so long, blocks so large that places are found by a division."""
    c = make_cache(1, (2, 1), [("i4", [9000])], block=1 << 20, spare=8)
    assert c.cfg[0].ring_blocks * 2 ** 20 // 64 * 2 ** 14 >= 1 << 31
    for T in (2, 200):
        q = rnd(T, 1, T, 2, 128)
        check(c, q, *attend(c, q))
    c.close()


def test_positions_behind_a_prefix_that_was_thinned_out():
    from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache
    p = TieredCache(1, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 6, weights=True)])
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 10 ** 9, 64, 6)], prefix=p, members=[True, False])
    rotary = Rotary(Rotary.frequencies(128))
    q, k, v = rnd(1, 1, 300, 8, 128), rnd(2, 1, 300, 2, 128), rnd(3, 1, 300, 2, 128)
    _, lse = p.prefill(rotary, q, k, v)
    p.add_weights(rotary.apply(q)[0], lse)
    p.evict_light(100, 20)
    assert p.len[0][0] == 108 and p.evicted[0] == 192
    q, k, v = rnd(4, 2, 9, 8, 128), rnd(5, 2, 9, 2, 128), rnd(6, 2, 9, 2, 128)
    turned, _ = rotary.apply(q, first_pos=[300, 0])
    out, lse = c.prefill(rotary, q, k, v)
    torch.cuda.synchronize()
    check(c, turned, out, lse)
    c.close()
    p.close()


@pytest.mark.parametrize("fmt,codes,group", [("i8", 128, 32), ("i4", 64, 64)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [3, 20, 70, 200])
def test_wild_scales_of_tokens_that_a_query_does_not_see(fmt, codes, group, dtype, T):
    """A value scale that is no number in a quantized tier's newer token: as above, in the channels of its group."""
    n = T + 70
    c = make_cache(1, (8, 2), [(fmt, [n])], wrap=False)
    q = rnd(6, 1, T, 8, 128, dtype=dtype)
    clean = attend(c, q)
    row = n - (T + 1) // 2
    at = (row // 64 * 2 + 1) * 64 * (2 * codes + 16) + 64 * (2 * codes + 8) + row % 64 * 8   # KV head 1, the row's first value scale
    c.pool[0].view(-1)[at:at + 2] = 255
    wild = attend(c, q)
    seen = T - (n - row)
    assert torch.equal(wild[0][:, :seen], clean[0][:, :seen]) and torch.equal(wild[1], clean[1])
    assert torch.isnan(wild[0][:, seen:, 4:, :group]).all()
    assert torch.equal(wild[0][:, :, 4:, group:], clean[0][:, :, 4:, group:]) and torch.equal(wild[0][:, :, :4], clean[0][:, :, :4])
    c.close()


@pytest.mark.parametrize("T", [20, 70])
def test_wild_values_behind_a_quantized_tier(T):
    """The step where a tier ends, and the fp tier behind it, whose first token nobody but the newest query sees."""
    c = make_cache(1, (8, 2), [("f16", [1]), ("i8", [T + 44])], wrap=False)
    q = rnd(6, 1, T, 8, 128)
    clean = attend(c, q)
    c.pool[0].view(torch.float16).view(-1, 2, 2, 64, 128)[0, 1, 1, 0, 100] = float("inf")
    wild = attend(c, q)
    assert torch.equal(wild[0][:, :-1], clean[0][:, :-1]) and torch.equal(wild[1], clean[1])
    assert not torch.isfinite(wild[0][:, -1, 4:, 100]).any()
    others = torch.arange(128, device=DEV) != 100
    assert torch.equal(wild[0][..., others], clean[0][..., others])
    c.close()
