"""What queries give each token of a tier, added up (64-bit definition), and the eviction of the lightest tokens (exact)."""
import math

import numpy as np
import pytest
import torch

from chunk_testlib import DEV, all_tokens, check, make_cache, quantized, rnd, tier_tokens
from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache

pytestmark = pytest.mark.gpu


def live(c, t, b):
    """Record and row of the live tokens of sequence b, oldest first."""
    bt, ring = c.cfg[t].block_tokens, c.cfg[t].ring_blocks
    o = int(c.start[t][b]) + np.arange(int(c.len[t][b]))
    r = (o // bt) % ring
    return torch.from_numpy(c.table[t][b][r].astype(np.int64) if c.table[t] is not None else b * ring + r).to(DEV), torch.from_numpy(o % bt).to(DEV)


def weights_of(c, t, b):
    rec, row = live(c, t, b)
    return c.weights[t][rec, :, row].t().contiguous()             # [Hkv][n]


def given(c, t, b, q, lse, part):
    """sum e^(scale q.k - lse) per token of the tier [Hkv][n], and how far it may be off: each term by its score's error (130 x 2^-24 of
    scale sum |q k|, the keys' parts where they are quantized, 2^-22 of the exponent's terms) and 2^-22 for the exponential, sums of n by (n / 16 + 64) 2^-24."""
    keys, _ = all_tokens(c, b)
    n, Hq = q.shape[:2]
    Hkv, total = keys.shape[:2]
    scale, G = float(c.c.softmax_scale), Hq // Hkv
    x = q.double().view(n, Hkv, G, 128).permute(1, 2, 0, 3).reshape(Hkv, G * n, 128)
    s = torch.bmm(x, keys.transpose(1, 2).contiguous()).view(Hkv, G, n, total) * scale
    big = torch.bmm(x.abs(), keys.abs().transpose(1, 2).contiguous()).view(Hkv, G, n, total) * scale
    hidden = torch.arange(total, device=DEV) > (total - n + torch.arange(n, device=DEV)).view(n, 1)
    l = lse.double().view(n, Hkv, G).permute(1, 2, 0).unsqueeze(-1)
    w = torch.exp(s - l).masked_fill(hidden | ~torch.isfinite(l), 0.0)
    u = (2.0 ** -21 if part == "f16" else 2.0 ** -16) if quantized(c) else 0.0
    off = big * (130 * 2.0 ** -24 + u) + (s.abs() + l.abs().nan_to_num(posinf=0.0)) * 2.0 ** -22 + 2.0 ** -22
    if u:
        off = off + scale * x.abs().sum(-1).view(Hkv, G, n, 1) * 2.0 ** -25
    rows = n * G
    lo = sum(int(c.len[i][b]) for i in range(t + 1, len(c.cfg)))
    if c.prefix is not None and (c.members is None or c.members[b]):
        lo += sum(int(x[0]) for x in c.prefix.len)
    hi = lo + int(c.len[t][b])
    return w.sum((1, 2))[:, lo:hi], ((w * off).sum((1, 2)) + w.sum((1, 2)) * (rows / 16 + 64) * 2.0 ** -24)[:, lo:hi]


def check_added(c, before, q, lse, counts, fresh, t=0, part=None):
    part = part or ("bf16" if c.cfg[t].k_fmt == "bf16" else "f16")
    for b in range(c.B):
        n = q.shape[1] if counts is None else int(counts[b])
        want, off = given(c, t, b, q[b, :n], lse[b, :n], part)
        newer = sum(int(c.len[i][b]) for i in range(t))
        old = before[b].double().clone()
        old[:, max(0, old.shape[1] - max(0, int(fresh[b]) - newer)):] = 0.0
        got = weights_of(c, t, b).double()
        err = (got - old - want).abs()
        assert (err <= off + (old + want) * 2.0 ** -23 + 1e-37).all(), (b, float(err.max()))


def start_weights(c, t=0):
    """Something in every live place; what lies elsewhere is no number."""
    for b in range(c.B):
        rec, row = live(c, t, b)
        c.weights[t][rec, :, row] = rnd(70 + b, len(rec), c.Hkv).float().abs()
    return [weights_of(c, t, b) for b in range(c.B)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2), (8, 2), (7, 1), (48, 3)])
@pytest.mark.parametrize("T,past", [(1, 0), (1, 64), (1, 500), (2, 255), (40, 0), (33, 300), (130, 70)])
def test_sizes(T, past, heads, dtype):
    c = make_cache(2, heads, [(dtype, [past + T, past + T])], weights=True)
    q = rnd(past, 2, T, heads[0], 128, dtype=dtype)
    _, lse = c.attend_chunk(q)
    before = start_weights(c)
    c.add_weights(q, lse, fresh=[T, 0])
    check_added(c, before, q, lse, None, [T, 0])
    rest = torch.ones_like(c.weights[0], dtype=torch.bool)
    for b in range(2):
        rec, row = live(c, 0, b)
        rest[rec, :, row] = False
    assert torch.isnan(c.weights[0][rest]).all()                  # nothing beside the live places
    total = sum(weights_of(c, 0, b).double().sum() for b in range(2)) - before[1].double().sum() - before[0][:, :past].double().sum()
    assert abs(float(total) / (2 * T * heads[0]) - 1) < 1e-4      # a query's weights make 1
    c.close()


@pytest.mark.parametrize("fmt", ["i8", "i4", "k8v4"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantized_keys(fmt, dtype):
    c = make_cache(2, (8, 2), [(fmt, [333, 65])], weights=True, paged=True)
    q = rnd(2, 2, 20, 8, 128, dtype=dtype)
    _, lse = c.attend_chunk(q)
    before = start_weights(c)
    c.add_weights(q, lse, fresh=[0, 65])
    check_added(c, before, q, lse, None, [0, 65], part=dtype)
    c.close()


@pytest.mark.parametrize("tier", [0, 1])
def test_tiers_and_prefix(tier):
    p = make_cache(1, (8, 2), [("f16", [130])], seed=40)
    c = make_cache(3, (8, 2), [("f16", [30, 100, 0]), ("i8", [200, 64, 128])], weights=True, prefix=p, members=[1, 0, 1])
    counts = [50, 20, 7]
    q = rnd(3, 3, 50, 8, 128)
    _, lse = c.attend_chunk(q, counts=counts)
    before = start_weights(c, tier)
    c.add_weights(q, lse, counts=counts, fresh=[40, 0, 10], tier=tier)
    check_added(c, before, q, lse, counts, [40, 0, 10], t=tier)
    c.close()
    p.close()


def test_counts_and_rows_that_give_nothing():
    """Sequences without queries; what lies behind a count or has no finite log-sum-exp is nothing; fresh places begin at 0 even then."""
    c = make_cache(4, (8, 2), [("f16", [100, 300, 70, 40])], weights=True)
    counts, fresh = [0, 30, 5, 0], [0, 10, 70, 40]
    q = rnd(3, 4, 30, 8, 128)
    _, lse = c.attend_chunk(q, counts=counts)
    lse[1, 3, 2], lse[1, 7, 5], lse[1, 9, 1] = -math.inf, math.inf, math.nan
    lse[2, 5:], q[2, 5:] = math.nan, math.nan
    before = start_weights(c)
    c.add_weights(q, lse, counts=counts, fresh=fresh)
    check_added(c, before, q, lse, counts, fresh)
    assert torch.equal(weights_of(c, 0, 0), before[0]) and not weights_of(c, 0, 3).any()
    c.close()


def test_step_after_step():
    """Decode steps: each adds its own weights, a new token begins at 0 although its place held another's before (the ring comes round)."""
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 256, 64, 6, weights=True), TierConfig("i8", "i8", 10 ** 9, 64, 9)])
    c.weights[0].fill_(float("nan"))
    k, v = rnd(1, 2, 2, 250, 128), rnd(2, 2, 2, 250, 128)
    c.append(0, k, v)
    q = rnd(3, 2, 8, 8, 128)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse)                                         # the last eight queries of the prompt; everything begins at 0
    want = {b: [weights_of(c, 0, b)[:, i].double() for i in range(250)] for b in range(2)}
    for step in range(150):
        q, kn, vn = rnd(10 + step, 2, 8, 128), rnd(600 + step, 2, 2, 1, 128), rnd(900 + step, 2, 2, 1, 128)
        out, lse = c.decode(q, new=(kn, vn))                      # (step() without its eviction: weights first)
        c.add_weights(q, lse)
        if step % 30 == 0 or step == 149:
            torch.cuda.synchronize()
        for b in range(2):
            if step in (0, 70, 149):
                now = weights_of(c, 0, b)
                assert torch.isfinite(now).all() and abs(float(now[:, -1].sum())) < 8.0
                assert now.shape[1] == c.len[0][b]
        c.demote()
    assert c.len[0][0] < 256 and c.len[1][0] > 0 and want
    c.close()


@pytest.mark.parametrize("fmt", ["f16", "bf16", "i8", "i4"])
@pytest.mark.parametrize("heads,T,lens", [((8, 8), 2, [70000, 100]), ((8, 4), 60, [17000, 300]), ((4, 1), 100, [300, 1000]), ((4, 4), 270, [17000, 1])])
def test_every_way_to_cut_it(fmt, heads, T, lens):
    """Few rows with several tiles of tokens to an item, a hundred rows, many rows that items share, many rows over many tokens."""
    dtype = "bf16" if fmt == "bf16" else "f16"
    c = make_cache(2, heads, [(fmt, lens)], weights=True, paged=True)
    q = rnd(2, 2, T, heads[0], 128, dtype=dtype)
    _, lse = c.attend_chunk(q)
    before = start_weights(c)
    c.add_weights(q, lse, fresh=[5, lens[1]])
    check_added(c, before, q, lse, None, [5, lens[1]], part=dtype)
    c.close()


def test_places_beyond_32_bits():
    c = make_cache(1, (8, 8), [("f16", [300])], spare=20000, weights=True)
    assert c.pool[0].numel() > 1 << 32
    for T in (3, 270):
        q = rnd(T, 1, T, 8, 128)
        _, lse = c.attend_chunk(q)
        before = start_weights(c)
        c.add_weights(q, lse, fresh=[0])
        check_added(c, before, q, lse, None, [0])
    evict_and_check(c, 100, 20)
    c.close()


def test_places_that_are_divided_for():
    c = make_cache(1, (2, 1), [("i4", [9000])], block=1 << 20, spare=8, weights=True)
    assert c.cfg[0].ring_blocks * 2 ** 20 // 64 * 2 ** 14 >= 1 << 31
    for T in (3, 270):
        q = rnd(T, 1, T, 2, 128)
        _, lse = c.attend_chunk(q)
        before = start_weights(c)
        c.add_weights(q, lse, fresh=[0])
        check_added(c, before, q, lse, None, [0])
    fill_weights(c, "plain")
    evict_and_check(c, 300, 20)
    c.close()


def test_tokens_that_were_taken_back():
    """Drafted tokens that were refused: those that come in their places begin at 0, also where a step brings them."""
    c = make_cache(1, (8, 2), [("f16", [100])], weights=True)
    q = rnd(1, 1, 8, 8, 128)
    _, lse = c.attend_chunk(q)
    c.add_weights(q, lse)
    for bring in ("append", "step"):
        c.len[0] -= 3
        before = [weights_of(c, 0, 0)]
        n = 4 if bring == "append" else 1
        k, v, q = rnd(2, 1, 2, n, 128), rnd(3, 1, 2, n, 128), rnd(4, 1, n, 8, 128)
        if bring == "append":
            c.append(0, k, v)
            _, lse = c.attend_chunk(q)
        else:
            _, lse = c.decode(q[:, 0].contiguous(), new=(k, v))
        before = [torch.cat([before[0], torch.full((2, n), 9.0, device=DEV)], 1)]
        c.add_weights(q, lse.view(1, n, 8))
        check_added(c, before, q, lse.view(1, n, 8), None, [n])
    c.close()


def test_two_streams_with_workspaces_that_grow():
    """Calls of two caches' kind at once: each stream has its own partial sums."""
    cs = [make_cache(1, (8, 2), [("f16", [n])], weights=True) for n in (600, 900)]
    cs[1]._streams_ws = cs[0]._streams_ws                         # one table of workspaces for both
    qs = [[rnd(10 * i + T, 1, T, 8, 128) for T in (70, 300, 100, 500)] for i in range(2)]
    lses = [[c.attend_chunk(q)[1].clone() for q in x] for c, x in zip(cs, qs)]
    want = []
    for c, x, ls in zip(cs, qs, lses):
        c.weights[0].zero_()
        for q, lse in zip(x, ls):
            c.add_weights(q, lse, fresh=[0])
        want.append(c.weights[0].clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c in cs:
            c.weights[0].zero_()
        torch.cuda.synchronize()
        for j in range(4):
            for c, x, ls, s in zip(cs, qs, lses, streams):
                with torch.cuda.stream(s):
                    c.add_weights(x[j], ls[j], fresh=[0])
        torch.cuda.synchronize()
        assert all(torch.equal(c.weights[0], w) for c, w in zip(cs, want))
    for c in cs:
        c.close()


# ------------------------------------------------------------------ eviction

def rows_of(c, t, b):
    """Per KV head the live rows' bytes [Hkv][n][all bytes], weights included as bits."""
    d = c.dump_tier(t, b)
    parts = [d[x] for x in ("k", "k_meta", "v", "v_meta") if d[x] is not None]
    w = weights_of(c, t, b).cpu().numpy().astype(np.float32).view(np.uint8).reshape(c.Hkv, -1, 4)
    return np.concatenate(parts + [w], -1)


def expected(rows, w, keep, recent, bt, swap):
    """One KV head's rows [n][bytes] after the eviction, and how many went: written from the header."""
    n = len(rows)
    gone = max(0, n - keep) // bt * bt
    if gone == 0:
        return rows, 0
    old = n - recent
    order = sorted(range(old), key=lambda i: (-math.inf if math.isnan(w[i]) else w[i] + 0.0, -i))   # lightest first, of equal ones the newest
    goes = set(order[:gone])
    src = [i for i in range(gone) if i not in goes]
    dst = [i for i in range(gone, old) if i in goes]
    assert len(src) == len(dst)
    new = rows.copy()
    for s, d in zip(src, dst):
        new[d] = rows[s]
        if swap:
            new[s] = rows[d]
    return (new, 0) if swap else (new[gone:], gone)


def evict_and_check(c, keep, recent, swap=False, t=0):
    before = [rows_of(c, t, b) for b in range(c.B)]
    w = [weights_of(c, t, b).cpu().numpy() for b in range(c.B)]
    start, length = c.start[t].copy(), c.len[t].copy()
    c.evict_light(keep, recent, tier=t, swap=swap)
    torch.cuda.synchronize()
    bt = c.cfg[t].block_tokens
    for b in range(c.B):
        want, gone = zip(*[expected(before[b][h], w[b][h].tolist(), keep, recent, bt, swap) for h in range(c.Hkv)])
        assert c.start[t][b] == start[b] + gone[0] and c.len[t][b] == length[b] - gone[0]
        got = rows_of(c, t, b)
        for h in range(c.Hkv):
            assert np.array_equal(got[h], want[h]), (b, h, np.flatnonzero((got[h] != want[h]).any(-1))[:5])


def fill_weights(c, kind, t=0):
    c.weights[t].fill_(-1e30)
    for b in range(c.B):
        rec, row = live(c, t, b)
        x = rnd(7 * b + 1, len(rec), c.Hkv).float()
        if kind == "ties":
            x = (x * 2).round()
        elif kind == "equal":
            x = torch.zeros_like(x)
        elif kind == "wild":
            x = torch.exp(20 * x)
            x[::7] = math.nan
            x[::11] = math.inf
            x[::13] = -math.inf
            x[::5] = -0.0
            x[1::5] = 0.0
        elif kind == "ordered":
            x = torch.arange(len(rec), device=DEV).float().unsqueeze(1).expand(-1, c.Hkv)
        elif kind == "backwards":
            x = -torch.arange(len(rec), device=DEV).float().unsqueeze(1).expand(-1, c.Hkv)
        c.weights[t][rec, :, row] = x


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "wild", "ordered", "backwards"])
@pytest.mark.parametrize("swap", [False, True])
@pytest.mark.parametrize("lens,keep,recent", [([64, 130, 700], 64, 0), ([64, 65, 128], 1, 1), ([1, 0, 300], 100, 37), ([300, 2500, 1100], 190, 190),
                                              ([4000, 63, 1500], 300, 20), ([128, 128, 128], 0, 0)])
def test_eviction(lens, keep, recent, swap, kind):
    c = make_cache(3, (4, 2), [("f16", lens)], weights=True, paged=True)
    fill_weights(c, kind)
    evict_and_check(c, keep, recent, swap)
    evict_and_check(c, keep, recent, swap)                        # nothing is left to do, or the same again
    c.close()


@pytest.mark.parametrize("fmt", ["bf16", "i8", "i4", "k8v4"])
@pytest.mark.parametrize("swap", [False, True])
def test_formats(fmt, swap):
    c = make_cache(2, (8, 4), [(fmt, [1000, 513])], weights=True, block=128)
    fill_weights(c, "plain")
    evict_and_check(c, 300, 50, swap)
    c.close()


def test_a_lower_tier():
    c = make_cache(2, (8, 2), [("f16", [100, 64]), ("i8", [700, 300])], weights=True)
    fill_weights(c, "plain", 1)
    evict_and_check(c, 200, 0, t=1)
    c.close()


def test_long_tier():
    """More tokens than a workgroup holds at once, blocks of 256."""
    c = make_cache(1, (2, 1), [("f16", [70000])], weights=True, block=256)
    fill_weights(c, "ties")
    evict_and_check(c, 3000, 256)
    c.close()


@pytest.mark.parametrize("lens", [[4160, 9000], [12345, 500], [31000, 4096], [32833, 64]])
@pytest.mark.parametrize("swap", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "wild"])
def test_lengths_that_waves_hold(lens, swap, kind):
    c = make_cache(2, (2, 1), [("i4", lens)], weights=True, paged=True)
    fill_weights(c, kind)
    evict_and_check(c, 2000, 65, swap)
    c.close()


def test_light_tokens_go_to_the_next_tier():
    """swap, then the FIFO cascade: the next tier receives the lightest tokens, the window keeps the others."""
    c = make_cache(2, (8, 2), [("f16", [256, 256]), ("i8", [64, 0])], weights=True, block=64, spare=6)
    c.c.tier[0].capacity_tokens = 128
    fill_weights(c, "plain")
    keys = [tier_tokens(c, 0, b)[0] for b in range(2)]
    w = [weights_of(c, 0, b) for b in range(2)]
    gone = 192                                                    # the cascade moves blocks while 128 or more are held
    c.evict_light(256 - gone, 16, swap=True)
    c.demote()
    torch.cuda.synchronize()
    assert (c.len[0] == 64).all() and c.len[1][0] == 64 + gone and (c.evicted == 0).all()
    for b in range(2):
        kept, _ = tier_tokens(c, 0, b)
        for h in range(2):
            heavy = torch.topk(w[b][h][:240], 48).indices.tolist() + list(range(240, 256))
            want = {keys[b][h][i].numpy().tobytes() for i in heavy}
            assert {x.numpy().tobytes() for x in kept[h]} == want
    c.close()


def test_captured_and_on_another_stream():
    c = make_cache(2, (8, 2), [("f16", [900, 500])], weights=True)
    q = rnd(1, 2, 3, 8, 128)
    _, lse = c.attend_chunk(q)
    fill_weights(c, "plain")
    first = c.weights[0].clone()
    pool = c.pool[0].clone()
    held = c.len[0].copy(), c.start[0].copy()

    def back():
        c.weights[0].copy_(first), c.pool[0].copy_(pool)
        c.len[0][:], c.start[0][:] = held
    c.add_weights(q, lse, fresh=[0, 0])
    c.evict_light(300, 40)
    torch.cuda.synchronize()
    want = c.weights[0].clone(), c.pool[0].clone()
    side = torch.cuda.Stream()
    back()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.add_weights(q, lse, fresh=[0, 0])
        c.evict_light(300, 40)
    side.synchronize()
    assert torch.equal(c.weights[0].nan_to_num(), want[0].nan_to_num()) and torch.equal(c.pool[0], want[1])
    back()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.add_weights(q, lse, fresh=[0, 0])
        c.evict_light(300, 40)
    for _ in range(3):
        back()
        c.attend_chunk(q)                                         # eager work beside it
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.weights[0].nan_to_num(), want[0].nan_to_num()) and torch.equal(c.pool[0], want[1])
    c.close()


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_prompt_in_chunks_then_steps(dtype):
    """A prompt comes in chunks through prefill, its last queries weigh its tokens, the lightest go, a few steps follow: every answer against
    the definition over what the cache holds, positions go on behind the dropped tokens."""
    c = TieredCache(2, 8, 2, [TierConfig(dtype, dtype, 10 ** 9, 64, 24, weights=True, paged_seed=4)])
    rotary = Rotary(Rotary.frequencies(128), norm=True)
    plain = Rotary(Rotary.frequencies(128), norm=True)
    pos = np.zeros(2, np.int64)
    for i, counts in enumerate(([300, 180], [1, 299], [300, 0], [77, 77])):
        T = max(counts)
        q, k, v = (rnd(20 * i + j, 2, T, h, 128, dtype=dtype) for j, h in enumerate((8, 2, 2)))
        out, lse = c.prefill(rotary, q, k, v, counts=counts)
        turned, _ = plain.apply(q, first_pos=pos)
        pos += counts
        assert (sum(c.len) == pos).all()
        torch.cuda.synchronize()
        check(c, turned, out, lse, counts=counts)
    c.add_weights(turned[:, -32:], lse[:, -32:].contiguous())
    for b in range(2):
        assert abs(float(weights_of(c, 0, b).sum()) / (32 * 8) - 1) < 1e-4
    evict_and_check(c, 200, 32)
    assert (c.evicted == pos - c.len[0]).all() and (c.len[0] >= 200).all() and (c.len[0] < 264).all()
    for i in range(3):
        q, k, v = (rnd(900 + 20 * i + j, 2, 1, h, 128, dtype=dtype) for j, h in enumerate((8, 2, 2)))
        out, lse = c.step_rotated(rotary, q, k, v)
        turned, _ = plain.apply(q, first_pos=pos)                 # behind all tokens of the lifetime, dropped ones too
        pos += 1
        torch.cuda.synchronize()
        chunk = c.attend_chunk(turned)
        check(c, turned, *chunk)
        assert (lse - chunk[1].view(2, 8)).abs().max() < 1e-3 and (out - chunk[0].view(2, 8, 128).float()).abs().max() < 2e-2
        c.add_weights(turned, lse)
    for b in range(2):
        assert torch.isfinite(weights_of(c, 0, b)).all()
    # a further chunk over the rearranged window
    q, k, v = (rnd(990 + j, 2, 40, h, 128, dtype=dtype) for j, h in enumerate((8, 2, 2)))
    out, lse = c.prefill(rotary, q, k, v)
    turned, _ = plain.apply(q, first_pos=pos)
    torch.cuda.synchronize()
    check(c, turned, out, lse)
    c.close()


def test_prefill_evicts_into_the_next_tier():
    c = TieredCache(2, 8, 2, [TierConfig("f16", "f16", 256, 64, 16), TierConfig("i8", "i8", 10 ** 9, 64, 40)])
    rotary = Rotary(Rotary.frequencies(128))
    for i, n in enumerate((500, 333, 90)):
        q, k, v = (rnd(20 * i + j, 2, n, h, 128) for j, h in enumerate((8, 2, 2)))
        held = c.len[0] + c.len[1]
        turned, _ = rotary.apply(q, first_pos=held)
        out, lse = c.prefill(rotary, q, k, v)
        assert (c.len[0] < 256).all() and (c.len[0] + c.len[1] == held + n).all()
        want_o, want_l = c.attend_chunk(turned)                   # the same tokens, some of them in int8 by now
        assert (lse - want_l).abs().max() < 0.05 and (out - want_o).abs().max() < 0.1
    c.close()
