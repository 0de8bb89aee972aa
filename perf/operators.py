"""Timing cases of the operators between a model's projections and the tiered decode attention:

  rotate   norm of queries and keys per head and position rotation, in one pass
  append   keys (normed and rotated on the way) and values appended to the paged window, the queries beside them
  shared   attention of a batch over a prefix that all its sequences share
  step     one decode step of a batch with a shared prefix: the token appended, prefix and own window attended

With `own` the calls are the framework's; without, the same mathematics in elementary torch operations, in 32 bits
(angles in 64).  A window is a pool of records [record][KV head][K or V][block token][128], found through a shuffled
block table where it is paged."""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
SCALE = 1.0 / math.sqrt(128.0)
BASE = 500000.0
EPS = 1e-6


def listed():
    def rope(name, kind, batch, tokens, heads, src, dst, rotary, interleaved, norm, far, ragged=1.0, block=128, paged=False):
        return {"name": name, "kind": kind, "batch": batch, "tokens": tokens, "q_heads": heads[0], "kv_heads": heads[1], "src": src,
                "dst": dst, "rotary": rotary, "interleaved": interleaved, "norm": norm, "far": far, "ragged": ragged, "block": block,
                "paged": paged}

    def attend(name, kind, batch, heads, dtype, prefix, window=0, ragged=1.0, block=128, paged=False):
        return {"name": name, "kind": kind, "batch": batch, "q_heads": heads[0], "kv_heads": heads[1], "src": dtype, "dst": dtype,
                "prefix": prefix, "window": window, "ragged": ragged, "block": block, "paged": paged}

    return [
        # one token of one conversation on a small model: launch and host time
        rope("rotate_one_token", "rotate", 1, 1, (8, 2), "bf16", "bf16", 128, False, True, 4096),
        # two prompts of a grouped-query model with normed heads, q and k where the packed projection left them
        rope("rotate_prompts", "rotate", 2, 4096, (32, 8), "bf16", "bf16", 128, False, True, 0),
        # half of the channels turn, pairs side by side, projections kept in 32 bits; odd lengths
        rope("rotate_partial_f32", "rotate", 3, 1021, (28, 4), "f32", "f32", 64, True, False, 130000),
        # a decode step of a full batch into paged windows, with its queries
        rope("append_step_x64", "append", 64, 1, (32, 8), "bf16", "bf16", 128, False, True, 9000, block=128, paged=True),
        # a padded batch of prompts of unequal length into pages of 256 tokens
        rope("append_ragged_prompts", "append", 7, 4999, (32, 8), "f16", "f16", 128, False, True, 0, ragged=0.3, block=256, paged=True),
        # a multi-head model's prompt, projections in 32 bits
        rope("append_mha_f32", "append", 1, 6000, (32, 32), "f32", "bf16", 96, False, False, 70000),
        # two short answers to one question: the smallest call
        attend("shared_two", "shared", 2, (8, 2), "f16", 1000),
        # a full batch behind one long document, grouped-query: 256 rows per KV head
        attend("shared_gqa_x64", "shared", 64, (32, 8), "f16", 32768),
        # a multi-head model's system prompt: the bytes of 32 KV heads against 24 rows each; odd length
        attend("shared_mha_x24", "shared", 24, (32, 32), "bf16", 8229),
        # a few sequences behind a very long document
        attend("shared_long_x5", "shared", 5, (28, 4), "bf16", 131072, block=256, paged=True),
        # one decode step of 48 conversations behind one prompt
        attend("step_prefix_x48", "step", 48, (32, 8), "f16", 16384, 1003, ragged=0.4, paged=True),
        # a few conversations of a bf16 model early on: windows of a handful of tokens behind a short prompt
        attend("step_prefix_x9", "step", 9, (16, 4), "bf16", 2003, 45, ragged=0.2, block=64),
    ]


HEADS = ((8, 2), (16, 16), (32, 32), (32, 16), (24, 8), (32, 8), (48, 8), (64, 8), (28, 4), (64, 4))


def draw(rng: random.Random):
    while True:
        kind = rng.choice(("rotate", "append", "append", "shared", "shared", "step"))
        hq, hkv = rng.choice(HEADS)
        if kind in ("rotate", "append"):
            batch = round(2 ** rng.uniform(0, 6))
            tokens = 1 if rng.random() < 0.3 else round(2 ** rng.uniform(1, 13))
            dst = rng.choice(("f16", "bf16", "f32") if kind == "rotate" else ("f16", "bf16"))
            case = {"kind": kind, "batch": batch, "tokens": tokens, "q_heads": hq, "kv_heads": hkv, "src": rng.choice((dst, dst, "f32")), "dst": dst,
                    "rotary": rng.choice((32, 64, 96, 128, 128, 128)), "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.6,
                    "far": round(2 ** rng.uniform(0, 18)), "ragged": 1.0 if kind == "rotate" or tokens == 1 else rng.choice((1.0, 0.5, 0.1)),
                    "block": rng.choice((64, 128, 256)), "paged": kind == "append" and rng.random() < 0.5}
            if batch * tokens <= 36000 and work(case)["bytes"] <= 4.4e8:
                return case
            continue
        dtype = rng.choice(("f16", "bf16"))
        case = {"kind": kind, "batch": round(2 ** rng.uniform(0, 6)), "q_heads": hq, "kv_heads": hkv, "src": dtype, "dst": dtype,
                "prefix": round(2 ** rng.uniform(7, 17)), "window": 0 if kind == "shared" else round(2 ** rng.uniform(0, 11)),
                "ragged": rng.choice((1.0, 0.5, 0.2)), "block": rng.choice((64, 128, 256)), "paged": rng.random() < 0.5}
        w = work(case)
        if w["flops"] <= 3.4e10 and w["bytes"] <= 4.4e8:
            return case


# ------------------------------------------------------------------ shapes

def counts(case):
    """Tokens that each sequence of a padded batch brings (append) or holds in its window (step)."""
    n = case["tokens"] if case["kind"] == "append" else case["window"]
    return [max(1, int(n * (case["ragged"] + (1.0 - case["ragged"]) * ((b * 0.6180339887 + 1.0) % 1.0)))) if b else n
            for b in range(case["batch"])]


def rings(case):
    """Tokens held before, first lifetime ordinal and blocks of a sequence's ring: a window that has been running."""
    bt = case["block"]
    held = [0] * case["batch"] if case["kind"] == "append" and case["tokens"] > 1 else counts(case)
    if case["kind"] == "append" and case["tokens"] == 1:
        held = [37 + 19 * b for b in range(case["batch"])]
    most = max(held) + (case["tokens"] if case["kind"] == "append" else 1)
    blocks = -(-most // bt) + 1
    return held, [(3 + 7 * b) % blocks * bt for b in range(case["batch"])], blocks


def work(case):
    B, hq, hkv, dst, src = case["batch"], case["q_heads"], case["kv_heads"], SIZE[case["dst"]], SIZE[case["src"]]
    if case["kind"] == "rotate":
        n = B * case["tokens"] * (hq + hkv) * 128
        return {"bytes": n * (src + dst), "flops": n * 8}
    if case["kind"] == "append":
        n = sum(counts(case)) * 128
        return {"bytes": n * (hq + 2 * hkv) * (src + dst), "flops": n * (hq + hkv) * 8}
    tokens, flops = case["prefix"], 4 * 128 * case["prefix"] * B * hq
    extra = B * hq * (128 * (src + 4) + 4)
    if case["kind"] != "shared":
        tokens += sum(counts(case))
        flops += 4 * 128 * sum(n + 1 for n in counts(case)) * hq
        extra += B * hkv * 128 * 2 * (src + dst)
    return {"bytes": tokens * hkv * 256 * dst + extra, "flops": flops}


# ------------------------------------------------------------------ inputs

def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def inputs(case, seed):
    """Everything that both forms and the exact one start from, drawn in one order."""
    B, hq, hkv, bt = case["batch"], case["q_heads"], case["kv_heads"], case["block"]
    g = generator(seed)
    src, dst = DT[case["src"]], DT[case["dst"]]

    def normal(shape, dtype, by=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * by).to(dtype)

    x = {}
    loud = torch.ones(hkv * 128, device=DEV)          # every 50th (head, channel) pair of the keys is large, as in trained models
    loud[torch.randperm(hkv * 128, generator=g, device=DEV)[:max(1, hkv * 128 // 50)]] = 8.0
    if case["kind"] in ("rotate", "append"):
        T = case["tokens"]
        scale = torch.cat((torch.ones(hq * 128, device=DEV), loud, torch.ones(hkv * 128, device=DEV)))
        x["qkv"] = normal((B, T, (hq + 2 * hkv) * 128), src, scale).view(B, T, hq + 2 * hkv, 128)
        if case["norm"]:
            x["q_weight"], x["k_weight"] = (1.0 + 0.1 * torch.randn(128, generator=g, device=DEV) for _ in range(2))
    if case["kind"] in ("shared", "step"):
        x["q"] = normal((B, hq, 128), src)
    if case["kind"] == "step":
        x["k_new"], x["v_new"] = normal((B, hkv, 1, 128), dst, loud.view(hkv, 1, 128)), normal((B, hkv, 1, 128), dst)
    if case["kind"] in ("shared", "step"):
        x["pk"], x["pv"] = normal((hkv, case["prefix"], 128), dst, loud.view(hkv, 1, 128)), normal((hkv, case["prefix"], 128), dst)
    if case["kind"] in ("append", "step"):
        held, first, blocks = rings(case)
        table = np.arange(B * blocks).reshape(B, blocks)
        if case["paged"]:
            table = np.random.Generator(np.random.Philox(7)).permutation(B * blocks).reshape(B, blocks)
        pool = normal((B * blocks, hkv, 2, bt, 128), dst)
        pool[:, :, 0] *= loud.view(hkv, 1, 128).to(dst)
        x.update(pool=pool, held=held, first=first, blocks=blocks, table=table)
    return x


def frequencies(rotary):
    return BASE ** (-np.arange(0, rotary, 2, dtype=np.float64) / rotary)


def positions(case):
    """Position of each sequence's first token."""
    return [case["far"] + 31 * b for b in range(case["batch"])]


def places(x, B, bt, first, n):
    """Record and row of tokens first[b] .. first[b] + n - 1 (lifetime ordinals) of each sequence: [B][n] each."""
    o = torch.as_tensor(first, device=DEV).view(B, 1) + torch.arange(n, device=DEV)
    ring = (o // bt) % x["blocks"]
    return torch.as_tensor(x["table"], device=DEV).gather(1, ring), o % bt


def prepare(case, seed):
    B, hq, hkv, bt, kind = case["batch"], case["q_heads"], case["kv_heads"], case["block"], case["kind"]
    x = inputs(case, seed)
    state = {"case": case, "x": x}
    if kind in ("rotate", "append"):
        T, qkv = case["tokens"], x["qkv"]
        x["q_in"], x["k_in"], x["v_in"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        freq = frequencies(case["rotary"])
        first = positions(case)
        state["first_pos"] = np.array(first, np.int64)
        state["q_out"] = torch.empty(B, T, hq, 128, dtype=DT[case["dst"]], device=DEV)
        state["k_out"] = torch.empty(B, T, hkv, 128, dtype=DT[case["dst"]], device=DEV)
        state["freq"], state["pos"] = torch.from_numpy(freq).to(DEV), torch.tensor(first, device=DEV).view(B, 1) + torch.arange(T, device=DEV)
    if kind == "append":
        n = counts(case)
        state["counts"] = np.array(n, np.int64) if len(set(n)) > 1 else None
        state["real"] = torch.arange(case["tokens"], device=DEV) < torch.tensor(n, device=DEV).view(B, 1)
        state["rows"] = places(x, B, bt, [f + h for f, h in zip(x["first"], x["held"])], case["tokens"])
        state["q_out"].zero_()
    if kind == "step":
        state["window"] = places(x, B, bt, x["first"], max(x["held"]) + 1)
        state["seen"] = torch.arange(max(x["held"]) + 1, device=DEV) <= torch.tensor(x["held"], device=DEV).view(B, 1)
        state["rows"] = places(x, B, bt, [f + h for f, h in zip(x["first"], x["held"])], 1)
        state["real"] = torch.ones(B, 1, dtype=torch.bool, device=DEV)
    if own:
        from paper_2604_19769_amd.cache import Rotary, TierConfig, TieredCache
        if kind in ("rotate", "append"):
            state["rotary"] = Rotary(freq, interleaved=case["interleaved"], norm=case["norm"], q_weight=x.get("q_weight"),
                                     k_weight=x.get("k_weight"), eps=EPS)
        prefix = None
        if "pk" in x:
            blocks = -(-case["prefix"] // bt)
            prefix = TieredCache(1, hq, hkv, [TierConfig(case["dst"], case["dst"], 10 ** 9, bt, blocks, paged_seed=5 if case["paged"] else None)])
            prefix.append(0, x["pk"], x["pv"], seq=0)
            state["prefix"] = prefix
        if "pool" in x:
            cache = TieredCache(B, hq, hkv, [TierConfig(case["dst"], case["dst"], 10 ** 9, bt, x["blocks"], paged_seed=7 if case["paged"] else None)],
                                prefix=prefix)
            cache.pool[0].copy_(x["pool"].view(torch.uint8).view(-1))
            cache.start[0][:], cache.len[0][:] = x["first"], x["held"]
            state["cache"], state["held"] = cache, np.array(x["held"], np.int64)
        x.pop("pk", None), x.pop("pv", None), x.pop("pool", None)     # the caches hold them now
    return state


# ------------------------------------------------------------------ one pass

def turned(case, h, weight, pos, freq):
    """Heads h [B][T][heads][128] normed (where the case says so) and rotated to their positions."""
    h = h.float()
    if case["norm"]:
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * weight
    angle = (pos.double().unsqueeze(-1) * freq).unsqueeze(2)
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    r = case["rotary"]
    if case["interleaved"]:
        a, b = h[..., 0:r:2], h[..., 1:r:2]
        t = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = h[..., :r // 2], h[..., r // 2:r]
        t = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((t, h[..., r:]), -1)


def attended(q, keys, values, seen):
    """Softmax over several sets of keys at once.  q [B][Hkv][G][128]; keys and values [Hkv][n][128] shared by all
    sequences or [B][Hkv][n][128], in the order of `seen`: None (all) or [B][n].  Returns out and log-sum-exp."""
    B, hkv, G, _ = q.shape

    def scores(k, ok):
        if k.dim() == 3:
            s = torch.matmul(q.transpose(0, 1).reshape(hkv, B * G, 128), k.transpose(1, 2).contiguous())
            return (s * SCALE).view(hkv, B, G, -1).transpose(0, 1)
        s = torch.matmul(q, k.transpose(2, 3).contiguous()) * SCALE
        return s.masked_fill(~ok.view(B, 1, 1, -1), -math.inf)

    def weighted(p, v):
        if v.dim() == 3:
            return torch.matmul(p.transpose(0, 1).reshape(hkv, B * G, -1), v).view(hkv, B, G, 128).transpose(0, 1)
        return torch.matmul(p, v)

    s = list(map(scores, keys, seen))
    m = torch.stack([x.amax(-1) for x in s]).amax(0).unsqueeze(-1)
    p = [torch.exp(x - m) for x in s]
    l = torch.stack([x.sum(-1) for x in p]).sum(0).unsqueeze(-1)
    out = torch.stack(list(map(weighted, p, values))).sum(0) / l
    return out.reshape(B, hkv * G, 128), (m + torch.log(l)).reshape(B, hkv * G)


def put(pool, rows, real, k, v):
    """k, v [B][T][Hkv][128] into the pool's rows where `real`."""
    rec, row = (r[real] for r in rows)
    pool[rec, :, 0, row] = k[real].to(pool.dtype)
    pool[rec, :, 1, row] = v[real].to(pool.dtype)


def plain(state, x):
    """The operators from their definition, in 32 bits; what a stored type rounds is rounded once."""
    case, kind = state["case"], state["case"]["kind"]
    B, hq, hkv, dst = case["batch"], case["q_heads"], case["kv_heads"], DT[case["dst"]]
    if kind in ("rotate", "append"):
        q = turned(case, x["q_in"], x.get("q_weight"), state["pos"], state["freq"]).to(dst)
        k = turned(case, x["k_in"], x.get("k_weight"), state["pos"], state["freq"]).to(dst)
        if kind == "rotate":
            return q, k
        put(x["pool"], state["rows"], state["real"], k, x["v_in"])
        return q * state["real"].view(B, -1, 1, 1), x["pool"].view(-1)
    keys, values, seen = [x["pk"].float()], [x["pv"].float()], [None]
    if kind == "step":
        put(x["pool"], state["rows"], state["real"], x["k_new"].transpose(1, 2), x["v_new"].transpose(1, 2))
        rec, row = state["window"]
        held = x["pool"][rec, :, :, row].float()               # [B][n][Hkv][2][128]
        keys.append(held[:, :, :, 0].transpose(1, 2).contiguous())
        values.append(held[:, :, :, 1].transpose(1, 2).contiguous())
        seen.append(state["seen"])
    out, lse = attended(x["q"].view(B, hkv, hq // hkv, 128).float(), keys, values, seen)
    return (out, lse) if kind == "shared" else (out, lse, x["pool"].view(-1))


def run(state):
    case, x = state["case"], state["x"]
    if not own:
        return plain(state, x)
    kind, dt = case["kind"], DT[case["dst"]]
    if kind == "rotate":
        return state["rotary"].apply(x["q_in"], x["k_in"], first_pos=state["first_pos"], q_out=state["q_out"], k_out=state["k_out"])
    if kind == "shared":
        return state["prefix"].attend_shared(x["q"])
    cache = state["cache"]
    cache.len[0][:] = state["held"]                            # every pass starts from the same window
    if kind == "append":
        cache.append_rotated(state["rotary"], x["k_in"], x["v_in"], q=x["q_in"], q_out=state["q_out"], counts=state["counts"],
                             first_pos=state["first_pos"])
        return state["q_out"], cache.pool[0].view(dt)
    out, lse = cache.step(x["q"], x["k_new"], x["v_new"])
    return out, lse, cache.pool[0].view(dt)


# ------------------------------------------------------------------ the same in 64 bits

def turned64(case, h, weight, first):
    """Heads [T][heads][128] of one sequence, in 64 bits: complex pairs turned by pos x freq."""
    h = h.double()
    if case["norm"]:
        h = h / torch.sqrt(h.square().sum(-1, keepdim=True) / 128 + EPS) * weight.double()
    r = case["rotary"]
    freq = torch.from_numpy(frequencies(r)).to(DEV)
    turn = torch.outer(torch.arange(first, first + h.shape[0], device=DEV).double(), freq)
    z = torch.polar(torch.ones_like(turn), turn).unsqueeze(1)
    out = h.clone()
    if case["interleaved"]:
        w = torch.complex(h[..., 0:r:2], h[..., 1:r:2]) * z
        out[..., 0:r:2], out[..., 1:r:2] = w.real, w.imag
    else:
        w = torch.complex(h[..., :r // 2], h[..., r // 2:r]) * z
        out[..., :r // 2], out[..., r // 2:r] = w.real, w.imag
    return out


def exact(case, seed):
    x = inputs(case, seed)
    B, hq, hkv, bt, kind, dst = case["batch"], case["q_heads"], case["kv_heads"], case["block"], case["kind"], DT[case["dst"]]
    G = hq // hkv
    pool = x["pool"].double() if "pool" in x else None

    def record(b, ordinal):
        return int(x["table"][b][ordinal // bt % x["blocks"]]), ordinal % bt

    if kind in ("rotate", "append"):
        first = positions(case)
        q = torch.stack([turned64(case, x["qkv"][b, :, :hq], x.get("q_weight"), first[b]) for b in range(B)])
        k = torch.stack([turned64(case, x["qkv"][b, :, hq:hq + hkv], x.get("k_weight"), first[b]) for b in range(B)])
        v = x["qkv"][:, :, hq + hkv:].double()
        if kind == "rotate":
            return q, k
    if kind == "append":
        for b, n in enumerate(counts(case)):
            q[b, n:] = 0.0
            at, done = x["first"][b] + x["held"][b], 0
            while done < n:                                    # block by block
                rec, row = record(b, at + done)
                m = min(n - done, bt - row)
                pool[rec, :, 0, row:row + m] = k[b, done:done + m].transpose(0, 1)
                pool[rec, :, 1, row:row + m] = v[b, done:done + m].transpose(0, 1)
                done += m
        return q, pool.view(-1)
    q = x["q"].double()
    out = torch.empty(B, hq, 128, dtype=torch.float64, device=DEV)
    lse = torch.empty(B, hq, dtype=torch.float64, device=DEV)
    window = []
    for b in range(B if kind == "step" else 0):
        rec, row = record(b, x["first"][b] + x["held"][b])
        pool[rec, :, 0, row], pool[rec, :, 1, row] = x["k_new"][b, :, 0].double(), x["v_new"][b, :, 0].double()
        where = torch.tensor([record(b, x["first"][b] + i) for i in range(x["held"][b] + 1)], device=DEV)
        window.append((where[:, 0], where[:, 1]))
    for h in range(hkv):
        pk, pv = x["pk"][h].double(), x["pv"][h].double()
        at = torch.arange(h * G, (h + 1) * G, device=DEV)
        if kind == "shared":
            s = torch.matmul(q[:, at].reshape(B * G, 128), pk.t().contiguous()) / math.sqrt(128.0)
            lse[:, at] = torch.logsumexp(s, -1).view(B, G)
            out[:, at] = torch.matmul(torch.softmax(s, -1), pv).view(B, G, 128)
            continue
        for b in range(B):
            rec, row = window[b]
            kk, vv = torch.cat((pk, pool[rec, h, 0, row])), torch.cat((pv, pool[rec, h, 1, row]))
            s = torch.matmul(q[b, at], kk.t().contiguous()) / math.sqrt(128.0)
            lse[b, at] = torch.logsumexp(s, -1)
            out[b, at] = torch.matmul(torch.softmax(s, -1), vv)
    return (out, lse) if kind == "shared" else (out, lse, pool.view(-1))
