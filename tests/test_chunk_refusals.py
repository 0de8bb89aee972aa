"""What the chunk, weight and eviction entry points refuse, before anything is enqueued (no GPU needed: the pointers are host memory
that must never be touched)."""
import ctypes as C

import numpy as np
import pytest

from paper_2604_19769_amd import binding as B
from test_abi import host_cache
from test_operator_refusals import ADDR, h, heads, status  # noqa: F401


def cache(fmts=(("f16", "f16"),), lens=(200, 0), **kw):
    c = host_cache(fmts=fmts, bt=(128,) * len(fmts), **kw)
    for t in range(len(fmts)):
        for b in range(c.batch):
            C.cast(c.tier[t].len, C.POINTER(C.c_int64))[b] = lens[b]
    return c


def i64(*x):
    a = np.array(x, np.int64)
    return (C.c_int64 * len(x)).from_buffer(a)


Q = dict(n=8, strides=(65536, 1024, 128))


def chunk(h, c, q=None, out=None, T=4, each=None, seq=-1, prefix=None, member=None, ws=None, size=0):  # noqa: F811
    return status(B.ttkv_chunk_attn, h, c, seq, prefix, member, q or heads(**Q), out or heads(**Q), None, T, each, ws, size, None)


def test_chunk_refusals(h):  # noqa: F811
    c = cache()
    assert status(B.ttkv_chunk_attn, None, c, -1, None, None, heads(**Q), heads(**Q), None, 4, None, None, 0, None) == B.ERR_INVALID_ARG
    for q, o in ((None, heads(**Q)), (heads(**Q), None)):
        assert status(B.ttkv_chunk_attn, h, c, -1, None, None, q, o, None, 4, None, None, 0, None) == B.ERR_INVALID_ARG
    for T, each, want in ((0, None, B.OK), (-1, None, B.ERR_INVALID_ARG), (4, i64(0, 0), B.OK), (4, i64(5, 0), B.ERR_INVALID_ARG),
                          (4, i64(-1, 0), B.ERR_INVALID_ARG), ((1 << 22) + 1, None, B.ERR_UNSUPPORTED)):
        assert chunk(h, c, T=T, each=each) == want, (T, want)
    wide = heads(n=64, strides=(1 << 40, 8192, 128))
    assert chunk(h, cache(Hq=64), q=wide, out=wide, T=1 << 22) == B.ERR_UNSUPPORTED             # 2^29 rows
    for seq in (-2, 2):
        assert chunk(h, c, seq=seq) == B.ERR_INVALID_ARG
    bad_q = [heads(n=4, strides=Q["strides"]), heads(n=8, data=None), heads(n=8, data=ADDR + 2, strides=Q["strides"]), heads(n=8, strides=(65536, 1024, 3)),
             heads(n=8, strides=(65536, -1024, 128))]
    for q in bad_q:
        assert chunk(h, c, q=q) == B.ERR_INVALID_ARG and chunk(h, c, out=q) == B.ERR_INVALID_ARG
    assert chunk(h, c, out=heads(n=8, strides=(65536, 1024, 64))) == B.ERR_INVALID_ARG       # rows that overlap
    assert chunk(h, c, q=heads(fmt=B.F32, n=8, strides=Q["strides"])) == B.ERR_UNSUPPORTED
    assert chunk(h, c, out=heads(fmt=B.F32, n=8, strides=Q["strides"])) == B.ERR_UNSUPPORTED
    assert chunk(h, c, q=heads(fmt=B.I8_SYM_G32, n=8, strides=Q["strides"])) == B.ERR_UNSUPPORTED
    # few rows are cut along the tokens: a workspace is needed, and asked for
    need = B.ttkv_chunk_workspace_bytes(h, cache(lens=(1000, 0)), -1, None, None, 4, None)
    assert need > 256 and chunk(h, cache(lens=(1000, 0))) == B.ERR_WORKSPACE and chunk(h, cache(lens=(1000, 0)), ws=ADDR, size=need - 600) == B.ERR_WORKSPACE


def test_chunk_tiers(h):  # noqa: F811
    bf = heads(fmt=B.BF16, n=8, strides=Q["strides"])
    assert chunk(h, cache(fmts=(("bf16", "bf16"),))) == B.ERR_UNSUPPORTED                    # a bf16 tier takes bf16 queries
    assert chunk(h, cache(fmts=(("f16", "f16"), ("bf16", "bf16"))), q=bf) == B.ERR_UNSUPPORTED
    assert chunk(h, cache(fmts=(("f16", "f16"), ("i8", "i8"), ("i4", "i4"))), T=0) == B.OK
    for fmts in ((("f16", "f16"), ("i4t", "i4")), (("f16", "f16"), ("i8", "i4c")), (("f16", "f16"), ("i4", "i8")), (("f16", "i8"),)):
        assert chunk(h, cache(fmts=fmts, lens=(256, 0)), T=0) == B.ERR_UNSUPPORTED, fmts
        assert B.ttkv_chunk_workspace_bytes(h, cache(fmts=fmts, lens=(256, 0)), -1, None, None, 4, None) == 0
    c = cache()
    c.tier[0].mem = B.MEM_HOST_PINNED
    assert chunk(h, c, T=0) == B.ERR_UNSUPPORTED
    c = cache(lens=(1 << 20, 0))
    assert chunk(h, c) == B.ERR_INVALID_ARG                                                  # more than the ring holds
    long = cache(fmts=(("f16", "f16"),) * 4)
    for t in range(4):                                                                       # places beyond 31 bits
        long.tier[t].ring_blocks = (1 << 30) // 128 - 1
        long.tier[t].pool_blocks = 2 * long.tier[t].ring_blocks
        C.cast(long.tier[t].len, C.POINTER(C.c_int64))[0] = (1 << 30) - 128
    assert chunk(h, long) == B.ERR_UNSUPPORTED and chunk(h, long, each=i64(0, 0)) == B.ERR_UNSUPPORTED


def test_chunk_prefixes(h):  # noqa: F811
    c = cache()
    one = cache(batch=1, lens=(100,))
    assert chunk(h, c, prefix=one, T=0) == B.OK and chunk(h, c, prefix=cache(), T=0) == B.ERR_INVALID_ARG
    assert chunk(h, c, prefix=cache(batch=1, Hq=16, lens=(100,)), T=0) == B.ERR_INVALID_ARG
    assert chunk(h, c, prefix=cache(batch=1, fmts=(("bf16", "bf16"),), lens=(100,)), T=0) == B.ERR_UNSUPPORTED
    one.softmax_scale = 0.5
    assert chunk(h, c, prefix=one, T=0) == B.ERR_INVALID_ARG


def weigh(h, c, q=None, lse=ADDR, T=4, each=None, fresh=None, tier=0, seq=-1, w=ADDR):  # noqa: F811
    return status(B.ttkv_add_weights, h, c, tier, seq, q or heads(**Q), lse, T, each, fresh, w, None, 0, None)


def test_weight_refusals(h):  # noqa: F811
    c = cache()
    assert status(B.ttkv_add_weights, None, c, 0, -1, heads(**Q), ADDR, 4, None, None, ADDR, None, 0, None) == B.ERR_INVALID_ARG
    assert status(B.ttkv_add_weights, h, c, 0, -1, None, ADDR, 4, None, None, ADDR, None, 0, None) == B.ERR_INVALID_ARG
    assert weigh(h, c, lse=None) == B.ERR_INVALID_ARG and weigh(h, c, w=None) == B.ERR_INVALID_ARG
    assert weigh(h, c, T=0) == B.OK and weigh(h, c, each=i64(0, 0)) == B.OK and weigh(h, cache(lens=(0, 0))) == B.OK
    for kw in (dict(tier=1), dict(tier=-1), dict(seq=2), dict(seq=-2), dict(T=-1), dict(each=i64(5, 0)), dict(each=i64(0, -1)), dict(fresh=i64(-1, 0)),
               dict(q=heads(n=2, strides=Q["strides"])), dict(q=heads(n=8, data=ADDR + 8, strides=Q["strides"]))):
        assert weigh(h, c, **kw) == B.ERR_INVALID_ARG, kw
    assert weigh(h, c, q=heads(fmt=B.F32, n=8, strides=Q["strides"])) == B.ERR_UNSUPPORTED and weigh(h, c, T=(1 << 22) + 1) == B.ERR_UNSUPPORTED
    assert weigh(h, cache(fmts=(("bf16", "bf16"),))) == B.ERR_UNSUPPORTED
    assert weigh(h, cache(fmts=(("f16", "f16"), ("i4t", "i4")), lens=(256, 0)), tier=1) == B.ERR_UNSUPPORTED
    c.tier[0].mem = B.MEM_HOST_PINNED
    assert weigh(h, c) == B.ERR_UNSUPPORTED


def light(h, c, keep=64, recent=8, tier=0, w=ADDR, ws=None, size=0):  # noqa: F811
    return status(B.ttkv_evict_light, h, c, tier, keep, recent, 0, w, ws, size, None)


def test_eviction_refusals(h):  # noqa: F811
    c = cache(lens=(900, 0))
    assert status(B.ttkv_evict_light, None, c, 0, 64, 8, 0, ADDR, None, 0, None) == B.ERR_INVALID_ARG
    for kw in (dict(keep=7), dict(recent=-1), dict(keep=-1, recent=-1), dict(tier=1), dict(tier=-1), dict(w=None)):
        assert light(h, c, **kw) == B.ERR_INVALID_ARG, kw
    need = B.ttkv_evict_light_workspace_bytes(h, c, 0, 64, 8)
    assert need > 256 and light(h, c) == B.ERR_WORKSPACE and light(h, c, ws=ADDR, size=need - 600) == B.ERR_WORKSPACE
    assert light(h, c, keep=773) == B.OK and light(h, c, keep=1 << 40) == B.OK               # less than a block too many: nothing to do
    assert C.cast(c.tier[0].len, C.POINTER(C.c_int64))[0] == 900
    for fmts in ((("f16", "f16"), ("i4t", "i4")), (("f16", "f16"), ("i8", "i4c"))):
        assert light(h, cache(fmts=fmts, lens=(256, 0)), tier=1, keep=64) == B.ERR_UNSUPPORTED, fmts
    c.tier[0].k_sum = c.tier[0].k_summary = ADDR
    assert light(h, c) == B.ERR_UNSUPPORTED
    c.tier[0].k_sum = c.tier[0].k_summary = None
    c.tier[0].mem = B.MEM_HOST_PINNED
    assert light(h, c) == B.ERR_UNSUPPORTED and B.ttkv_evict_light_workspace_bytes(h, c, 0, 64, 8) == 0


def test_blocks_beyond_32_bits(h):  # noqa: F811
    """A KV head's part of a block of 2^22 tokens has more bytes than 31 bits count."""
    c = cache(lens=(0, 0))
    c.tier[0].block_tokens, c.tier[0].ring_blocks, c.tier[0].pool_blocks, c.tier[0].capacity_tokens = 1 << 22, 2, 4, 1 << 23
    assert chunk(h, c, T=0) == B.ERR_UNSUPPORTED and weigh(h, c, T=0) == B.ERR_UNSUPPORTED and light(h, c) == B.ERR_UNSUPPORTED
    c.tier[0].block_tokens = c.tier[0].capacity_tokens = 1 << 21
    assert chunk(h, c, T=0) == B.OK and weigh(h, c, T=0) == B.OK and light(h, c) == B.OK
