"""What the norm / rotation / append and shared-prefix entry points refuse, before anything is enqueued (no GPU needed: the
pointers are host memory that must never be touched)."""
import ctypes as C

import numpy as np
import pytest

from paper_2604_19769_amd import binding as B
from test_abi import host_cache

BUF = np.zeros(4096, np.uint8)
ADDR = (BUF.ctypes.data + 255) // 256 * 256


def heads(n=2, fmt=B.F16, data=ADDR, strides=(4096, 1024, 128)):
    return B.ttkv_heads(data, fmt, n, *strides)


def rope(dim=128, norm=3, eps=1e-6, freq=None, **kw):
    f = np.ones(64) if freq is None else freq
    r = B.ttkv_rope(dim, 0, norm, eps, 1.0, f.ctypes.data, None, None)
    for k, v in kw.items():
        setattr(r, k, v)
    r._keep = f
    return r


@pytest.fixture()
def h():
    handle = B.ttkv_create()
    yield handle
    B.ttkv_destroy(handle)


def status(call, *args):
    try:
        call(*args)
    except B.TTKVError as e:
        return e.status
    return B.OK


def norm_rope(h, r=None, q=None, q_out=None, k=None, k_out=None, n_seq=1, n_tokens=4):
    return status(B.ttkv_norm_rope, h, r or rope(), q, q_out, k, k_out, n_seq, n_tokens, None, None, None)


def test_norm_rope_refusals(h):
    q, o = heads(), heads()
    assert norm_rope(h) == B.ERR_INVALID_ARG                                              # nothing to do it to
    assert norm_rope(h, q=q) == B.ERR_INVALID_ARG and norm_rope(h, q_out=o) == B.ERR_INVALID_ARG
    assert norm_rope(None, q=q, q_out=o) == B.ERR_INVALID_ARG
    for n_seq, n_tokens, want in ((0, 4, B.OK), (1, 0, B.OK), (-1, 4, B.ERR_INVALID_ARG), (65, 4, B.ERR_INVALID_ARG), (1, -1, B.ERR_INVALID_ARG),
                                  (1, (1 << 28) + 1, B.ERR_INVALID_ARG)):
        assert norm_rope(h, q=q, q_out=o, n_seq=n_seq, n_tokens=n_tokens) == want, (n_seq, n_tokens)
    for bad in (heads(n=3), heads(n=0), heads(data=None), heads(data=ADDR + 2), heads(fmt=B.I8_SYM_G32), heads(strides=(4096, 1024, 64)),
                heads(strides=(4096, 1027, 128)), heads(strides=(4096, 1024, 0)), heads(strides=(4096, -1024, 128))):
        assert norm_rope(h, q=q, q_out=bad) == B.ERR_INVALID_ARG
    assert norm_rope(h, q=q, q_out=heads(fmt=B.BF16), k=heads(), k_out=heads(fmt=B.F16)) == B.ERR_UNSUPPORTED
    assert norm_rope(h, q=q, q_out=o, k=heads(fmt=B.F32), k_out=o) == B.ERR_UNSUPPORTED
    # strides of dimensions of one entry are not looked at
    assert norm_rope(h, q=heads(n=1, strides=(-7, -7, 3)), q_out=heads(n=1, strides=(1, 2, 3)), n_seq=0, n_tokens=1) == B.OK


def test_rope_description_refusals(h):
    q, o = heads(), heads()
    for dim, want in ((-16, B.ERR_INVALID_ARG), (8, B.ERR_UNSUPPORTED), (100, B.ERR_UNSUPPORTED), (144, B.ERR_INVALID_ARG)):
        assert norm_rope(h, rope(dim), q, o) == want, dim
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(norm=4), dict(q_weight=ADDR + 4), dict(k_weight=ADDR + 8)):
        assert norm_rope(h, rope(**kw), q, o) == B.ERR_INVALID_ARG, kw
    for bad in (float("nan"), float("inf"), 1e7):
        f = np.ones(64)
        f[63] = bad
        assert norm_rope(h, rope(freq=f), q, o) == B.ERR_INVALID_ARG
        assert norm_rope(h, rope(112, freq=f), q, o, n_seq=0) == B.OK                     # frequencies behind the rotated channels
    r = rope()
    r.freq = None
    assert norm_rope(h, r, q, o) == B.ERR_INVALID_ARG
    r.rotary_dim = 0
    assert norm_rope(h, r, q, o, n_seq=0) == B.OK


def append(h, c, tier=0, seq=-1, r=None, q=None, q_out=None, k=None, v=None, n_tokens=4, n_each=None):
    n = None if n_each is None else np.array(n_each, np.int64)
    return status(B.ttkv_rope_append, h, c, tier, seq, r or rope(), q, q_out, k or heads(), v or heads(), n_tokens,
                  None if n is None else n.ctypes.data, None, None, None)


def test_rope_append_refusals(h):
    c = host_cache()
    lens = c._keep[2]
    assert append(h, c, n_tokens=0) == B.OK and append(h, c, n_each=[0, 0]) == B.OK
    assert append(None, c) == B.ERR_INVALID_ARG
    for kw in (dict(tier=3), dict(tier=-1), dict(seq=2), dict(seq=-2), dict(n_tokens=-1), dict(q=heads(8)), dict(k=heads(1)), dict(v=heads(3)),
               dict(n_each=[5, 0]), dict(n_each=[0, -1]), dict(k=heads(data=ADDR + 8)), dict(q=heads(8), q_out=heads(7))):
        assert append(h, c, **kw) == B.ERR_INVALID_ARG, kw
    assert status(B.ttkv_rope_append, h, c, 0, -1, rope(), None, None, None, heads(), 4, None, None, None, None) == B.ERR_INVALID_ARG
    assert append(h, c, tier=1) == B.ERR_UNSUPPORTED                                      # int8 rows
    assert append(h, c, k=heads(fmt=B.F32)) == B.ERR_UNSUPPORTED                          # keys and values of two types
    assert append(h, c, q=heads(8), q_out=heads(8, fmt=B.BF16)) == B.ERR_UNSUPPORTED      # queries of another type than the tier's
    c.tier[0].mem = B.MEM_HOST_PINNED
    assert append(h, c) == B.ERR_UNSUPPORTED
    c.tier[0].mem = B.MEM_DEVICE
    c.tier[0].k_sum = c.tier[0].k_summary = ADDR
    assert append(h, c) == B.ERR_UNSUPPORTED
    c.tier[0].k_sum = c.tier[0].k_summary = None
    lens[:] = [8 * 128 - 4, 8 * 128 - 3]
    assert append(h, c) == B.ERR_CAPACITY
    assert lens.tolist() == [8 * 128 - 4, 8 * 128 - 3]


def prefix_cache(fmt="f16", **kw):
    return host_cache(batch=1, fmts=((fmt, fmt),), bt=(128,), **kw)


def shared(h, p, q=ADDR, q_fmt=B.F16, n_seq=4, out=ADDR, ws=ADDR, ws_bytes=1 << 30):
    return status(B.ttkv_shared_attn, h, p, q, q_fmt, n_seq, out, None, ws, ws_bytes, None)


def test_shared_attn_refusals(h):
    p = prefix_cache()
    p._keep[2][:] = 500
    assert shared(h, p, n_seq=0) == B.OK
    for kw in (dict(q=None), dict(out=None), dict(n_seq=-1), dict(n_seq=65537), dict(q_fmt=B.F32), dict(q=ADDR + 2)):
        assert shared(h, p, **kw) == B.ERR_INVALID_ARG, kw
    assert shared(None, p) == B.ERR_INVALID_ARG
    need = B.ttkv_shared_workspace_bytes(h, p, 4)
    assert need >= 4 * 8 * 130 * 4 * B.ttkv_prefix_parts(h, p, 4) > 0
    assert shared(h, p, ws=None) == B.ERR_WORKSPACE and shared(h, p, ws_bytes=need // 2) == B.ERR_WORKSPACE
    big = host_cache(batch=1, Hq=128, fmts=(("f16", "f16"),), bt=(128,))
    assert shared(h, big, n_seq=65536) == B.ERR_UNSUPPORTED                               # 2^23 rows
    two = host_cache(batch=2, fmts=(("f16", "f16"),), bt=(128,))
    assert shared(h, two) == B.ERR_INVALID_ARG and B.ttkv_prefix_parts(h, two, 4) == -1
    for pair in (("i4t", "i4"), ("i8", "i4c"), ("i4", "i4c")):                            # layouts of other kernels
        packed = host_cache(batch=1, fmts=(("f16", "f16"), pair), bt=(128, 128))
        assert shared(h, packed) == B.ERR_UNSUPPORTED
        assert B.ttkv_prefix_parts(h, packed, 4) == -1 and B.ttkv_shared_workspace_bytes(h, packed, 4) == 0
    assert shared(h, prefix_cache("bf16")) == B.ERR_UNSUPPORTED                           # bf16 keys, fp16 queries
    p.tier[0].mem = B.MEM_HOST_PINNED
    assert shared(h, p) == B.ERR_UNSUPPORTED
    p.tier[0].mem = B.MEM_DEVICE
    p.head_dim = 64
    assert shared(h, p) == B.ERR_UNSUPPORTED
    p.head_dim = 128
    p.tier[0].len = None
    assert shared(h, p) == B.ERR_INVALID_ARG


def test_prefix_parts_follow_the_lengths(h):
    p = prefix_cache()
    assert B.ttkv_prefix_parts(h, p, 4) == 0 and B.ttkv_shared_workspace_bytes(h, p, 0) == 256
    for n in (1, 64, 65, 500, 1024):
        p._keep[2][:] = n
        assert 1 <= B.ttkv_prefix_parts(h, p, 4) <= -(-n // 64)
        assert B.ttkv_prefix_parts(h, p, 0) == 0
    assert B.ttkv_prefix_parts(h, p, -1) == -1


def step(h, c, p, member=None, q=ADDR, q_fmt=B.F16, k=ADDR, v=ADDR, fmt=B.F16, out=ADDR, ws=ADDR, ws_bytes=1 << 30):
    m = None if member is None else np.array(member, np.int32)
    return status(B.ttkv_decode_step_shared, h, c, p, None if m is None else m.ctypes.data, q, q_fmt, k, v, fmt, out, None, ws, ws_bytes, None)


def test_decode_step_shared_refusals(h):
    c, p = host_cache(fmts=(("f16", "f16"),), bt=(128,)), prefix_cache()
    p._keep[2][:] = 500
    lens = c._keep[2]
    lens[:] = 5
    for kw in (dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(fmt=B.F32), dict(q_fmt=B.I8_SYM_G32), dict(q=ADDR + 8)):
        assert step(h, c, p, **kw) == B.ERR_INVALID_ARG, kw
    assert step(None, c, p) == B.ERR_INVALID_ARG
    assert step(h, c, prefix_cache(Hq=4)) == B.ERR_INVALID_ARG and step(h, c, prefix_cache(Hkv=4)) == B.ERR_INVALID_ARG
    other = prefix_cache()
    other.softmax_scale = 0.1
    assert step(h, c, other) == B.ERR_INVALID_ARG
    assert step(h, c, host_cache(batch=2, fmts=(("f16", "f16"),), bt=(128,))) == B.ERR_INVALID_ARG
    assert step(h, c, host_cache(batch=1, fmts=(("f16", "f16"), ("i8", "i4c")), bt=(128, 128))) == B.ERR_UNSUPPORTED
    assert step(h, c, prefix_cache("bf16")) == B.ERR_UNSUPPORTED
    assert step(h, c, p, fmt=B.BF16) == B.ERR_UNSUPPORTED                                 # the fp tier takes its own format
    parts = B.ttkv_count_parts(h, c, None, None, 0, 0) + B.ttkv_prefix_parts(h, p, 2)
    assert step(h, c, p, ws=None) == B.ERR_WORKSPACE
    assert step(h, c, p, ws_bytes=2 * 8 * 130 * 4 * (parts - 1)) == B.ERR_WORKSPACE       # one part too few
    lens[:] = 8 * 128
    assert step(h, c, p) == B.ERR_CAPACITY
    assert lens.tolist() == [8 * 128, 8 * 128]
    i8 = host_cache(fmts=(("i8", "i8"),), bt=(128,))
    assert step(h, i8, p) == B.ERR_UNSUPPORTED                                            # the token goes to an fp tier


def test_more_rows_than_32_bits_count(h):
    """2^16 sequences of 2^20 heads: refused before the rows are multiplied out."""
    p = prefix_cache(Hq=1 << 20, Hkv=1)
    p._keep[2][:] = 500
    assert shared(h, p, n_seq=65536) == B.ERR_UNSUPPORTED
    assert B.ttkv_prefix_parts(h, p, 65536) == -1 and B.ttkv_shared_workspace_bytes(h, p, 65536) == 0
    c = host_cache(Hq=1 << 25, Hkv=1, batch=64, fmts=(("f16", "f16"),), bt=(128,))
    wide = prefix_cache(Hq=1 << 25, Hkv=1)
    wide._keep[2][:] = 500
    assert step(h, c, wide) == B.ERR_UNSUPPORTED


def test_more_tokens_than_a_launch_has_waves(h):
    """A wave per token: 2^26 of them would be 2^32 threads along the grid's first dimension."""
    wide = heads(n=1, strides=(1 << 40, 128, 128))
    for n, want in (((1 << 25) + 1, B.ERR_INVALID_ARG), (1 << 26, B.ERR_INVALID_ARG)):
        assert norm_rope(h, q=wide, q_out=wide, n_tokens=n) == want
        assert append(h, host_cache(), n_tokens=n, n_each=[0, 0]) == want
    assert append(h, host_cache(), n_tokens=1 << 25, n_each=[0, 0]) == B.OK
