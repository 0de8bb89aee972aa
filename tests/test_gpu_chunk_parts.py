"""Chunks whose sequences are cut along the tokens differently: partials of some, results of the others."""
import pytest

from chunk_testlib import all_tokens, check, make_cache, rnd
from paper_2604_19769_amd import binding as B
from test_gpu_chunk import attend

pytestmark = pytest.mark.gpu


def parts(c, T, counts=None):
    """Partials of a launch, from its workspace (520 bytes each)."""
    each = None if counts is None else (B.C.c_int64 * len(counts))(*counts)
    return (B.ttkv_chunk_workspace_bytes(c.h, c.c, -1, None, None, T, each) - 256) // 520


@pytest.mark.parametrize("dtype,older", [("f16", None), ("bf16", None), ("f16", "i8"), ("bf16", "i4")])
@pytest.mark.parametrize("heads,T,counts,past", [((8, 1), 300, [300, 5, 1, 0], [0, 20000, 700, 90]), ((8, 2), 20, [1, 20, 3, 20], [9000, 0, 0, 300]),
                                                 ((28, 4), 40, [2, 40, 0, 40], [30000, 10, 64, 3000])])
def test_batches_of_all_lengths(heads, T, counts, past, dtype, older):
    """A long sequence's rows are many items' and meet in the merge, beside rows that one item answers."""
    new = [p + n for p, n in zip(past, counts)]
    tiers = [(dtype, new)] if older is None else [(dtype, counts), (older, past)]
    c = make_cache(4, heads, tiers, paged=True)
    q = rnd(5, 4, T, heads[0], 128, dtype=dtype)
    assert parts(c, T, counts) > 0
    check(c, q, *attend(c, q, counts), counts=counts, untouched=7.0)
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_long_sequence_beside_many_rows(dtype):
    """189 row tiles of prompts, and a sequence of few new tokens that is cut all the same."""
    new = [130] * 63 + [4]
    p = make_cache(1, (32, 8), [(dtype, [40_000])], seed=40)
    c = make_cache(64, (32, 8), [(dtype, new)], prefix=p, members=[False] * 63 + [True])
    each = (B.C.c_int64 * 64)(*new)
    assert B.ttkv_chunk_workspace_bytes(c.h, c.c, -1, p.c, c.members.ctypes.data, 130, each) > 4 * 4 * 8 * 520 + 256
    q = rnd(5, 64, 130, 32, 128, dtype=dtype)
    check(c, q, *attend(c, q, new), counts=new, untouched=7.0)
    c.close()
    p.close()


@pytest.mark.parametrize("fmt", ["f16", "bf16", "i8", "i4"])
@pytest.mark.parametrize("T", [1, 5])
def test_more_parts_than_a_wave_has_lanes(T, fmt):
    """A row's parts are more than 64: what has the largest score lies in one of the first, of the last, or nowhere in particular."""
    dtype = "bf16" if fmt == "bf16" else "f16"
    c = make_cache(1, (8, 1), [(fmt, [30_000 + T])])
    assert parts(c, T) > 64 * T * 8
    keys, _ = all_tokens(c, 0)
    q = rnd(5, 1, T, 8, 128, dtype=dtype)
    check(c, q, *attend(c, q))
    for at in (700, 29_000):                                      # most of the weight on one token
        x = (q + 3.0 * keys[0, at].to(q.dtype)).contiguous()
        check(c, x, *attend(c, x))
    c.close()


@pytest.mark.parametrize("fmt", ["f16", "bf16", "i8"])
def test_one_part_beside_many(fmt):
    dtype = "bf16" if fmt == "bf16" else "f16"
    c = make_cache(3, (8, 1), [(fmt, [40, 60_000, 3000])])
    q = rnd(5, 3, 5, 8, 128, dtype=dtype)
    counts = [5, 2, 1]
    assert parts(c, 5, counts) > 64 * 2 * 8
    check(c, q, *attend(c, q, counts), counts=counts, untouched=7.0)
    c.close()
