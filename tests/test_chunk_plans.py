"""How a chunk's launch is cut, as far as the workspace that it asks for tells (no GPU needed)."""
import ctypes as C

import pytest

from paper_2604_19769_amd import binding as B
from test_abi import host_cache
from test_chunk_refusals import i64
from test_operator_refusals import h  # noqa: F401

PART = 520                                                        # a row's part: 128 sums, maximum, sum of weights


def cache(lens, Hq=32, Hkv=8):
    c = host_cache(batch=len(lens), Hq=Hq, Hkv=Hkv, fmts=(("f16", "f16"),), bt=(128,))
    c.tier[0].ring_blocks = (1 << 24) // 128
    c.tier[0].pool_blocks = len(lens) * c.tier[0].ring_blocks
    for b, n in enumerate(lens):
        C.cast(c.tier[0].len, C.POINTER(C.c_int64))[b] = n
    return c


def parts(h, lens, new, **kw):  # noqa: F811
    """Parts of a launch, from its workspace."""
    need = B.ttkv_chunk_workspace_bytes(h, cache(lens, **kw), -1, None, None, max(new), i64(*new))
    assert need >= 256
    return (need - 256) // PART


@pytest.mark.parametrize("prompt,few,past", [(1024, 4, 100_000), (4096, 4, 500_000), (2000, 1, 2_000_000), (600, 16, 1_000_000)])
def test_a_prompt_beside_a_long_sequence(h, prompt, few, past):  # noqa: F811
    """The prompt's rows have as many parts as the prompt is cut into, not as many as the long sequence is: a workgroup leaves 256 parts at most, and
    cutting adds 6 rounds of 256 workgroups at most to one per row tile and KV head."""
    got = parts(h, [prompt, past + few], [prompt, few])
    assert 0 < got <= 256 * (8 * (-(-prompt * 4 // 256) + 1) + 6 * 256)


@pytest.mark.parametrize("prompts,few,past", [([8192], 4, 500_000), ([8192], 1, 2_000_000), ([4000, 5000, 3000], 8, 300_000), ([20_000], 4, 900_000)])
def test_a_long_sequence_beside_many_rows(h, prompts, few, past):  # noqa: F811
    """As many row tiles as fill the chip several times: a sequence that would take longer than the rest of the batch by itself is cut all the
    same, into items of no more than a fair share of the steps of 32 tokens; the prompts are not."""
    new, lens = [*prompts, few], [*prompts, past + few]
    tiles = [-(-n * 4 // 256) for n in new]
    steps = [-(-n // 32) for n in lens]
    assert sum(tiles) * 8 >= 1024
    fair = sum(a * b for a, b in zip(tiles, steps)) * 8 // 256
    cut, rest = divmod(parts(h, lens, new), few * 4 * 8)
    assert rest == 0 and cut > 1 and steps[-1] <= cut * fair


@pytest.mark.parametrize("lens,new", [([8192], None), ([8192] * 4, None), ([9000, 2000, 4000, 8000], None), ([32768], [8192]), ([40_000, 30_000], [4096, 4096])])
def test_prompts_of_many_rows(h, lens, new):  # noqa: F811
    """Their own row tiles are items enough: nothing is cut."""
    assert parts(h, lens, new or lens) == 0
