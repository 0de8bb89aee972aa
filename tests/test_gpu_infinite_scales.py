"""Quantized tiers whose stored scales or zero points are infinite (rows of values beyond what fp16 scales hold): no finite number comes of them."""
import pytest
import torch

from chunk_testlib import DEV, make_cache, rnd
from test_gpu_chunk import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,k_codes,v_codes,group,what", [("i8", 128, 128, 32, "scale"), ("i4", 64, 64, 64, "scale"), ("i4", 64, 64, 64, "zero"),
                                                            ("k8v4", 128, 64, 64, "scale"), ("k8v4", 128, 64, 64, "zero")])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [3, 20, 70, 200])
def test_values(T, dtype, fmt, k_codes, v_codes, group, what):
    """A newer token's first value scale (zero point): the rows that see it have nothing finite in the group's channels, the others every bit."""
    n = T + 70
    c = make_cache(1, (8, 2), [(fmt, [n])], wrap=False)
    q = rnd(6, 1, T, 8, 128, dtype=dtype)
    clean = attend(c, q)
    row = n - (T + 1) // 2
    at = (row // 64 * 2 + 1) * 64 * (k_codes + v_codes + 16) + 64 * (k_codes + 8 + v_codes) + row % 64 * 8   # KV head 1, the row's first value scale
    at += 2 if what == "zero" else 0
    c.pool[0].view(-1)[at:at + 2] = torch.tensor([0x00, 0x7c], dtype=torch.uint8, device=DEV)
    wild = attend(c, q)
    seen = T - (n - row)
    assert torch.equal(wild[0][:, :seen], clean[0][:, :seen]) and torch.equal(wild[1], clean[1])
    assert not torch.isfinite(wild[0][:, seen:, 4:, :group]).any()
    assert torch.equal(wild[0][:, :, 4:, group:], clean[0][:, :, 4:, group:]) and torch.equal(wild[0][:, :, :4], clean[0][:, :, :4])
    c.close()
