"""How much an eviction by weight moves, as far as its workspace tells (no GPU needed)."""
import ctypes as C

from paper_2604_19769_amd import binding as B
from test_abi import host_cache
from test_chunk_refusals import light
from test_operator_refusals import h  # noqa: F401


def test_more_moves_than_a_launch_has_threads_for(h):  # noqa: F811
    """A launch has fewer than 2^32 threads, and the moves take 256 for every 16: 2^28 - 16 tokens of a KV head that may move are the most."""
    block = 1 << 16
    for n, fits in (((1 << 29) - block, True), ((1 << 29) + block, False)):
        c = host_cache(batch=1, Hq=1, Hkv=1, fmts=(("i4", "i4"),), bt=(block,))
        T = c.tier[0]
        T.ring_blocks = T.pool_blocks = (1 << 30) // block - 1
        C.cast(T.len, C.POINTER(C.c_int64))[0] = n
        keep = n // 2 // block * block                            # half of them go
        most = min(keep, n - keep)
        assert (most <= (1 << 28) - 16) == fits
        need = B.ttkv_evict_light_workspace_bytes(h, c, 0, keep, 0)
        assert (need >= 8 * most if fits else need == 0)
        assert light(h, c, keep=keep, recent=0) == (B.ERR_WORKSPACE if fits else B.ERR_UNSUPPORTED)
        assert C.cast(T.len, C.POINTER(C.c_int64))[0] == n
