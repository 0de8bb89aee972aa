"""One prefix attended from several streams at once: every stream's calls have a workspace and results of their own."""
import pytest
import torch

from test_gpu_rotary import DEV, rnd
from test_gpu_shared_prefix import check, make_prefix, reference, window

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 2500), (32, 8, 9000)])
def test_calls_that_overlap(Hq, Hkv, n):
    """Different numbers of sequences, no synchronization in between, workspaces that grow on one stream while the other's call is on its way."""
    c, k, v = make_prefix(Hq, Hkv, "f16", n)
    sizes = [[3, 40, 70, 200], [64, 2, 300, 5]]
    qs = [[rnd(10 * i + j, s, Hq, 128, dtype="f16") for j, s in enumerate(x)] for i, x in enumerate(sizes)]
    want = [[[y.clone() for y in c.attend_shared(q)] for q in x] for x in qs]
    check(*want[0][0], [reference(x, [(k, v)], c.c.softmax_scale) for x in qs[0][0]])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    for _ in range(5):
        got = [[], []]
        for j in range(4):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    got[i].append([y.clone() for y in c.attend_shared(qs[i][j])])
        torch.cuda.synchronize()
        for i in range(2):
            for j in range(4):
                assert torch.equal(got[i][j][0], want[i][j][0]) and torch.equal(got[i][j][1], want[i][j][1]), (i, j)
    c.close()


def test_results_stay_until_the_stream_s_next_call():
    c, k, v = make_prefix(8, 2, "f16", 700)
    q = rnd(1, 6, 8, 128, dtype="f16")
    out, lse = c.attend_shared(q)
    kept = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.attend_shared(-q)
        assert other[0].data_ptr() != out.data_ptr() and other[1].data_ptr() != lse.data_ptr()
    torch.cuda.synchronize()
    assert torch.equal(out, kept[0]) and torch.equal(lse, kept[1])
    assert c.attend_shared(q)[0].data_ptr() == out.data_ptr()              # the buffers of the call before
    assert torch.equal(out, kept[0])
    c.close()


def test_a_workspace_that_another_stream_still_uses_is_not_handed_out():
    """A cache's step grows its workspace on a stream that did not allocate it: the old one stays out of use until that stream is through."""
    p, _, _ = make_prefix(8, 2, "f16", 700)
    c, _ = window(2, 8, 2, "f16", [10, 300], p)
    q = rnd(1, 2, 8, 128, dtype="f16")
    c.decode(q)                                                             # allocated here
    torch.cuda.synchronize()
    old, size = c.ws.data_ptr(), c.ws.numel()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                                      # some 50 ms
        c.decode(q)
        c._workspace(4 * c.ws_parts)
    fresh = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(3)]
    assert not side.query()
    assert all(x.data_ptr() != old for x in fresh)
    torch.cuda.synchronize()
    c.close(), p.close()
