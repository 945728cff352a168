"""The windowed kernels' bounded waits and their status word."""
import pytest
import torch

from paper_2609_25869_b200 import bsa

pytestmark = pytest.mark.gpu
TIMEOUT = 6  # BSA_ERR_DEVICE_TIMEOUT


def tensors(n, nk, d, heads=4, heads_kv=2):
    g = torch.Generator(device="cuda")
    g.manual_seed(41)
    shapes = ((1, heads, n, d), (1, heads_kv, nk, d), (1, heads_kv, nk, d), (1, heads, n, d))
    return [torch.empty(s, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g) for s in shapes]


class withheld_tiles:
    """First tiles never arrive, and a wait lasts about 10 ms of SM clocks."""

    def __enter__(self):
        bsa.debug_set_wait_limit(20_000_000)
        bsa.debug_withhold_arrival(True)

    def __exit__(self, *exc):
        bsa.debug_withhold_arrival(False)
        bsa.debug_set_wait_limit(0)


# rows, keys: few rows (one CTA; a cluster), tiles of rows (one tile per list, so that the producers reach their ends; several)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nk,left", [(1, 100, -1), (2, 5000, -1), (128, 128, -1), (700, 700, 200)])
def test_a_wait_that_runs_out_ends_in_a_status_not_a_hang(n, nk, left, d):
    """Both directions: the launches return, the status says so once, and the next calls have the bits of those before."""
    q, k, v, g = tensors(n, nk, d)
    kw = dict(left=left, right=0, sinks=2)
    O, L = bsa.window_forward(q, k, v, **kw)
    G = bsa.window_backward(q, k, v, O, L, g, **kw)
    assert bsa.window_status() == 0
    with withheld_tiles():
        bsa.window_forward(q, k, v, **kw)
        assert bsa.window_status() == TIMEOUT and bsa.window_status() == 0
        bsa.window_backward(q, k, v, O, L, g, **kw)
        assert bsa.window_status() == TIMEOUT and bsa.window_status() == 0
    O2, L2 = bsa.window_forward(q, k, v, **kw)
    G2 = bsa.window_backward(q, k, v, O, L, g, **kw)
    assert bsa.window_status() == 0
    assert torch.equal(O, O2) and torch.equal(L, L2) and all(torch.equal(a, b) for a, b in zip(G, G2))


@pytest.mark.parametrize("n", [2, 300])
def test_the_status_waits_for_streams_that_do_not_block(n):
    """A look behind calls on a side stream, while that stream still has work in front of them, is a look at them."""
    q, k, v, g = tensors(n, 600, 64)
    bsa.window_forward(q, k, v, left=50)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with withheld_tiles():
        with torch.cuda.stream(side):
            torch.cuda._sleep(400_000_000)  # about 0.2 s
            O, L = bsa.window_forward(q, k, v, left=50)
        assert bsa.window_status() == TIMEOUT and side.query()
        assert bsa.window_status() == 0
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        O, L = bsa.window_forward(q, k, v, left=50)
        bsa.window_backward(q, k, v, O, L, g, left=50)
    assert bsa.window_status() == 0 and side.query()
