"""Outputs that a call allocates while another stream than the current one is to write them."""
import pytest
import torch

from paper_2609_25869_b200 import bsa

pytestmark = pytest.mark.gpu


def behind_queued_work(call, sizes, stream):
    """``call(stream)`` right after tensors of ``sizes`` were dropped that the current stream is still going to write."""
    torch.empty(8, dtype=torch.uint8, device="cuda").fill_(1)  # (a kernel's first launch waits for the device)
    torch.cuda._sleep(1)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    pending = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda._sleep(200_000_000)  # about 0.1 s
    for x in pending:
        x.fill_(1)
    del pending, x
    out = call(stream)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("op", ["rope", "forward", "backward"])
def test_fresh_outputs_come_from_the_pool_of_the_stream_that_writes_them(op, handle):
    g = torch.Generator(device="cuda")
    g.manual_seed(51)
    q, k, v, dO = [torch.empty(s, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g)
                   for s in ((2, 8, 4096, 128), (2, 4, 4096, 128), (2, 4, 4096, 128), (2, 8, 4096, 128))]
    O, L = bsa.window_forward(q, k, v, left=100)
    calls = {"rope": lambda s: bsa.rope(q, k, axes=(128,), grid=(4096,), stream=s),
             "forward": lambda s: bsa.window_forward(q, k, v, left=100, stream=s),
             "backward": lambda s: bsa.window_backward(q, k, v, O, L, dO, left=100, stream=s)}
    want = calls[op](None)
    sizes = [t.numel() * t.element_size() for t in want]
    side = torch.cuda.Stream()
    got = behind_queued_work(calls[op], sizes, side.cuda_stream if handle else side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = calls[op](0 if handle else torch.cuda.default_stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("op", ["forward", "request", "statistics"])
def test_so_do_the_outputs_of_plans(op, handle):
    g = torch.Generator(device="cuda")
    g.manual_seed(52)
    h, n, d = 8, 4096, 128
    q, k, v = [torch.empty((h, n, d), device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g) for _ in range(3)]
    mask = torch.ones((h, n // 64, n // 64), dtype=torch.uint8, device="cuda")
    with bsa.plan_create(mask, 64, 64, n, h, d) as plan:
        other = []

        def request(s):
            p, O, L = bsa.request(mask, 64, 64, n, h, d, q, k, v, stream=s)
            other.append(p)
            return O, L
        calls = {"forward": lambda s: plan.forward(q, k, v, stream=s), "request": request,
                 "statistics": lambda s: (bsa.mask_stats_noalloc(mask, stream=s),)}
        want = calls[op](None)
        sizes = [t.numel() * t.element_size() for t in want]
        side = torch.cuda.Stream()
        got = behind_queued_work(calls[op], sizes, side.cuda_stream if handle else side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for p in other:
            p.destroy()
