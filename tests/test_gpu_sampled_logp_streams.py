"""SampledLogp with its forward on a stream of the caller's: backward runs on the current stream, and what it reads stays until
it has."""
import torch
import pytest

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu


def test_forward_on_another_stream():
    T, V = 300, 5000
    gen = torch.Generator("cuda").manual_seed(2)
    z = torch.randn(T, V, device="cuda", generator=gen)
    act = z.argmax(1).to(torch.int32)
    up = torch.randn(T, device="cuda", generator=gen)
    par = dict(temperature=0.9, top_k=30)
    x = z.clone().requires_grad_()
    grpo.SampledLogp.apply(x, act, par).backward(up)
    want = x.grad.clone()
    busy = torch.ones(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for rep in range(3):
        x = z.clone().requires_grad_()
        side.wait_stream(torch.cuda.current_stream())
        logp = grpo.SampledLogp.apply(x, act, dict(par, stream=side))
        torch.cuda.current_stream().wait_stream(side)
        logp.record_stream(torch.cuda.current_stream())
        for _ in range(20):  # the current stream is behind when backward is called
            busy = (busy @ busy).mul_(1 / 4096)
        logp.backward(up)
        del logp
        with torch.cuda.stream(side):  # takes the memory that has become free on the side stream
            held = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (T * 32,) * 8]
        torch.cuda.synchronize()
        assert torch.equal(x.grad, want), rep
        del held
