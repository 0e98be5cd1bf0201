"""SampledLogp captured into a graph, forward and backward, and replayed; and calls of more rows than one launch takes."""
import pytest
import torch

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("par", [dict(temperature=0.8), dict(temperature=0.9, top_k=40, top_p=0.95)], ids=str)
def test_captured_forward_and_backward(dtype, par):
    T, V, ld = 33, 4990, 5000
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(T, ld, device="cuda", generator=gen).to(dtype).requires_grad_()
    act = x.detach()[:, :V].argmax(1).to(torch.int32)
    up = torch.randn(T, device="cuda", generator=gen)

    def step():
        logp = grpo.SampledLogp.apply(x, act, dict(par, V=V))
        (d,) = torch.autograd.grad(logp, x, up)
        return logp.detach(), d

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for rep in range(4):
        with torch.no_grad():
            x.mul_(0.9)
            up.mul_(-1.1)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in got:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rep
        assert not got[1][:, V:].any()


@pytest.mark.parametrize("par", [{}, dict(top_k=2), dict(top_p=0.6)], ids=str)
def test_more_rows_than_a_launch_takes(par):
    """2^20 + 77 rows repeat the first 1,000, and so do their outputs."""
    n, T, V = 1000, (1 << 20) + 77, 5
    gen = torch.Generator("cuda").manual_seed(4)
    few, u = torch.randn(n, V, device="cuda", generator=gen), torch.rand(n, device="cuda", generator=gen)
    at = torch.arange(T, device="cuda") % n
    want = grpo.grpo_sample(few, u, **par)
    many = few[at].contiguous()
    for a, b in zip(grpo.grpo_sample(many, u[at].contiguous(), **par), want):
        assert torch.equal(a, b[at])
    up = torch.randn(n, device="cuda", generator=gen)
    lp, k, rows = grpo.grpo_sampled_logp(few, want[0], **par)
    lp2, k2, rows2 = grpo.grpo_sampled_logp(many, want[0][at].contiguous(), **par)
    assert torch.equal(lp2, lp[at]) and torch.equal(k2, k[at]) and torch.equal(rows2, rows[at])
    d = grpo.grpo_sampled_logp_bwd(few, want[0], rows, up)
    assert torch.equal(grpo.grpo_sampled_logp_bwd(many, want[0][at].contiguous(), rows2, up[at].contiguous()), d[at])
