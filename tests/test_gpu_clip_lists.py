"""Plain lists of gradients beside a GradList: refused while a graph is captured, which goes on."""
import pytest
import torch

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu


def test_a_plain_list_in_a_capture_is_refused():
    g = torch.full((1000,), 0.5, device="cuda")
    out = torch.empty_like(g)
    lst = grpo.GradList([g], out=[out])
    grpo.grpo_clip_grad_norm_(lst, 1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: grpo.GradList([g]), lambda: grpo.grpo_clip_grad_norm_([g], 1.0),
                     lambda: grpo.grpo_grad_sumsq([g]), lambda: grpo.grpo_clip_grad_norm_([], 1.0)):
            with pytest.raises(RuntimeError, match="captured"):
                call()
        grpo.grpo_clip_grad_norm_(lst, 1.0)
    for v in (0.5, 2.0, 0.001):
        g.fill_(v)
        norm = v * 1000**0.5
        want = v * min(1.0, 1.0 / (norm + 1e-6))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert ((out - want).abs() <= 1e-6 * want).all() and (g == g[0]).all()
