"""Operands of the product that are columns of one buffer, whose rows lie in turn, give what operands of their own give; ones that
share elements are refused, and nothing is written."""
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_linear import BF16, F32, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 40), (9, 72, 128), (300, 264, 520), (70, 99, 131)])
def test_columns_of_one_buffer(M, K, N, w):
    x, wt, b, res, dy = tensors(M, K, N, w, F32)
    want = grpo.grpo_linear(x, wt, b, res, act="silu", keep_z=True)
    grads = grpo.grpo_linear_bwd(dy, x, wt, want[1], act="silu", dbias=torch.empty_like(b))
    wide = torch.full((M, K + 3 * N), 3.0, dtype=BF16, device="cuda")
    xs, rs, ys, ds = wide.split([K, N, N, N], dim=1)
    xs.copy_(x), rs.copy_(res), ds.copy_(dy)
    got = grpo.grpo_linear(xs, wt, b, rs, act="silu", out=ys, keep_z=True)
    assert torch.equal(ys, want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(xs, x) and torch.equal(rs, res) and torch.equal(ds, dy)
    again = grpo.grpo_linear_bwd(ds, xs, wt, got[1], act="silu", dbias=torch.empty_like(b))
    assert all(torch.equal(p, q) for p, q in zip(again, grads))


def test_shared_elements_are_refused():
    M, K, N = 40, 64, 64
    x, w, b, res, dy = tensors(M, K, N, "kn", BF16)
    flat = torch.full((M * N + 64,), 2.0, dtype=BF16, device="cuda")
    y = flat[:M * N].view(M, N)
    for bad in (dict(residual=flat[8:8 + M * N].view(M, N), out=y), dict(residual=flat[N:N + M * N].view(M, N), out=y),
                dict(residual=res, out=x), dict(residual=res, out=w[:M]), dict(residual=res, out=y, bias=y[3])):
        with pytest.raises(grpo.GrpoError):
            grpo.grpo_linear(x, w, **bad)
    for bad in (dict(dx=dy), dict(dx=x), dict(dw=w), dict(dbias=dy[1])):
        with pytest.raises(grpo.GrpoError):
            grpo.grpo_linear_bwd(dy, x, w, **bad)
    assert (flat == 2.0).all()
    grpo.grpo_linear(x, w, b, y, out=y)  # y itself is in order
