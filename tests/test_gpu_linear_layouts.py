"""How results of the product lie, and what lies beside them: dW's strides by W's layout, the columns beside a residual and a result
in wider rows, and dbias within the partial sums' own length (64 rows in fp32, joined in fp64)."""
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_linear import ACTS, BF16, E, F32, act64, half, tensors, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("ldw", [0, 1047])
@pytest.mark.parametrize("M", [3, 130])
def test_dw_lies_as_w(M, w, ldw):
    K, N = 264, 520
    x, wt, b, _, dy = tensors(M, K, N, w, F32, ldw=ldw)
    _, dw, _ = grpo.grpo_linear_bwd(dy, x, wt)
    assert dw.shape == (K, N) and dw.stride() == ((N, 1) if w == "kn" else (1, K))
    into = torch.full((K, N) if w == "kn" else (N, K), float("nan"), device="cuda")
    _, got, _ = grpo.grpo_linear_bwd(dy, x, wt, dw=into if w == "kn" else into.t())
    assert got.data_ptr() == into.data_ptr() and got.stride() == dw.stride() and torch.equal(got.to(BF16), dw)


@pytest.mark.parametrize("M,K,N", [(3, 264, 520), (300, 264, 520), (33, 100, 131), (1, 72, 9), (700, 65, 33)])
@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("out", [F32, BF16], ids=str)
def test_columns_beside_the_result_and_the_residual(M, K, N, w, out):
    x, wt, b, res, _ = tensors(M, K, N, w, F32, out)
    want, _ = grpo.grpo_linear(x, wt, b, res, act="gelu", out_dtype=out)
    left, wide, other = 7, torch.full((M, N + 30), 5.0, device="cuda").to(out), torch.full((M, N + 11), 6.0, device="cuda").to(out)
    y, r = wide[:, left:left + N], other[:, 3:3 + N]
    r.copy_(res)
    before = other.clone()
    grpo.grpo_linear(x, wt, b, r, act="gelu", out=y)
    assert torch.equal(y, want) and torch.equal(other, before)
    assert (wide[:, :left] == 5).all() and (wide[:, left + N:] == 5).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N", [(16, 40), (17, 300), (1113, 2856), (4001, 3584), (8000, 1024), (70000, 264)])
def test_dbias_within_its_partial_sums(M, N, act):
    """z is given, so that dz is off by the slope's own error (tests/test_gpu_linear.py: 16 e (1 + |z| + |z|^3 / 8)) and two
    roundings; a thread adds 8 rows of 64 and eight threads' sums are joined in fp32: at most 16 additions."""
    g = torch.Generator("cuda").manual_seed(M + N)
    x, w = torch.zeros((M, 8), dtype=BF16, device="cuda"), torch.zeros((8, N), dtype=BF16, device="cuda")
    dy = torch.randn((M, N), generator=g, device="cuda") + 0.5
    z = None if act == "none" else torch.randn((M, N), generator=g, device="cuda") * 2
    db = torch.full((N,), float("nan"), device="cuda")
    grpo.grpo_linear_bwd(dy, x, w, z, act=act, dx=False, dw=False, dbias=db)
    slope, own = torch.ones((), dtype=torch.float64, device="cuda"), torch.zeros((), dtype=torch.float64, device="cuda")
    if act != "none":
        t = z.double().requires_grad_()
        (slope,) = torch.autograd.grad(act64(act, t).sum(), t)
        if act != "relu":
            own = 16 * E * (1 + z.double().abs() + z.double().abs()**3 / 8)
    dz = dy.double() * slope
    bound = (dy.double().abs() * own + 2 * E * dz.abs()).sum(0) + 16 * E * dz.abs().sum(0)
    within(db, dz.sum(0), 1.01 * (bound + half(F32) * dz.sum(0).abs()) + 1e-30, "dbias")
