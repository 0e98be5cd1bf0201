"""Products whose sum is split over workgroups: the epilogue, z and an accumulated dW come after the splits' join; bounds as in
tests/test_gpu_linear.py."""
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_linear import BF16, F32, check, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M,K,N", [(4096, 64, 128), (2000, 40, 24), (9, 8192, 64), (100, 8000, 72), (130, 5000, 131), (31, 4096, 3)])
def test_sums_far_longer_than_the_result(M, K, N, w):
    check(M, K, N, "gelu", w, F32, True, F32, dw_dtype=F32)
    check(M, K, N, "silu", w, BF16, True, BF16, seed=1)
    check(M, K, N, "none", w, None, False, BF16, dw_dtype=F32, seed=2)


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M,N", [(2, 126224), (20, 20001)])
def test_dx_over_a_vocabulary(M, N, w):
    check(M, 24, N, "none", w, BF16, False, BF16)


def test_the_same_bits_every_time():
    for M, K, N in ((5, 8192, 64), (64, 8192, 256), (3000, 96, 96)):
        x, w, b, res, dy = tensors(M, K, N, "kn", F32)
        first = grpo.grpo_linear(x, w, b, res, act="silu", keep_z=True)
        grads = grpo.grpo_linear_bwd(dy, x, w, first[1], act="silu", dbias=torch.empty_like(b))
        for _ in range(4):
            again = grpo.grpo_linear(x, w, b, res, act="silu", keep_z=True)
            assert all(torch.equal(p, q) for p, q in zip(first, again))
            more = grpo.grpo_linear_bwd(dy, x, w, first[1], act="silu", dbias=torch.empty_like(b))
            assert all(torch.equal(p, q) for p, q in zip(grads, more))
