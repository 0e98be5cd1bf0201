"""Clipping factors below fp32's normal range: of gradients near its upper end, and of bounds near its lower one.

The factor has 24 bits (2^-24), the product is rounded (2^-24) and for a bf16 out once more (2^-8); below the types' normal
range half a step of the smallest is 2^-150 (fp32) and 2^-134 (bf16, twice rounded: 2^-133)."""
import pytest
import torch

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("n", [7, 5000, 1_000_003])
@pytest.mark.parametrize("scale,max_norm", [(1e38, 1.0), (3e38, 0.01), (1e38, 1e-25), (2e30, 1e-12), (1e-10, 1e-40),
                                            (1.0, 1e-37), (1e38, 1e38)], ids=str)
@pytest.mark.parametrize("src,dst", [(F32, "same"), (BF16, "same"), (F32, BF16), (BF16, F32)], ids=str)
def test_far_factors(src, dst, scale, max_norm, n):
    g = ((torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)) * 2 - 1) * scale).to(src)
    x = g.double()
    norm64 = x.square().sum().sqrt().item()
    f = min(1.0, max_norm / (norm64 + 1e-6))
    out = None if dst == "same" else [torch.full((n,), float("nan"), dtype=dst, device="cuda")]
    flags = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    norm = grpo.grpo_clip_grad_norm_([g], max_norm, out=out, error_flags=flags).item()
    assert flags.item() == 0
    assert norm == float("inf") if norm64 > 3.5e38 else abs(norm - norm64) <= 2.0**-24 * norm64 * 1.01
    got, want = (g if out is None else out[0]), x * f
    half, least = (2.0**-8, 2.0**-133) if got.dtype == BF16 else (0.0, 2.0**-150)
    off = (got.double() - want).abs()
    assert (off <= want.abs() * (2 * 2.0**-24 + half) * 1.01 + least * 1.01).all(), (off / want.abs()).max()


def test_a_factor_just_below_a_power_of_two():
    """Its significand rounds to 1, and it is no factor of 1: gradients in place are scaled."""
    g = torch.full((4,), 2.0**120, device="cuda")  # the norm is 2^121
    grpo.grpo_clip_grad_norm_([g], 2.0**-10 * (1 - 2.0**-40))
    assert torch.equal(g, torch.full((4,), 2.0**-11, device="cuda"))
