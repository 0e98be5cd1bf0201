"""Short rows of which there are many (one wave to a row): reports and gradients against the oracle, as tests/test_gpu_top.py
derives their bounds, and against the same rows in a call of few."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_top import BF16, F32, KINDS, actions, check, make

pytestmark = pytest.mark.gpu

T = 2100


@pytest.mark.parametrize("kind", KINDS + ["masked"])
@pytest.mark.parametrize("V,dtype", [(300, BF16), (521, F32), (2048, F32), (4090, BF16)], ids=str)
def test_values(V, dtype, kind):
    logits, z = make(kind, T, V, dtype, V)
    act = actions(z, V)
    for n, tau in ((8, "rows"), (48, 1.0)):
        check(logits, z, act, n, tau, flags_want=grpo.GRPO_FLAG_NONFINITE if kind == "masked" else 0)


@pytest.mark.parametrize("V", [1, 5, 8, 63, 65, 1003])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_sizes(V, dtype):
    logits, z = make("normal", T, V, dtype, V, V + 5)
    act = actions(z, 2)
    act[::7] = -1
    for n in (0, 1, 33):
        check(logits, z, act, n, 0.8, flags_want=grpo.GRPO_FLAG_ACTION)
    check(logits, z, act, 33, 0.8, in_place=True, flags_want=grpo.GRPO_FLAG_ACTION)


def test_the_alternatives_of_few_and_of_many_rows():
    """Ids and flags of a row do not depend on how many rows a call has."""
    for kind in ("ties", "clustered", "equal"):
        logits, z = make(kind, T, 2000, BF16, 3)
        act = torch.zeros(T, dtype=torch.int32, device="cuda")
        many = grpo.grpo_token_logp_top(logits, act, 40)
        for r in (0, 700, T - 50):
            few = grpo.grpo_token_logp_top(logits[r:r + 50], act[:50], 40)
            assert torch.equal(few[2], many[2][r:r + 50]), kind
            assert np.allclose(few[3].cpu(), many[3][r:r + 50].cpu(), rtol=1e-5, atol=1e-5)
