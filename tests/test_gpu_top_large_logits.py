"""Finite rows whose exponents pass fp32's range, (max - z) log2(e) / tau > 3.4e38: reports and gradients against the oracle, with
the bounds of tests/test_gpu_top.py (a word that far below the maximum weighs 0 on both sides)."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_top import BF16, F32, check, make

pytestmark = pytest.mark.gpu


def large(T, V, dtype, big):
    """Normal logits; in turn a row has one word at `big`, several below it, one beside words next to the mask, two equal ones,
    masked words beside it, and none."""
    _, z = make("normal", T, V, F32, V)
    rng = np.random.default_rng(T)
    at = rng.integers(0, V - 8, T)
    for t in range(T):
        kind, a = t % 6, at[t]
        if kind < 5:
            z[t, a] = big
        if kind == 1:
            z[t, a + 1:a + 8] = big * np.linspace(0.99, 0.4, 7)
        elif kind == 2:
            z[t, :a:3] = -9e7
        elif kind == 3:
            z[t, a + 5] = big
        elif kind == 4:
            z[t, a + 1::2] = -np.inf
    x = torch.from_numpy(z).to(dtype)
    return x.cuda(), x.double().numpy(), at


# one wave to a row, 256 threads, rows cut into parts, 1,024 threads, and 256 to long rows
@pytest.mark.parametrize("T,V", [(2100, 500), (7, 3000), (7, 40000), (60, 20003), (410, 17001)])
@pytest.mark.parametrize("big,tau", [(3e38, 1.0), (3e32, 1e-6), (2.5e38, 0.8), (1e30, 1e-6)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_words_far_below_the_maximum(T, V, big, tau, dtype):
    logits, z, at = large(T, V, dtype, big)
    act = np.where(np.arange(T) % 2 == 0, at, np.argmax(z == 0.0, axis=1))
    for n, ups in ((9, (True, True, True)), (9, (True, False, True)), (0, (True, True, False))):
        check(logits, z, act, n, tau, ups=ups)


@pytest.mark.parametrize("T,V", [(2100, 500), (7, 3000), (7, 40000), (60, 20003)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_an_action_whose_log_prob_passes_fp32_is_no_masked_word(T, V, dtype):
    """Its log-prob is -inf; the gradient is that of a word of weight 0, d / tau, against the largest word's -d / tau (one
    rounding of each to the type, two of fp32 before it); a masked action's is 0."""
    tau, big = float(np.float32(1e-6)), 1e38
    x, z, at = large(T, V, dtype, big)
    act = torch.zeros(T, dtype=torch.int32, device="cuda")
    some = [t for t in range(T) if t % 6 in (0, 1) and at[t] > 0]
    x[some[0], 0] = -float("inf")
    logp, ent, ids, _, rows = grpo.grpo_token_logp_top(x, act, 2, temperature=tau)
    up = torch.linspace(0.5, 2.0, T, device="cuda")
    d = grpo.grpo_token_logp_top_bwd(x, act, ids, rows, up, None, None).double().cpu().numpy()
    half = torch.finfo(dtype).eps / 2
    for t in some:
        want = np.zeros(V)
        if t != some[0]:
            want[0], want[at[t]] = float(up[t]) / tau, -float(up[t]) / tau
        assert logp[t] == -float("inf") and ent[t] == 0
        assert (np.abs(d[t] - want) <= 1.01 * (half + 2 * 2.0**-24) * np.abs(want)).all(), t
