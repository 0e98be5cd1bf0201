"""Rows of up to 2^22 words that weigh about the same, so that one bin of weight holds most of a row: its integer sum has to
hold all of them.  Tolerances are those of test_gpu_sampling.py; a share's sum over 2^22 words is off by 1.2e-13 of itself at
most, 5e-7 of a word, and u lies 1e-9 off the borders of the cdf."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_sampled_logp import actions, check as check_logp
from tests.test_gpu_sampling import BF16, F32, check, uniform

pytestmark = pytest.mark.gpu

MOST = grpo.GRPO_SAMPLING_MAX_V


def row(kind, V):
    rng = np.random.default_rng(V)
    if kind == "equal":
        return np.full((1, V), 1.5)
    if kind == "zeros":
        return np.zeros((1, V))
    if kind == "two":  # three words in four at 5, the others a factor e lighter
        return np.where(np.arange(V) % 4 == 1, 4.0, 5.0)[None]
    if kind == "close":  # words of one bin, told apart
        return rng.normal(0, 1e-3, (1, V))
    if kind == "above_zero":  # three words in four at zero, the others likelier
        return np.where(np.arange(V) % 4 == 1, 1.0, 0.0)[None]
    raise AssertionError(kind)


def on_gpu(z, dtype):
    x = torch.from_numpy(z).to(dtype)
    return x.cuda(), x.double().numpy()


@pytest.mark.parametrize("V", [1 << 21, MOST - 3, MOST])
@pytest.mark.parametrize("kind", ["equal", "zeros", "two"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_shares_of_equal_words(dtype, kind, V):
    logits, z = on_gpu(row(kind, V), dtype)
    for par in (dict(top_p=0.9), dict(top_k=V - 5, top_p=0.77)):
        check(logits, z, par, uniform(z, par, 1), V)
    check_logp(logits, z, par, actions(z, par, 2), V)


def test_shares_of_words_in_one_bin():
    for V in (1 << 21, MOST):
        logits, z = on_gpu(row("close", V), F32)
        for par in (dict(top_p=0.9), dict(top_k=V // 2 + 1, top_p=0.3, temperature=0.5)):
            check(logits, z, par, uniform(z, par, 1), V)


@pytest.mark.parametrize("kind", ["equal", "two"])
def test_many_such_rows(kind):
    """Rows whose tiles are not reduced by a launch of their own: each as a single one's."""
    T, V = 65, MOST
    logits, z = on_gpu(row(kind, V), F32)
    par = dict(top_p=0.9)
    u = uniform(z, par, 1)
    check(logits, z, par, u, V)
    want = grpo.grpo_sample(logits, torch.from_numpy(u).cuda(), **par)
    rows = logits.expand(T, V).contiguous()
    got = grpo.grpo_sample(rows, torch.from_numpy(u).cuda().expand(T).contiguous(), **par)
    for a, b in zip(got, want):
        assert (a == b).all()


@pytest.mark.parametrize("V", [1 << 21, MOST - 3, MOST])
def test_many_zeros_below_the_cut(V):
    """bf16 words too small to be told apart are weighed together; the cut is among likelier ones, or takes them all."""
    logits, z = on_gpu(row("above_zero", V), BF16)
    for par in (dict(top_p=0.4), dict(min_p=0.3), dict(top_p=0.3, min_p=0.2, temperature=2.0),
                dict(top_k=V // 5, top_p=0.7)):
        check(logits, z, par, uniform(z, par, 1), V)
        check_logp(logits, z, par, actions(z, par, 2), V)
