"""Rows of one word, or of one that is all but certain: log-probs are at most 0 and entropies at least 0, exactly 0 where the
definition is.

The largest word's weight is 1, so that a sum of weights is at least 1 in any order of additions; the entropy of a row of one
word is the rounding of its one moment alone, 2^-25 of an exponent that is at most 1/4.
"""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_top import BF16, F32

pytestmark = pytest.mark.gpu

SHAPES = [(3000, 700), (200, 3000), (40, 40000), (100, 20003), (500, 17001)]


def temperatures(T, seed):
    tau = np.exp(np.random.default_rng(seed).uniform(np.log(1e-6), np.log(1e3), T)).astype(np.float32)
    tau[::3] = np.float32(1 / 3)
    return tau


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_rows_of_one_word(T, V, dtype):
    rng = np.random.default_rng(V)
    at = rng.integers(0, V, T)
    z = rng.normal(0, 1, T) * 10.0 ** rng.uniform(-3, 6, T)
    x = torch.full((T, V), -float("inf"), dtype=dtype)
    x[torch.arange(T), torch.from_numpy(at)] = torch.from_numpy(z).to(dtype)
    tau = torch.from_numpy(temperatures(T, V)).cuda()
    act = torch.from_numpy(at.astype(np.int32)).cuda()
    logits = x.cuda()
    logp, ent, ids, top, rows = grpo.grpo_token_logp_top(logits, act, 3, temperature=tau)
    assert torch.equal(ids[:, 0], act) and (ids[:, 1:] == -1).all()
    assert not logp.any() and not top[:, 0].any()
    assert (ent >= 0).all() and (ent <= 2.0**-27).all(), ent.max()
    d = grpo.grpo_token_logp_top_bwd(logits, act, ids, rows, torch.ones_like(logp), None, None)
    assert not d.any()  # (1 - p) / tau


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_one_word_that_is_all_but_certain(T, V, dtype):
    rng = np.random.default_rng(T)
    z = rng.normal(0, 2, (T, V))
    at = rng.integers(0, V, T)
    z[np.arange(T), at] += rng.uniform(10, 60, T)
    logits = torch.from_numpy(z).to(dtype).cuda()
    act = logits.argmax(1).int()
    for tau in (1.0, 0.3, torch.from_numpy(temperatures(T, T)).cuda()):
        logp, ent, ids, top, _ = grpo.grpo_token_logp_top(logits, act, 5, temperature=tau)
        assert (logp <= 0).all() and (top <= 0).all() and (ent >= 0).all()
        assert not torch.log1p(-torch.exp(logp.double())).isnan().any()
