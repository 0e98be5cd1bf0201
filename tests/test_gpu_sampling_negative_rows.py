"""bf16 rows whose logits are all negative, at temperatures that put zero far above their maximum, 2^1024 of its weight and
more; and rows whose largest words are below 2^-15 in size, at temperatures that tell these apart.  Tolerances are those of
test_gpu_sampling.py."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_sampled_logp import actions, check as check_logp
from tests.test_gpu_sampling import BF16, check, uniform

pytestmark = pytest.mark.gpu


def tau_of(octaves, top=1.0):
    """The temperature at which a logit of 2^-15 weighs 2^octaves of one at -top."""
    return float(np.float32((top + 2.0**-15) * np.log2(np.e) / octaves))


@pytest.mark.parametrize("octaves", [100.0, 1023.0, 1024.0, 1024.4, 1025.0, 2048.0, 5120.2, 1e5])
@pytest.mark.parametrize("T,V", [(2, 9001), (260, 20000)])
def test_all_negative(T, V, octaves):
    rng = np.random.default_rng(int(octaves))
    # at -1 a few, the others a little lighter or far below
    z = -1.0 - 2.0**-7 * rng.integers(0, 40, (T, V)) * (rng.random((T, V)) < 0.9)
    x = torch.from_numpy(z).to(BF16)
    z = x.double().numpy()
    assert z.max() == -1.0
    pars = (dict(top_p=0.4), dict(top_k=V // 2, top_p=0.3), dict(min_p=0.5), dict(top_k=V - 100))
    for par in pars if T < 10 else pars[:1]:
        par = dict(par, temperature=tau_of(octaves))
        check(x.cuda(), z, par, uniform(z, par, 1), V)
        check_logp(x.cuda(), z, par, actions(z, par, 2), V)


@pytest.mark.parametrize("tau", [1e-6, 1.7e-6, 4e-6, 1.5e-5, 1e-4, 1.0])
@pytest.mark.parametrize("kind", ["below_zero", "around_zero", "zeros", "likelier_beside"])
def test_largest_words_near_zero(kind, tau):
    T, V, times = 3, 17001, 100
    rng = np.random.default_rng(V)
    if kind == "below_zero":
        z = -np.abs(rng.normal(0, 1, (T, V))) * 10.0 ** rng.uniform(-7, 0, (T, 1))
    elif kind == "around_zero":
        z = rng.normal(0, 2.0**-17, (T, V))
    elif kind == "zeros":
        z = np.where(rng.random((T, V)) < 0.5, 0.0, -1.0)
    else:
        z = np.where(rng.random((T, V)) < 0.9, rng.normal(0, 2.0**-17, (T, V)), rng.normal(0, 2.0**-13, (T, V)))
    x = torch.from_numpy(z).to(BF16)
    z = x.double().numpy()
    x = x.cuda()
    for par in (dict(top_k=V - 1), dict(min_p=1e-18), dict(top_k=V // 2, top_p=0.3), dict(top_p=0.9), dict(top_p=1 - 2.0**-23),
                dict(min_p=0.05)):
        par = dict(par, temperature=tau)
        u = uniform(z, par, 1)
        check(x, z, par, u, V)
        check_logp(x, z, par, actions(z, par, 2), V)
        # as rows of many, which smaller workgroups take
        u = torch.from_numpy(u).cuda()
        want, got = grpo.grpo_sample(x, u, **par), grpo.grpo_sample(x.repeat(times, 1), u.repeat(times), **par)
        assert torch.equal(got[0], want[0].repeat(times)) and torch.equal(got[2], want[2].repeat(times))
        assert ((got[1] - want[1].repeat(times)).abs() <= 2.0**-23 * want[1].abs().repeat(times) + 1e-12).all()
