"""bf16 rows with live words beyond the size at which values are counted, cut by a share of the weight whose sum is not known
beforehand.  Tolerances are those of test_gpu_sampling.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sampled_logp import actions, check as check_logp
from tests.test_gpu_sampling import BF16, check, uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["third_at_-1e4", "one_below", "all_above", "far_apart", "cut_at_zero"])
@pytest.mark.parametrize("T,V", [(2, 9001), (3, 151936), (260, 17001), (520, 9000)])
def test_shares(T, V, kind):
    rng = np.random.default_rng(V)
    z = rng.normal(0, 2, (T, V))
    if kind == "third_at_-1e4":
        z[:, ::3] = -1e4
    elif kind == "one_below":
        z[:, 5] = -70.0
    elif kind == "all_above":
        z += 70.0
    elif kind == "far_apart":
        z *= 100.0
    else:  # words too small to be told apart by value, each beside the cut
        z = np.where(rng.random((T, V)) < 0.9, z * 2.0**-18, np.abs(z) * 0.1)
    x = torch.from_numpy(z).to(BF16)
    z = x.double().numpy()
    pars = (dict(top_p=0.9), dict(top_p=0.3, temperature=1.4), dict(top_p=0.999, min_p=0.02), dict(top_k=V // 2, top_p=0.6))
    for par in pars if T < 10 else pars[:1]:
        check(x.cuda(), z, par, uniform(z, par, 1), V)
        check_logp(x.cuda(), z, par, actions(z, par, 2), V)
