"""bf16 rows whose logits are all negative, at temperatures that put zero far above their maximum: 2^1024 of its weight and
more.  Tolerances are those of test_gpu_sampling.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sampled_logp import actions, check as check_logp
from tests.test_gpu_sampling import BF16, check, uniform

pytestmark = pytest.mark.gpu


def tau_of(octaves, top=1.0):
    """The temperature at which a logit of 2^-15 weighs 2^octaves of one at -top."""
    return float(np.float32((top + 2.0**-15) * np.log2(np.e) / octaves))


@pytest.mark.parametrize("octaves", [100.0, 1023.0, 1024.0, 1024.4, 1025.0, 2048.0, 3072.2, 1e5])
@pytest.mark.parametrize("T,V", [(2, 9001), (260, 20000)])
def test_all_negative(T, V, octaves):
    rng = np.random.default_rng(int(octaves))
    # at -1 a few, the others a little lighter or far below
    z = -1.0 - 2.0**-7 * rng.integers(0, 40, (T, V)) * (rng.random((T, V)) < 0.9)
    x = torch.from_numpy(z).to(BF16)
    z = x.double().numpy()
    assert z.max() == -1.0
    for par in (dict(top_p=0.4), dict(top_k=V // 2, top_p=0.3), dict(min_p=0.5), dict(top_k=V - 100)):
        par = dict(par, temperature=tau_of(octaves))
        check(x.cuda(), z, par, uniform(z, par, 1), V)
        check_logp(x.cuda(), z, par, actions(z, par, 2), V)
