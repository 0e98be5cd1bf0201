"""Long rows of few distinct values, whose words' weights are all rounded the same way: log-probs and entropies as near to the
definition in 64 bits as those of short rows.

As tests/test_gpu_top.py derives its bounds, with the sums that are fp32: those of 32 words at most.  With e = 2^-24, t =
log2(e) (z - max) / tau: a term is off by (3 |t| ln 2 + 2) e, a sum of 32 by 32 e, one raised maximum 4 e and 4 e for the rest;
log S by s = (3 ln2 E|t| + 42) e, the entropy by s and the moment's (3 ln2 E|t|^2 + 46 E|t|) ln2 e and s E|t| ln2.
"""
import math

import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_top import BF16, F32

pytestmark = pytest.mark.gpu

E = 2.0**-24


@pytest.mark.parametrize("T,V,dtype", [(402, 200000, F32), (402, 200000, BF16), (49, 2100001, F32), (1, 4194304, F32),
                                       (2, 4194304, BF16), (420, 1500000, F32), (60, 151936, BF16)], ids=str)
def test_two_values(T, V, dtype):
    g = torch.Generator("cuda").manual_seed(V)
    act = torch.zeros(T, dtype=torch.int32, device="cuda")
    some = sorted({0, T // 2, T - 1})
    for lower, share in ((-0.3, 0.5), (-1.7, 0.9), (-0.0123, 0.1), (-5.3, 0.999)):
        x = torch.empty((T, V), dtype=dtype, device="cuda")
        for t in range(T):
            x[t] = torch.where(torch.rand(V, generator=g, device="cuda") < share, 1.0 + lower, 1.0).to(dtype)
        for tau in (1.0, 0.7):
            logp, ent, _, top, _ = grpo.grpo_token_logp_top(x, act, 3, temperature=tau)
            for t in some:
                z = x[t].double() / float(torch.tensor(tau, dtype=F32))
                lp = torch.log_softmax(z, 0)
                p = lp.exp()
                k = (z.max() - z) / math.log(2)
                m1, m2 = float((p * k).sum()), float((p * k * k).sum())
                s = (3 * math.log(2) * m1 + 42) * E
                h = s + math.log(2) * ((3 * math.log(2) * m2 + 46 * m1) * E + m1 * s)
                want = float(-(p * lp).sum())
                for got, w in ((logp[t], lp[0]), (top[t, 0], lp.max()), (top[t, 2], lp.max())):
                    assert abs(float(got) - float(w)) <= s + 1.01 * E * abs(float(w)), (lower, tau, t, float(got) - float(w), s)
                assert abs(float(ent[t]) - want) <= h + 1.01 * E * want, (lower, tau, t, float(ent[t]) - want, h)
