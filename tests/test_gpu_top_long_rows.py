"""Rows so long that several chunks share one maximum of their own: many rows, few that are cut, and some that are not; and the
largest vocabulary.  Alternatives of every row against a stable sort, a few rows' numbers and gradients against the oracle
(bounds: tests/test_gpu_top.py)."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from oracle import top as oracle_top
from tests.test_gpu_top import BF16, E, F32, bounds

pytestmark = pytest.mark.gpu


def rows_of(kind, T, V, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((T, V), generator=g, device="cuda").mul_(2)
    if kind == "ties":
        x.round_()
    elif kind == "clustered":
        at = torch.randint(0, V - 3000, (T, 1), generator=g, device="cuda")
        x.scatter_add_(1, at + torch.arange(3000, device="cuda"), torch.full((T, 3000), 12.0, device="cuda"))
    elif kind == "last":  # the largest words at the row's end, the masked ones before them
        x[:, V // 2:-300] = -float("inf")
        x[:, -40:] += 20
    return x.to(dtype)


@pytest.mark.parametrize("kind", ["normal", "ties", "clustered", "last"])
@pytest.mark.parametrize("T,V,dtype", [(401, 140003, F32), (430, 300001, BF16), (49, 2100001, F32), (60, 1100007, BF16),
                                       (1, 4194304, F32), (2, 4194304, BF16), (49, 4194303, BF16)], ids=str)
def test_alternatives_and_numbers(T, V, dtype, kind):
    x = rows_of(kind, T, V, dtype, V)
    act = torch.randint(0, V, (T,), device="cuda", generator=torch.Generator("cuda").manual_seed(T)).int()
    act[::2] = x[::2].argmax(1).int()
    some = sorted({0, T // 2, T - 1})
    for n, tau in ((20, 1.0), (64, 0.7)):
        logp, ent, ids, top, rows = grpo.grpo_token_logp_top(x, act, n, temperature=tau)
        for t in range(T):
            want = torch.sort(x[t], descending=True, stable=True).indices[:n]
            assert torch.equal(ids[t].long(), want), t
        up = [torch.linspace(0.5, 1.5, T, device="cuda"), torch.full((T,), 0.3, device="cuda"),
              torch.linspace(-1, 1, T * n, device="cuda").view(T, n)]
        d = grpo.grpo_token_logp_top_bwd(x, act, ids, rows, *up)
        tau = float(np.float32(tau))
        half = torch.finfo(dtype).eps / 2
        for t in some:
            z, a = x[t].double().cpu().numpy(), int(act[t])
            lp, h, want_ids, want_top, every = oracle_top.row(z, a, n, tau)
            s, he, k, ls = bounds(z, every, tau)
            got = [(float(logp[t]), lp)] if np.isfinite(lp) else []
            for p, q in got + list(zip(top[t].tolist(), want_top)):
                assert abs(p - q) <= s + 1.01 * E * abs(q), (t, p, q)
            assert np.isfinite(lp) or float(logp[t]) == lp
            assert abs(float(ent[t]) - h) <= he + 1.01 * E * h, t
            dl, de, dt = float(up[0][t]), float(up[1][t]), up[2][t].double().cpu().numpy()
            want = oracle_top.gradient(every, h, a, want_ids, dl, de, dt, tau)
            C, Ca = dl + dt.sum(), abs(dl) + np.abs(dt).sum()
            p, l = np.exp(every), np.where(np.isinf(every), 0.0, every)
            l2 = (2 * k + np.abs(l) / np.log(2) + ls) * E * np.log(2) + s
            size = np.abs(C + de * h) + np.abs(de * l)
            bound = p / tau * (size * (l2 + 8 * E) + de * (l2 + he) + (Ca + de * h) * 4 * E)
            bound += np.abs(want) * half + 2.0**-126 * (Ca + de * (1 + h)) * 256 / tau
            special = list(want_ids) + [a]
            bound[special] += np.abs(want[special]) * 2 * E + 1e-13 * (Ca + de) / tau
            off = np.abs(d[t].double().cpu().numpy() - want)
            assert (off <= 1.01 * bound).all(), (t, int(np.argmax(off - bound)), off.max())
