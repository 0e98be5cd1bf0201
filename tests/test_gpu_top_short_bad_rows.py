"""One wave to a row: rows with a NaN, +inf, no words or a temperature out of range beside ordinary ones, and ids that the caller
brings."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from oracle import top as oracle_top
from tests.test_gpu_top import BF16, E, F32, bounds, make

pytestmark = pytest.mark.gpu

T = 2100
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("V", [1, 7, 500, 2041])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_bad_rows(V, dtype):
    logits, _ = make("normal", T, V, dtype, 1)
    clean, n = logits.clone(), min(6, V)
    bad = {1: NAN, 700: INF, 1402: -INF, 2099: NAN}
    for t, v in bad.items():
        logits[t, V // 3] = v
    logits[1402] = -INF
    temp = torch.ones(T, device="cuda")
    wrong = {3: 0.0, 701: NAN, 1403: 2e6, 2098: -1.0}
    for t, v in wrong.items():
        temp[t] = v
    act = torch.zeros(T, dtype=torch.int32, device="cuda")
    act[5] = V
    act[6] = -3
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    logp, ent, ids, top, rows = grpo.grpo_token_logp_top(logits, act, n, temperature=temp, error_flags=flags)
    assert flags.item() == grpo.GRPO_FLAG_ACTION | grpo.GRPO_FLAG_NONFINITE | grpo.GRPO_FLAG_SETTING
    one = torch.ones(T, device="cuda")
    d = grpo.grpo_token_logp_top_bwd(logits, act, ids, rows, one, one, one[:, None].expand(T, n).contiguous())
    gone = [1, 700, 2099, *wrong]
    assert ent[gone].isnan().all() and top[gone].isnan().all() and (ids[gone] == -1).all() and logp[gone].isnan().all()
    assert d[gone].isnan().all()
    assert logp[1402] == -INF and ent[1402] == 0 and (top[1402] == -INF).all() and (ids[1402] == -1).all() and not d[1402].any()
    assert logp[5] == 0 and logp[6] == 0
    rest = torch.tensor([t for t in range(T) if t not in gone and t != 1402], device="cuda")
    want = grpo.grpo_token_logp_top(clean, act, n)
    for p, q in zip((logp, ent, ids, top, rows), want):
        assert torch.equal(p[rest], q[rest])
    assert d[rest].isfinite().all()


@pytest.mark.parametrize("V", [12, 700, 2041])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_ids_of_the_callers_own(V, dtype):
    """The same id twice adds up; ids outside [0, V) count for nothing, their gradients unread."""
    logits, z = make("normal", T, V, dtype, 2)
    act = torch.full((T,), 5, dtype=torch.int32, device="cuda")
    rows = grpo.grpo_token_logp_top(logits, act, 0)[4]
    ids = torch.tensor([[5, 5, 2, 2, V, -7, V - 1, 2]] * T, dtype=torch.int32, device="cuda")
    up = torch.tensor([[0.5, 1.5, 2, 3, NAN, INF, -1, 4]] * T, device="cuda")
    d = grpo.grpo_token_logp_top_bwd(logits, act, ids, rows, torch.ones(T, device="cuda"), None, up).double().cpu().numpy()
    half = torch.finfo(dtype).eps / 2
    for t in range(0, T, 60):
        _, h, _, _, every = oracle_top.row(z[t], 5, 0)
        want = oracle_top.gradient(every, h, 5, [5, 2, V - 1], 1.0, 0.0, [2.0, 9.0, -1.0])
        s = bounds(z[t], every, 1.0)[0]
        assert (np.abs(d[t] - want) <= np.exp(every) * 13 * (s + 60 * E) + (2 * E + half) * np.abs(want)).all(), t
