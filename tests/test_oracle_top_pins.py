"""The oracle of log-probs, entropy and alternatives: hand values, central differences, torch's own derivative."""
import numpy as np
import pytest
import torch

from oracle import top


def test_hand_values():
    z = np.log([1.0, 2.0, 1.0, 4.0]) + 3
    lp, h, ids, tlp, _ = top.row(z, 1, 3)
    assert lp == pytest.approx(np.log(0.25)) and ids.tolist() == [3, 1, 0]
    assert h == pytest.approx(-(0.25 * np.log(0.125) + 0.25 * np.log(0.25) + 0.5 * np.log(0.5)))
    assert tlp == pytest.approx(np.log([0.5, 0.25, 0.125]))
    assert top.row(2 * z, 1, 0, tau=2.0)[0] == pytest.approx(np.log(0.25))


def test_masks_ties_and_few_words():
    z = np.array([0.0, -1e8, 1.0, -np.inf, 1.0, -3e38])
    lp, h, ids, tlp, every = top.row(z, 1, 5)
    assert lp == -np.inf and ids.tolist() == [2, 4, 0, -1, -1] and tlp[3] == -np.inf
    assert np.exp(every).sum() == pytest.approx(1)
    lp, h, ids, tlp, _ = top.row(np.full(4, -np.inf), 2, 2)
    assert lp == -np.inf and h == 0 and ids.tolist() == [-1, -1]
    assert top.row(z, 6, 1)[0] == 0.0 and top.row(z, -1, 1)[0] == 0.0


@pytest.mark.parametrize("tau", [0.5, 1.0, 1.7])
def test_gradient(tau):
    rng = np.random.default_rng(3)
    z = rng.normal(size=12)
    z[[3, 8]] = -np.inf
    act, n, up = 5, 4, (0.7, -0.4, rng.normal(size=4))

    def value(z):
        lp, h, _, _, every = top.row(z, act, n, tau)
        return up[0] * lp + up[1] * h + (up[2] * every[ids]).sum()

    lp, h, ids, _, every = top.row(z, act, n, tau)
    d = top.gradient(every, h, act, ids, *up, tau=tau)
    assert d.sum() == pytest.approx(0, abs=1e-12) and not d[[3, 8]].any()
    for v in range(12):
        if np.isfinite(z[v]):
            e = np.zeros(12)
            e[v] = 1e-5
            assert d[v] == pytest.approx((value(z + e) - value(z - e)) / 2e-5, abs=1e-8)
    live = np.flatnonzero(np.isfinite(z))
    t = torch.tensor(z[live], requires_grad=True)
    q = torch.log_softmax(t / tau, 0)
    at = torch.from_numpy(np.searchsorted(live, ids))
    loss = up[0] * q[np.searchsorted(live, act)] + up[1] * torch.special.entr(q.exp()).sum() + (torch.tensor(up[2]) * q[at]).sum()
    (want,) = torch.autograd.grad(loss, t)
    assert d[live] == pytest.approx(want.numpy(), abs=1e-12)


def test_action_masked_or_outside_has_no_gradient_of_its_own():
    z = np.array([0.0, -np.inf, 1.0])
    lp, h, ids, _, every = top.row(z, 1, 1)
    assert not top.gradient(every, h, 1, [], 3.0, 0.0, []).any()
    assert not top.gradient(every, h, 7, [], 3.0, 0.0, []).any()
