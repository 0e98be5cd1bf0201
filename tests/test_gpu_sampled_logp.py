"""Log-probs of given actions under the sampling distribution, and their gradient, against the fp64 oracle.

Counts are equal.  Errors, with e = 2^-24 (half a step of fp32) and t = log2(e) (z - max) / tau a word's exponent:
- log-prob where words are cut off: sums in fp64, one rounding: e |logp| + 1e-12;
- log-prob of a row with nothing cut: terms and sums of a lane's 32 words in fp32.  A term's exponent is off by 3 e |t|
  (the difference, the factor, the product), the term by 2 e more, a sum of 32 by 31 e: weighted over the row, log S is off
  by at most (3 ln2 E|t| + 33) e, with E|t| the mean under the distribution, at most log2(V) + 1;
- d logits: scale P, P = 2^(t - log2 S): exponent off by (3 |t| + |t - log2 S| + |log2 S|) e, exp2 and two products by 4 e
  more, plus S's error above, then one rounding to the type.  The action's own is formed in fp64 from the same S: the
  error of S times P, e of the value.  Below 2^-126 the exponential is 0.
"""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from oracle import sampling as so
from tests.test_gpu_sampling import BF16, F32, make, settings_of, tensors

pytestmark = pytest.mark.gpu

E = 2.0**-24


def s_error(V, cut):
    return 1e-12 if cut else (3 * np.log(2) * (np.log2(V) + 1) + 33) * E


def check(logits, z, par, act, V, dlogits=True, in_place=False, flags_want=None):
    T = z.shape[0]
    dtype = logits.dtype
    half = torch.finfo(dtype).eps / 2
    dlogp = torch.randn(T, generator=torch.Generator().manual_seed(T + V)).cuda()
    a = torch.from_numpy(act.astype(np.int32)).cuda()
    flags = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    logp, n, rows = grpo.grpo_sampled_logp(logits, a, V=V, error_flags=flags, **tensors(par))
    d = grpo.grpo_sampled_logp_bwd(logits, a, rows, dlogp, V=V, dlogits=logits if in_place else True)
    logp, n, d = logp.cpu().numpy(), n.cpu().numpy(), d[:, :V].double().cpu().numpy()
    up = dlogp.double().cpu().numpy()
    want_flag = 0
    for t in range(T):
        st = settings_of(par, t)
        lp, k, dz = so.logp(z[t], int(act[t]), **st)
        cut = 0 < st["top_k"] < V or st["top_p"] < 1 or st["min_p"] > 0 or st["tau"] == 0
        if not 0 <= act[t] < V:
            want_flag |= grpo.GRPO_FLAG_ACTION
            lp, dz = 0.0, np.zeros(V)
        assert n[t] == k, (t, n[t], k)
        err_s = s_error(V, cut)
        if np.isinf(lp):
            assert logp[t] == lp, (t, logp[t])
            dz = np.zeros(V)
        else:
            assert abs(float(logp[t]) - lp) <= E * abs(lp) * 1.01 + err_s, (t, logp[t], lp)
        want = dz * up[t]
        if st["tau"] > 0 and dz.any():
            at, w, top = so.kept(z[t], **st)
            x = np.zeros(V)
            x[at] = np.abs(np.log2(np.e) * (z[t][at] - top) / st["tau"])
            ls = np.log2(w.sum())
            rel = ((4 * x + 2 * ls + 6) * E + err_s) * 1.02
            bound = np.abs(want) * (rel + half) + 2.0**-126 * (abs(up[t] / st["tau"]) + 1)
            p = np.exp(lp)
            i = int(act[t])
            bound[i] = np.abs(want[i]) * (half + 2 * E) + abs(up[t] / st["tau"]) * p * err_s * 1.02 + 1e-14
        else:
            bound = np.zeros(V)
        off = np.abs(d[t] - want)
        assert (off <= bound).all(), (t, int(np.argmax(off - bound)), off.max())
    assert flags.item() == (want_flag if flags_want is None else flags_want)


def actions(z, par, seed):
    """For each row a kept word, for one in five any word."""
    rng = np.random.default_rng(seed)
    act = np.zeros(z.shape[0], np.int64)
    for t in range(z.shape[0]):
        at, w, _ = so.kept(z[t], **settings_of(par, t))
        act[t] = rng.choice(at, p=w / w.sum()) if at.size and rng.random() < 0.8 else rng.integers(0, z.shape[1])
    return act


PARS = [{}, dict(temperature=0.0), dict(temperature=0.6), dict(temperature=1.4, top_k=1), dict(top_k=40),
        dict(top_p=0.9), dict(temperature=0.7, top_k=50, top_p=0.95), dict(min_p=0.05),
        dict(temperature=1.3, top_k=5000, top_p=0.99, min_p=0.001)]


@pytest.mark.parametrize("par", PARS, ids=lambda p: "-".join(f"{k}{v}" for k, v in p.items()) or "off")
@pytest.mark.parametrize("kind", ["normal", "peaked", "ties", "masked"])
@pytest.mark.parametrize("T,V,dtype", [(7, 1024, F32), (3, 2049, BF16), (4, 32003, F32), (3, 151936, BF16)], ids=str)
def test_settings(T, V, dtype, kind, par):
    logits, z = make(kind, T, V, dtype, 3 * V + T)
    check(logits, z, par, actions(z, par, V), V)


@pytest.mark.parametrize("V", [1, 2, 7, 9, 64, 65, 2047, 8192, 8193, 16391])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_sizes(V, dtype):
    for i, par in enumerate([{}, dict(top_k=3), dict(temperature=0.5, top_p=0.8)]):
        logits, z = make("normal", 3, V, dtype, V + i)
        check(logits, z, par, actions(z, par, V + i), V)


@pytest.mark.parametrize("kind", ["equal", "zeros", "near_zero", "far"])
@pytest.mark.parametrize("V", [500, 20001])
def test_values(V, kind):
    for i, par in enumerate([{}, dict(top_k=V // 2), dict(top_p=0.37), dict(min_p=0.2)]):
        logits, z = make(kind, 2, V, F32, V + i)
        check(logits, z, par, actions(z, par, V + i), V)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("ld,offset", [(5003, 1), (5120, 3), (5001, 5)])
def test_strides_alignment_and_in_place(dtype, ld, offset):
    V = 5001
    for par in ({}, dict(top_k=70)):
        logits, z = make("peaked", 6, V, dtype, ld + offset, ld=ld, offset=offset)
        check(logits, z, par, actions(z, par, 3), V)
        past = logits[:, V:].clone()
        check(logits[:, :V], z, par, actions(z, par, 4), V)
        check(logits, z, par, actions(z, par, 5), V, in_place=True)
        assert torch.equal(past.view(torch.uint8), logits[:, V:].contiguous().view(torch.uint8))


def test_actions_outside_the_vocabulary():
    V = 900
    logits, z = make("normal", 4, V, F32, 4)
    for par in ({}, dict(top_p=0.9)):
        check(logits, z, par, np.array([-1, V, 5, 2**31 - 1]), V)


def test_own_settings_per_row():
    T, V = 300, 9000
    rng = np.random.default_rng(T)
    par = dict(temperature=rng.choice([0.0, 0.5, 1.0, 1.7], T).astype(np.float32),
               top_k=rng.choice([0, 1, 30, 3000, V], T).astype(np.int32),
               top_p=rng.choice([0.0, 0.3, 0.9, 1.0], T).astype(np.float32),
               min_p=rng.choice([0.0, 0.0, 0.1], T).astype(np.float32))
    logits, z = make("peaked", T, V, BF16, T)
    check(logits, z, par, actions(z, par, T), V)


def test_rows_without_a_distribution():
    V = 3000
    logits, z = make("normal", 6, V, F32, 1)
    logits[1, 2999] = float("nan")
    logits[2, 0] = float("inf")
    logits[3] = -1e8
    a = torch.full((6,), 4, dtype=torch.int32, device="cuda")
    tau = torch.tensor([1, 1, 1, 1, -1, 1.0], device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    logp, n, rows = grpo.grpo_sampled_logp(logits, a, temperature=tau, top_k=9, error_flags=flags)
    assert flags.item() == grpo.GRPO_FLAG_NONFINITE | grpo.GRPO_FLAG_SETTING
    assert n[1:5].tolist() == [0] * 4
    assert torch.isnan(logp[[1, 2, 4]]).all() and logp[3] == -float("inf")
    d = grpo.grpo_sampled_logp_bwd(logits, a, rows, torch.ones(6, device="cuda"))
    assert torch.isnan(d[[1, 2, 4]]).all()
    assert not d[3].any() and torch.isfinite(d[[0, 5]]).all()


def test_autograd_and_differences():
    """Through autograd, with a padded head: the gradient against central differences of the fp64 oracle, whose own error
    is h^2 / 6 of a third derivative of at most 1 / tau^3 and 1e-16 / h."""
    T, V, ld, tau = 5, 61, 64, 0.7
    logits, z = make("normal", T, V, F32, 11, ld=ld)
    logits = logits.nan_to_num(0.0).requires_grad_(True)
    par = dict(temperature=tau, top_k=40)
    act = actions(z, par, 1)
    a = torch.from_numpy(act.astype(np.int32)).cuda()
    logp = grpo.SampledLogp.apply(logits, a, dict(par, V=V))
    wts = torch.arange(1.0, T + 1, device="cuda")
    (logp * wts).sum().backward()
    assert logits.grad.shape == (T, ld) and not logits.grad[:, V:].any()
    h = 1e-5
    for t in range(T):
        st = settings_of(par, t)
        at, _, _ = so.kept(z[t], **st)
        lp = so.logp(z[t], int(act[t]), **st)[0]
        if np.isinf(lp):
            assert not logits.grad[t].any()
            continue
        for v in range(V):
            if v not in at:
                assert logits.grad[t, v] == 0
                continue
            def value(dv):
                q = z[t][at].copy()
                q[np.searchsorted(at, v)] += dv
                q = q / st["tau"]
                return q[np.searchsorted(at, act[t])] - q.max() - np.log(np.exp(q - q.max()).sum())
            num = (value(h) - value(-h)) / (2 * h) * (t + 1)
            tol = (t + 1) * (h * h / 6 / tau**3 + 4e-16 * 10 / h) + 1e-5 * abs(num)
            assert abs(float(logits.grad[t, v]) - num) <= tol
    with pytest.raises(RuntimeError):
        out = grpo.SampledLogp.apply(logits, a, dict(par, V=V)).sum()
        (g,) = torch.autograd.grad(out, logits, create_graph=True)
        g.sum().backward()


def test_graph_replays():
    T, V = 33, 30000
    logits, z = make("peaked", T, V, BF16, 6)
    par = dict(temperature=0.9, top_k=100)
    a = torch.from_numpy(actions(z, par, 2).astype(np.int32)).cuda()
    g_in = torch.randn(T, device="cuda")
    d, lp = torch.empty_like(logits), torch.empty(T, device="cuda")

    def call():
        logp, _, rows = grpo.grpo_sampled_logp(logits, a, **par)
        lp.copy_(logp)
        grpo.grpo_sampled_logp_bwd(logits, a, rows, g_in, dlogits=d)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(4):
        logits.mul_(0.95)
        call()
        want = d.clone(), lp.clone()
        torch.cuda.synchronize()
        d.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, want[0]) and torch.equal(lp, want[1]), rep


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_autograd_of_padded_columns_in_wider_rows(dtype):
    T, cols, V, ld = 5, 700, 650, 800
    buf = torch.randn((T, ld), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    act = torch.arange(T, dtype=torch.int32, device="cuda") * 100
    g = torch.rand(T, device="cuda") + 0.5

    for par in (dict(temperature=0.7, top_k=60), dict(temperature=0.7)):

        def grad(x):
            x = x.detach().requires_grad_()
            logp = grpo.SampledLogp.apply(x, act, dict(par, V=V))
            logp.backward(g)
            return x.grad, torch.isfinite(logp.detach())

        (strided, kept), (packed, _) = grad(buf[:, :cols]), grad(buf[:, :cols].contiguous())
        assert torch.equal(strided, packed) and (strided[:, V:] == 0).all()
        # rows whose action is not kept have no gradient; with nothing cut every row has one
        assert torch.equal((strided[:, :V] != 0).any(1), kept) and (kept.all() or "top_k" in par)
