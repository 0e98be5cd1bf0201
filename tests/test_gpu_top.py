"""grpo_token_logp_top and its gradient against the fp64 oracle.

Ids are equal.  Errors, with e = 2^-24 (half a step of fp32), t = log2(e) (z - max) / tau a word's exponent, and k the
words of one thread (a row of V goes to 256 threads or more) with k / 32 + 1 steps of its running maximum:
- a term's exponent is off by 3 e |t| (the difference, the factor, the product) and the term by 2 e more; a thread's sum by
  k e, its raised maxima by 4 e each: log S is off by at most s = (3 ln2 E|t| + k + 4 (k / 32 + 1) + 8) e, E|t| the mean
  under the distribution;
- the moment T = sum 2^t t / S is a sum of one sign: off by its own size times (3 ln2 E|t|^2 / E|t| + k + 4 (k / 32 + 1)
  + 12) e, and by s, in S; the entropy log S - ln2 T by that and s;
- a log-prob by s and e of its size (one rounding; the rest is fp64);
- d logits of a word without a coefficient, p (A log2 p + B): log2 p is off by (2 |t| + |log2 p| + |log2 S|) e and by s / ln2,
  p by ln2 times that and 4 e more, A, B and the sum by 3 e of their sizes and by the entropy's error times the gradient g;
  of the action and the alternatives, fp64 from the same S and H: s and the entropy's error in p, lp and H.  Then one
  rounding to the type (two for the latter).  Below 2^-126 the exponential is 0.
"""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from oracle import top as oracle_top

pytestmark = pytest.mark.gpu

E = 2.0**-24
F32, BF16 = torch.float32, torch.bfloat16


def make(kind, T, V, dtype, seed, ld=None):
    """Logits [T, ld] on the GPU and their first V columns in fp64."""
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 2, (T, V))
    if kind == "peaked":
        z[np.arange(T), rng.integers(0, V, T)] += 30
    elif kind == "ties":
        z = np.round(z)
    elif kind == "equal":
        z[:] = rng.normal(size=(T, 1))
    elif kind == "rising":
        z = np.sort(z, axis=1)
    elif kind == "falling":
        z = -np.sort(-z, axis=1)
    elif kind == "clustered":  # the largest words beside one another
        at = rng.integers(0, max(1, V - 2000), T)
        for t in range(T):
            z[t, at[t]:at[t] + 2000] += 12
    elif kind == "masked":
        z[rng.random((T, V)) < 0.999] = -np.inf
        z[0] = -np.inf
        z[T - 1, V // 2:] = -3e38
    elif kind == "border":  # words next to the mask's border
        z = -1e8 + rng.integers(-4, 40, (T, V)) * 8.0
    elif kind == "large":
        z *= 1e4
    elif kind == "zeros":
        z = np.where(rng.random((T, V)) < 0.5, 0.0, -0.0)
    x = torch.full((T, ld or V), float("nan"), dtype=dtype)
    x[:, :V] = torch.from_numpy(z).to(dtype)
    return x.cuda(), x[:, :V].double().numpy()


def taus(tau, T):
    if tau == "rows":
        v = np.float32(np.random.default_rng(T).choice([0.3, 0.7, 1.0, 2.5], T))
        return torch.from_numpy(v).cuda(), v.astype(np.float64)
    return tau, np.full(T, float(np.float32(tau)))


def bounds(z, lp, tau):
    """(error of log S, of the entropy, |t|, log2 S)."""
    live = lp > -np.inf
    t = np.zeros(z.size)
    t[live] = np.log2(np.e) * (z[live].max() - z[live]) / tau
    p = np.exp(lp)
    k = z.size / 256 + 8
    steps = k + 4 * (k / 32 + 1)
    m1, m2 = (p * t).sum(), (p * t * t).sum()
    s = (3 * np.log(2) * m1 + steps + 8) * E
    h = s + np.log(2) * ((3 * np.log(2) * m2 + (steps + 12) * m1) * E + m1 * s)
    return s, h, t, -lp[live].max() / np.log(2)


def check(logits, z, act, n, tau=1.0, grad=True, in_place=False, flags_want=0, ups=(True, True, True)):
    T, V = z.shape
    temp, tau = taus(tau, T)
    a = torch.from_numpy(np.asarray(act, np.int32)).cuda()
    flags = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    logp, ent, ids, tlp, rows = grpo.grpo_token_logp_top(logits, a, n, temperature=temp, V=V, error_flags=flags)
    gen = torch.Generator().manual_seed(T + V + n)
    up = [torch.randn(s, generator=gen) for s in ((T,), (T,), (T, n))]
    if grad:
        dev = [u.cuda() if on else None for u, on in zip(up, ups)]
        d = grpo.grpo_token_logp_top_bwd(logits, a, ids, rows, *dev, V=V, dlogits=logits if in_place else True)
        d = d[:, :V].double().cpu().numpy()
        half = torch.finfo(logits.dtype).eps / 2
    up = [u.double().numpy() * on for u, on in zip(up, ups)]
    logp, ent, ids, tlp = (x.double().cpu().numpy() for x in (logp, ent, ids, tlp))
    for t in range(T):
        lp, h, want_ids, want_top, every = oracle_top.row(z[t], int(act[t]), n, tau[t])
        assert ids[t].tolist() == want_ids.tolist(), (t, ids[t], want_ids)
        if not (every > -np.inf).any():
            assert logp[t] == lp and ent[t] == 0 and (tlp[t] == -np.inf).all()
            assert not grad or not d[t].any()
            continue
        s, he, x, ls = bounds(z[t], every, tau[t])
        assert 0 <= act[t] < V or logp[t] == 0
        own = [(logp[t], lp)] if 0 <= act[t] < V else []
        for got, want in own + list(zip(tlp[t], want_top)):
            if np.isinf(want):
                assert got == want, (t, got, want)
            else:
                assert abs(got - want) <= s + 1.01 * E * abs(want), (t, got, want, s)
        assert abs(ent[t] - h) <= he + 1.01 * E * h, (t, ent[t], h, he)
        if not grad:
            continue
        dl, de, dt = up[0][t], up[1][t], up[2][t]
        want = oracle_top.gradient(every, h, int(act[t]), want_ids, dl, de, dt, tau[t])
        on = 0 <= act[t] < V and every[act[t]] > -np.inf
        C = (dl if on else 0.0) + dt[want_ids >= 0].sum()
        Ca = (abs(dl) if on else 0.0) + np.abs(dt[want_ids >= 0]).sum()
        p, l = np.exp(every), np.where(np.isinf(every), 0.0, every)
        l2 = (2 * x + np.abs(l) / np.log(2) + ls) * E * np.log(2) + s  # of log p
        size = np.abs(C + de * h) + np.abs(de * l)
        bound = p / tau[t] * (size * (l2 + 8 * E) + np.abs(de) * (l2 + he) + (Ca + np.abs(de) * h) * 4 * E)
        bound += np.abs(want) * half + 2.0**-126 * (Ca + np.abs(de) * (1 + h)) * 256 / tau[t]
        special = [i for i in list(want_ids) + [act[t] if on else -1] if i >= 0]
        bound[special] += np.abs(want[special]) * 2 * E + 1e-13 * (Ca + abs(de)) / tau[t]
        bound *= 1.01
        off = np.abs(d[t] - want)
        assert (off <= bound).all(), (t, int(np.argmax(off - bound)), off.max(), bound[np.argmax(off - bound)])
    assert flags.item() == flags_want


def actions(z, seed):
    rng = np.random.default_rng(seed)
    return np.where(rng.random(z.shape[0]) < 0.5, np.argmax(z, axis=1), rng.integers(0, z.shape[1], z.shape[0]))


KINDS = ["normal", "peaked", "ties", "equal", "rising", "falling", "clustered", "large", "zeros"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,V,dtype", [(5, 300, BF16), (4, 1024, F32), (3, 2049, BF16), (130, 4100, F32), (3, 16384, BF16),
                                       (3, 32003, F32), (130, 32003, BF16), (2, 151936, BF16), (129, 70001, F32)], ids=str)
def test_values(T, V, dtype, kind):
    logits, z = make(kind, T, V, dtype, 5 * V + T)
    act = actions(z, V)
    for n, tau in ((20, 1.0), (64, "rows")):
        check(logits, z, act, n, tau)


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 65, 255, 2047, 2048, 8193, 16391, 65537])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_sizes(V, dtype):
    for n in (0, 1, 5, 33, 64):
        for T in (1, 3):
            logits, z = make("normal", T, V, dtype, V + n)
            check(logits, z, actions(z, n), n, 0.8)


@pytest.mark.parametrize("T,V", [(6, 1000), (6, 40000), (200, 9000), (66, 151936)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_masked_rows(T, V, dtype):
    logits, z = make("masked", T, V, dtype, V)
    act = np.array([int(np.argmax(r)) for r in z])
    act[1] = 3  # masked, very likely
    check(logits, z, act, 20, "rows", flags_want=grpo.GRPO_FLAG_NONFINITE)
    logits, z = make("border", T, V, F32, V)
    check(logits, z, actions(z, V), 7, 3.0)


@pytest.mark.parametrize("tau", [1e-6, 0.01, 50.0, 1e6])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_far_temperatures(tau, dtype):
    for kind in ("normal", "large"):
        logits, z = make(kind, 3, 20001, dtype, 4)
        check(logits, z, actions(z, 2), 9, tau)


@pytest.mark.parametrize("T,V,ld", [(3, 151669, 151936), (150, 5001, 5120), (4, 999, 1003)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_padded_columns_and_in_place(T, V, ld, dtype):
    logits, z = make("normal", T, V, dtype, V, ld)
    act = actions(z, 1)
    act[0] = -1
    act[1] = V  # a padding column is no action
    check(logits, z, act, 8, 0.7, flags_want=grpo.GRPO_FLAG_ACTION)
    pad = logits[:, V:].clone()
    check(logits, z, act, 8, 0.7, in_place=True, flags_want=grpo.GRPO_FLAG_ACTION)
    assert torch.equal(logits[:, V:].isnan(), pad.isnan())


@pytest.mark.parametrize("ups", [(True, False, False), (False, True, False), (False, False, True), (False, False, False)])
def test_gradients_of_one_result(ups):
    logits, z = make("normal", 4, 10007, F32, 9)
    check(logits, z, actions(z, 3), 12, 1.3, ups=ups)


@pytest.mark.parametrize("T,V", [(8, 500), (8, 60000), (300, 20000)])
def test_bad_rows(T, V):
    logits, z = make("normal", T, V, F32, 1)
    logits[1, V // 3] = float("nan")
    logits[2, V - 1] = float("inf")
    logits[3] = float("-inf")
    temp = torch.ones(T, device="cuda")
    temp[4], temp[5], temp[6] = 0.0, float("nan"), 2e6
    act = torch.zeros(T, dtype=torch.int32, device="cuda")
    act[2] = V
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = 6
    logp, ent, ids, tlp, rows = grpo.grpo_token_logp_top(logits, act, n, temperature=temp, error_flags=flags)
    assert flags.item() == grpo.GRPO_FLAG_ACTION | grpo.GRPO_FLAG_NONFINITE | grpo.GRPO_FLAG_SETTING
    for t in (1, 2, 4, 5, 6):
        assert ent[t].isnan() and tlp[t].isnan().all() and (ids[t] == -1).all()
        assert logp[t].isnan() if t != 2 else logp[t] == 0
    assert logp[3] == -float("inf") and ent[3] == 0 and (tlp[3] == -float("inf")).all() and (ids[3] == -1).all()
    one = torch.ones(T, device="cuda")
    d = grpo.grpo_token_logp_top_bwd(logits, act, ids, rows, one, one, one[:, None].expand(T, n).contiguous())
    for t in range(T):
        if t in (1, 2, 4, 5, 6):
            assert d[t].isnan().all()
        elif t == 3:
            assert not d[t].any()
        else:
            assert d[t].isfinite().all()


def test_no_rows():
    x = torch.empty((0, 77), device="cuda")
    a = torch.empty(0, dtype=torch.int32, device="cuda")
    logp, ent, ids, tlp, rows = grpo.grpo_token_logp_top(x, a, 4)
    assert ids.shape == (0, 4) and grpo.grpo_token_logp_top_bwd(x, a, ids, rows, logp, ent, tlp).shape == (0, 77)


def test_more_rows_than_a_launch_takes():
    """2^20 + 77 rows repeat the first 1,000, and so do their outputs."""
    k, T, V, n = 1000, (1 << 20) + 77, 9, 3
    gen = torch.Generator("cuda").manual_seed(4)
    few = torch.randn(k, V, device="cuda", generator=gen)
    act = torch.randint(0, V, (k,), device="cuda", generator=gen).int()
    at = torch.arange(T, device="cuda") % k
    want = grpo.grpo_token_logp_top(few, act, n)
    many, act2 = few[at].contiguous(), act[at].contiguous()
    got = grpo.grpo_token_logp_top(many, act2, n)
    assert all(torch.equal(a, b[at]) for a, b in zip(got, want))
    d = grpo.grpo_token_logp_top_bwd(few, act, want[2], want[4], want[0], want[1], want[3])
    got = grpo.grpo_token_logp_top_bwd(many, act2, got[2], got[4], got[0], got[1], got[3])
    assert torch.equal(got, d[at])


@pytest.mark.parametrize("V", [12, 700, 20000])
def test_ids_of_the_callers_own(V):
    """The same id twice adds up; ids outside [0, V) count for nothing, their gradients unread."""
    T = 3
    logits, z = make("normal", T, V, F32, 2)
    act = torch.full((T,), 5, dtype=torch.int32, device="cuda")
    rows = grpo.grpo_token_logp_top(logits, act, 0)[4]
    ids = torch.tensor([[5, 5, 2, 2, V, -7, V - 1, 2]] * T, dtype=torch.int32, device="cuda")
    up = torch.tensor([[0.5, 1.5, 2, 3, float("nan"), float("inf"), -1, 4]] * T, device="cuda")
    d = grpo.grpo_token_logp_top_bwd(logits, act, ids, rows, torch.ones(T, device="cuda"), None, up).double().cpu().numpy()
    for t in range(T):
        _, h, _, _, every = oracle_top.row(z[t], 5, 0)
        want = oracle_top.gradient(every, h, 5, [5, 2, V - 1], 1.0, 0.0, [2.0, 9.0, -1.0])
        s = bounds(z[t], every, 1.0)[0]
        assert (np.abs(d[t] - want) <= np.exp(every) * 13 * (s + 60 * E) + 2 * E * np.abs(want)).all()


@pytest.mark.parametrize("T,V,dtype", [(2, 40000, BF16), (150, 3000, F32)], ids=str)
def test_autograd_and_graph(T, V, dtype):
    gen = torch.Generator("cuda").manual_seed(3)
    ld, n = V + 8, 5
    x = torch.randn(T, ld, device="cuda", generator=gen).to(dtype).requires_grad_()
    act = x.detach()[:, :V].argmax(1).to(torch.int32)
    up = [torch.randn(s, device="cuda", generator=gen) for s in ((T,), (T,), (T, n))]

    def step():
        logp, ent, ids, top = grpo.TokenLogpTop.apply(x, act, n, dict(temperature=0.9, V=V))
        (d,) = torch.autograd.grad((logp, ent, top), x, up)
        return logp.detach(), ent.detach(), ids, top.detach(), d

    rows = grpo.grpo_token_logp_top(x.detach(), act, n, temperature=0.9, V=V)
    d = grpo.grpo_token_logp_top_bwd(x.detach(), act, rows[2], rows[4], *up, V=V)
    got = step()
    assert all(torch.equal(a, b) for a, b in zip(got[:4], rows[:4]))
    assert torch.equal(got[4][:, :V], d[:, :V]) and not got[4][:, V:].any()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    del got
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for rep in range(4):
        with torch.no_grad():
            x.mul_(0.9)
            up[0].mul_(-1.1)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in got:
            t.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rep


def test_one_result_of_the_autograd_call():
    x = torch.randn(6, 500, device="cuda", requires_grad=True)
    act = torch.arange(6, dtype=torch.int32, device="cuda")
    _, ent, ids, _ = grpo.TokenLogpTop.apply(x, act, 3)
    assert not ids.requires_grad
    ent.sum().backward()
    y = x.detach().double().requires_grad_()
    torch.special.entr(torch.softmax(y, 1)).sum().backward()
    assert torch.allclose(x.grad.double(), y.grad, atol=2e-6, rtol=0)


def test_two_streams_with_workspaces_of_their_own():
    T, V, n = 4, 151936, 20
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    xs = [make("normal", T, V, BF16, i)[0] for i in range(2)]
    act = torch.zeros(T, dtype=torch.int32, device="cuda")
    want = [grpo.grpo_token_logp_top(x, act, n) for x in xs]
    torch.cuda.synchronize()
    for rep in range(5):
        got = [grpo.grpo_token_logp_top(x, act, n, stream=s) for x, s in zip(xs, sides)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_a_row_beyond_32_bit_offsets():
    T, V = 40000, 60000  # 4.8 GB of bf16
    x = torch.zeros(T, V, dtype=BF16, device="cuda")
    x[T - 1] = torch.randn(V, device="cuda", generator=torch.Generator("cuda").manual_seed(8)).to(BF16)
    act = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    got = grpo.grpo_token_logp_top(x, act, 4)
    want = grpo.grpo_token_logp_top(x[T - 1:].clone(), act[:1], 4)
    assert torch.equal(got[2][-1], want[2][0]) and torch.equal(got[2][0], torch.arange(4, device="cuda").int())
    assert abs(got[0][-1] - want[0][0]) < 1e-4 and abs(got[1][0] - np.log(V)) < 1e-4
    d = grpo.grpo_token_logp_top_bwd(x, act, got[2], got[4], torch.ones(T, device="cuda"), None, None)
    assert torch.equal(d[-1:], grpo.grpo_token_logp_top_bwd(x[T - 1:].clone(), act[:1], got[2][-1:].contiguous(), got[4][-1:].contiguous(),
                                                           torch.ones(1, device="cuda"), None, None))


@pytest.mark.parametrize("kind", ["equal", "clustered", "zeros"])
def test_the_same_bits_every_time(kind):
    logits, _ = make(kind, 40, 32003, F32, 6)
    act = torch.zeros(40, dtype=torch.int32, device="cuda")
    want = grpo.grpo_token_logp_top(logits, act, 64)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(grpo.grpo_token_logp_top(logits, act, 64), want))
