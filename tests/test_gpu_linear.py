"""grpo_linear and its gradient against the formulas in 64 bits.

With e = 2^-24 (half a step of fp32), h half a step of the result's type and b = 2^-8 that of bf16:
- z: products of bf16 numbers are exact in fp32; their K sums, in any order, are off by at most K e sum |x w| (and the bias
  by e of the result).  Roundings that are independent of one another keep the norm of all errors below 4 e sqrt(K) of
  the norm of the sums' sizes;
- act(z): |act'| <= 1.13 times z's error, and 8 e (|z| + 1) of its own; y adds the residual (e of the result) and h;
- act'(z): 16 e (1 + |z| + |z|^3 / 8) of its own (the last from 1 - tanh^2 times the argument's slope), 1 times z's error;
- dz in fp32 by that; in the products b of each term more, and the sum as above: dx by (b + N e) sum |dz w| and h;
- dbias: partial sums of at most 1,024 rows in fp32, joined in fp64: 1024 e sum |dz|, the terms' own errors, and h.
"""
import math

import pytest
import torch

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu

E, B = 2.0**-24, 2.0**-8
F32, BF16 = torch.float32, torch.bfloat16
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def act64(act, z):
    f = torch.nn.functional
    return {"none": lambda t: t.clone(), "relu": f.relu, "gelu": f.gelu, "silu": f.silu,
            "gelu_tanh": lambda t: f.gelu(t, approximate="tanh")}[act](z)


def half(dtype):
    return torch.finfo(dtype).eps / 2


def within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bad.any():
        i = int((off - bound).flatten().argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()}, worst at {i}: {got.flatten()[i]} for "
                             f"{want.flatten()[i]}, off {off.flatten()[i]} > {bound.expand_as(off).flatten()[i]}")


def norm_within(got, want, size, rel, what):
    """The norm of the errors, where there are enough of them."""
    if want.numel() >= 1000:
        off = (got.double() - want).norm()
        assert off <= rel * size.norm(), (what, float(off), float(rel * size.norm()))


def tensors(M, K, N, w="kn", bias=None, out=BF16, ldx=0, ldw=0, ldy=0, offset=0, seed=0):
    g = torch.Generator("cuda").manual_seed(seed * 1000003 + M * 7919 + K * 31 + N)

    def mat(r, c, ld, dtype, scale=1.0):
        flat = torch.full((offset + r * max(ld, c) + 8,), float("nan"), device="cuda").to(dtype)
        t = flat[offset:offset + r * max(ld, c)].view(r, max(ld, c))[:, :c]
        t.copy_((torch.randn((r, c), generator=g, device="cuda") * scale).to(dtype))
        return t

    x = mat(M, K, ldx, BF16)
    wt = mat(K, N, ldw, BF16, K**-0.5) if w == "kn" else mat(N, K, ldw, BF16, K**-0.5).t()
    b = None if bias is None else (torch.randn(N, generator=g, device="cuda") * 0.5).to(bias)
    return x, wt, b, mat(M, N, ldy, out), mat(M, N, ldy, out, 0.3)


def forward_check(x, w, b, res, act, out, y, z):
    K = x.shape[1]
    xd, wd = x.double(), w.double()
    zw = xd @ wd
    size = xd.abs() @ wd.abs()
    zw = zw if b is None else zw + b.double()
    ez = K * E * size + E * zw.abs()
    if z is not None:
        within(z, zw, 1.01 * ez + 1e-30, "z")
        norm_within(z, zw, size.square().div(K).sqrt() + zw.abs(), 4 * E * math.sqrt(K), "z")
    a = act64(act, zw)
    want = a if res is None else a + res.double()
    ey = 1.13 * ez + (8 * E * (zw.abs() + 1) if act != "none" else 0) + E * want.abs()
    within(y, want, 1.01 * (ey + half(out) * want.abs()) + 1e-30, "y")
    norm_within(y, want, want.abs() + zw.abs() + size / math.sqrt(K), half(out) + (8 + 4 * math.sqrt(K)) * E, "y")
    return zw, ez, want


def backward_check(x, w, zw, ez, act, dy, dx, dw, db, dw_before=None):
    xd, wd = x.double(), w.double()
    t = zw.clone().requires_grad_()
    (slope,) = torch.autograd.grad(act64(act, t).sum(), t) if act != "none" else (torch.ones_like(zw),)
    dyd = dy.double()
    dz = dyd * slope
    own = 16 * E * (1 + zw.abs() + zw.abs()**3 / 8) if act != "none" else torch.zeros_like(zw)
    err = dyd.abs() * (own + (ez if act != "none" else 0)) + 2 * E * dz.abs()
    if act == "relu":  # a z within its error of 0 may be on either side
        err = torch.where(zw.abs() <= ez, dyd.abs(), err)
    exact = act == "none" and dy.dtype == BF16
    rounding = 0.0 if exact else B
    term = err + rounding * dz.abs()
    M, N = dz.shape
    for got, want, bound, size, n, what in (
            (dx, dz @ wd.t(), (term + N * E * dz.abs()) @ wd.t().abs(), (dz.square() @ wd.t().square()).sqrt(), N, "dx"),
            (dw, xd.t() @ dz, xd.t().abs() @ (term + M * E * dz.abs()), (xd.t().square() @ dz.square()).sqrt(), M, "dw")):
        if got is None:
            continue
        if what == "dw" and dw_before is not None:
            want = want + dw_before.double()
            bound = bound + 2 * E * want.abs()
        within(got, want, 1.01 * (bound + half(got.dtype) * want.abs()) + 1e-30, what)
        if act != "relu":
            norm_within(got, want, size + want.abs(), rounding + half(got.dtype) + (4 * math.sqrt(n) + 16) * E, what)
    if db is not None:
        want = dz.sum(0)
        bound = err.sum(0) + min(M, 1024) * E * dz.abs().sum(0)
        within(db, want, 1.01 * (bound + half(db.dtype) * want.abs()) + 1e-30, "dbias")


def check(M, K, N, act="none", w="kn", bias=None, residual=False, out=BF16, grad=True, dw_dtype=BF16, seed=0, **lie):
    x, wt, b, res, dy = tensors(M, K, N, w, bias, out, seed=seed, **lie)
    res = res if residual else None
    keep = grad and act != "none"
    y, z = grpo.grpo_linear(x, wt, b, res, act=act, out_dtype=out, keep_z=keep)
    assert (z is not None) == keep and y.dtype == out
    zw, ez, _ = forward_check(x, wt, b, res, act, out, y, z)
    if not grad:
        return
    db = None if b is None else torch.full_like(b, float("nan"))
    dw, before = True, None
    if dw_dtype == F32:
        dw = torch.randn(wt.t().shape if w == "nk" else wt.shape, device="cuda")
        dw = dw.t() if w == "nk" else dw
        before = dw.clone()
    dx, dw, _ = grpo.grpo_linear_bwd(dy, x, wt, z, act=act, dw=dw, dbias=db, accumulate_dw=dw_dtype == F32)
    assert dw.stride() == (wt.stride() if wt.t().is_contiguous() or wt.is_contiguous() else dw.stride())
    backward_check(x, wt, zw, ez, act, dy, dx, dw, db, before)


SIZES = [(1, 1, 1), (1, 8, 8), (3, 7, 5), (1, 64, 1000), (4, 64, 1000), (2, 3584, 640), (8, 100, 2049), (16, 264, 8),
         (17, 100, 33), (31, 128, 4096), (33, 1000, 520), (48, 72, 1003), (64, 256, 256), (65, 257, 259), (100, 2048, 16),
         (130, 512, 300), (200, 96, 31), (256, 64, 256), (257, 1032, 520), (300, 1000, 1003), (513, 136, 776),
         (700, 65, 1), (1025, 264, 513), (2000, 8, 24)]


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_sizes(M, K, N, w):
    check(M, K, N, w=w, bias=F32, out=F32)
    check(M, K, N, w=w, act="silu", bias=BF16, residual=True, out=BF16, seed=1)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("bias,residual,out,dw_dtype", [(None, False, BF16, BF16), (BF16, True, F32, BF16),
                                                       (F32, True, BF16, F32), (F32, False, F32, F32)], ids=str)
@pytest.mark.parametrize("M,K,N", [(7, 200, 392), (270, 328, 600)])
def test_forms(M, K, N, act, w, bias, residual, out, dw_dtype):
    check(M, K, N, act, w, bias, residual, out, dw_dtype=dw_dtype)


@pytest.mark.parametrize("lie", [dict(ldx=1040), dict(ldx=1003), dict(ldw=1048), dict(ldw=1047), dict(ldy=1056),
                                 dict(ldy=1049), dict(offset=1), dict(offset=4), dict(ldx=1033, ldw=1041, ldy=1043, offset=3)],
                         ids=str)
@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M", [5, 40, 290])
def test_strides_and_alignment(M, w, lie):
    check(M, 1000, 1024, "gelu", w, BF16, True, BF16, **lie)
    check(M, 1000, 1024, "none", w, F32, True, F32, **lie)


@pytest.mark.parametrize("M,K,N,w", [(4096, 1024, 2048, "kn"), (4001, 3584, 1280, "nk"), (1, 3584, 32003, "kn"),
                                     (2048, 512, 16000, "kn"), (20, 8192, 16384, "nk"), (8192, 64, 512, "nk")])
def test_larger(M, K, N, w):
    check(M, K, N, "gelu_tanh", w, BF16, True, BF16)
    check(M, K, N, "none", w, None, False, BF16, seed=2)


def test_one_wanted_gradient_at_a_time():
    x, w, b, _, dy = tensors(70, 136, 264, "nk", F32)
    y, z = grpo.grpo_linear(x, w, b, act="silu", keep_z=True)
    db = torch.empty_like(b)
    dx, dw, _ = grpo.grpo_linear_bwd(dy, x, w, z, act="silu", dbias=db)
    one = torch.full_like(dx, 7.0)
    got = grpo.grpo_linear_bwd(dy, x, w, z, act="silu", dx=one, dw=False)
    assert got[0] is one and got[1] is None and torch.equal(one, dx)
    got = grpo.grpo_linear_bwd(dy, x, w, z, act="silu", dx=False)
    assert got[0] is None and torch.equal(got[1], dw)
    db2 = torch.empty_like(b)
    assert grpo.grpo_linear_bwd(dy, x, w, z, act="silu", dx=False, dw=False, dbias=db2)[:2] == (None, None)
    assert torch.equal(db, db2)
    assert grpo.grpo_linear_bwd(dy, x, w, z, act="silu", dx=False, dw=False) == (None, None, None)


def test_no_rows():
    x, w = torch.empty((0, 24), dtype=BF16, device="cuda"), torch.randn(24, 40, device="cuda").to(BF16)
    y, z = grpo.grpo_linear(x, w, act="relu", keep_z=True)
    assert y.shape == z.shape == (0, 40)
    for b in (torch.full((40,), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda", dtype=BF16)):
        dx, dw, db = grpo.grpo_linear_bwd(y, x, w, z, act="relu", dbias=b)
        assert dx.shape == (0, 24) and not dw.any() and not db.any()
    dw = torch.ones(24, 40, device="cuda")
    grpo.grpo_linear_bwd(y, x, w, z, act="relu", dw=dw, accumulate_dw=True)
    assert (dw == 1).all()
    grpo.grpo_linear_bwd(y, x, w, z, act="relu", dw=dw)
    assert not dw.any()


@pytest.mark.parametrize("M", [3, 300])
@pytest.mark.parametrize("out", [F32, BF16], ids=str)
def test_residual_in_place_and_rows_beside_others(M, out):
    x, w, b, res, _ = tensors(M, 264, 520, "kn", F32, out, ldy=528)
    base = res._base if res._base is not None else res
    want, _ = grpo.grpo_linear(x, w, b, res, act="gelu", out_dtype=out)
    wide = torch.full((M, 600), 5.0, device="cuda").to(out)
    wide[:, 7:527] = res
    got, _ = grpo.grpo_linear(x, w, b, wide[:, 7:527], act="gelu", out=wide[:, 7:527])
    assert torch.equal(got, want) and (wide[:, :7] == 5).all() and (wide[:, 527:] == 5).all()
    assert base is not None


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("M", [2, 70])
def test_values_that_are_not_finite_stay_in_their_rows(M, value):
    """Also where operands are copied with padding, or rows past the end of an operand are read as zeros."""
    for K, N in ((100, 300), (128, 257)):
        x, w, b, _, dy = tensors(M, K, N, "kn", F32)
        want, _ = grpo.grpo_linear(x, w, b)
        x[1, K - 1] = value
        y, _ = grpo.grpo_linear(x, w, b)
        assert torch.equal(y[0], want[0]) and torch.equal(y[2:], want[2:]) and not y[1].isfinite().any()
        dy[0, N - 1] = value
        dx, dw, db = grpo.grpo_linear_bwd(dy, x, w, dbias=torch.empty_like(b))
        assert not dx[0].isfinite().any() and dx[1:].isfinite().all() and db[:-1].isfinite().all() and not db[-1].isfinite()
        assert not dw[:, -1].isfinite().any() and not dw[K - 1].isfinite().any() and dw[:K - 1, :-1].isfinite().all()


@pytest.mark.parametrize("M,K,N,w", [(5, 64, 1000, "kn"), (300, 264, 515, "nk"), (40, 2048, 1024, "kn")])
def test_autograd_and_graph(M, K, N, w):
    x, wt, b, res, dy = tensors(M, K, N, w, F32)
    leaves = [t.contiguous() if t is not wt else (t if w == "kn" else t.t().contiguous()) for t in (x, wt, b, res)]
    leaves = [t.detach().clone().requires_grad_() for t in leaves]
    dy = dy.contiguous()

    def step():
        xx, ww, bb, rr = leaves
        y = grpo.Linear.apply(xx, ww if w == "kn" else ww.t(), bb, rr, dict(act="gelu"))
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    got = step()
    ww = leaves[1].detach() if w == "kn" else leaves[1].detach().t()
    y, z = grpo.grpo_linear(leaves[0].detach(), ww, leaves[2].detach(), leaves[3].detach(), act="gelu", keep_z=True)
    dx, dw, db = grpo.grpo_linear_bwd(dy, leaves[0].detach(), ww, z, act="gelu", dbias=torch.empty_like(leaves[2]))
    for a, c in zip(got, (y, dx, dw if w == "kn" else dw.t(), db, dy)):
        assert torch.equal(a, c)
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
            leaves[0].mul_(0.9)
            dy.mul_(-1.1)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in got[:4]:
            t.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), rep


def test_gradient_against_differences():
    """Central differences in 64 bits of the operator's formula with y's own rounding left out: fp32 outputs, a direction in
    which x, w and b change by bf16 numbers' sizes."""
    M, K, N = 6, 40, 56
    x, w, b, _, dy = tensors(M, K, N, "kn", F32, F32)
    for act in ACTS[2:]:
        y, z = grpo.grpo_linear(x, w, b, act=act, out_dtype=F32, keep_z=True)
        dw = torch.empty((K, N), device="cuda")
        dx, dw, db = grpo.grpo_linear_bwd(dy, x, w, z, act=act, dw=dw, dbias=torch.empty_like(b))
        g = torch.Generator("cuda").manual_seed(1)
        vx, vw, vb = (torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for t in (x, w, b))
        f = lambda h: (dy.double() * act64(act, (x.double() + h * vx) @ (w.double() + h * vw) + b.double() + h * vb)).sum()  # noqa: E731
        want = (f(1e-5) - f(-1e-5)) / 2e-5
        parts = [(dx.double() * vx).abs().sum(), (dw.double() * vw).abs().sum(), (db.double() * vb).abs().sum()]
        got = (dx.double() * vx).sum() + (dw.double() * vw).sum() + (db.double() * vb).sum()
        # dx: one rounding to bf16 of the result and one of each term; dw: of each term
        assert abs(got - want) <= 2.5 * B * sum(parts), (act, got, want)


def test_two_streams():
    a, c = tensors(100, 257, 1003, "kn", F32, seed=1), tensors(100, 257, 1003, "kn", F32, seed=2)
    want = [grpo.grpo_linear(t[0], t[1], t[2], act="relu")[0] for t in (a, c)]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [grpo.grpo_linear(t[0], t[1], t[2], act="relu", stream=s)[0] for t, s in zip((a, c), sides)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_rows_beyond_32_bit_offsets():
    M, K, N = 70000, 16, 32008  # y: 4.5 GB
    x, w, b, _, _ = tensors(M, K, N, "kn", F32)
    y, _ = grpo.grpo_linear(x, w, b)
    for r in (0, 35000, M - 300):
        want, _ = grpo.grpo_linear(x[r:r + 300].clone(), w, b)
        assert torch.equal(y[r:r + 300], want)
    dx, dw, _ = grpo.grpo_linear_bwd(y, x, w, dw=False)
    want = (y[-5:].double() @ w.double().t())
    bound = (N * E) * (y[-5:].double().abs() @ w.double().t().abs()) + B * want.abs()
    within(dx[-5:], want, 1.01 * bound, "dx")
