"""The gradients' norm and clipping against fp64.

norm: fp64 sums, one rounding to fp32: 2^-24.  Clipped values: the factor is rounded to fp32 (2^-24), the product is (2^-24),
and for a bf16 out once more (2^-8); below fp32's normal range by half a step of its smallest.
"""
import pytest
import torch

import paper_2606_05597_amd as grpo

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def bucket(sizes, dtypes, seed, pad=0, scale=0.01):
    """Tensors one behind the other, `pad` elements apart, one buffer for each type; and the buffers."""
    flats = {t: torch.full((sum(n + pad for n, d in zip(sizes, dtypes) if d == t) + pad,), float("nan"), dtype=t,
                           device="cuda") for t in set(dtypes)}
    at = {t: pad for t in flats}
    g = torch.Generator("cuda").manual_seed(seed)
    views = []
    for n, t in zip(sizes, dtypes):
        v = flats[t][at[t]:at[t] + n]
        v.copy_(torch.randn(n, device="cuda", generator=g) * scale)
        views.append(v)
        at[t] += n + pad
    return views, flats


def check(grads, max_norm, outs=None, flats=()):
    before = [g.clone() for g in grads]
    norm64 = sum(g.double().square().sum() for g in grads).sqrt() if grads else torch.zeros(())
    lst = grpo.GradList(grads, out=outs)
    norm = grpo.grpo_clip_grad_norm_(lst, max_norm)
    assert norm.shape == () and norm.dtype == F32
    assert abs(norm.item() - norm64.item()) <= 2.0**-24 * norm64.item() * 1.01
    f = min(1.0, max_norm / (norm64.item() + 1e-6))
    for i, b in enumerate(before):
        o = grads[i] if outs is None else outs[i]
        want = b.double() * f
        half = 2.0**-8 if o.dtype == BF16 else 0.0
        if f == 1.0 and o.dtype == b.dtype:
            assert torch.equal(o, b)
        tol = want.abs() * (2 * 2.0**-24 + half) * 1.01 + 2.0**-133
        assert ((o.double() - want).abs() <= tol).all(), i
        if outs is not None:
            assert torch.equal(grads[i], b)


SIZES = [1, 2, 7, 8, 9, 255, 4096, 8191, 8192, 8193, 0, 16385, 100_001, 3]


@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("src", ["f32", "bf16", "mix"])
@pytest.mark.parametrize("dst", ["same", "f32", "bf16", "mix"])
def test_types_sizes_and_alignment(src, dst, pad):
    pick = {"f32": lambda i: F32, "bf16": lambda i: BF16, "mix": lambda i: (F32, BF16)[i % 2]}
    dts = [pick[src](i) for i in range(len(SIZES))]
    for max_norm in (1.0, 1e9):
        grads, flats = bucket(SIZES, dts, 3, pad)
        outs = oflats = None
        if dst != "same":
            outs, oflats = bucket(SIZES, [pick[dst](i // 2) for i in range(len(SIZES))], 4, pad)
        check(grads, max_norm, outs)
        for fl in list(flats.values()) + list((oflats or {}).values()):  # what lies between the tensors stays
            assert int(torch.isnan(fl).sum()) == (0 if pad == 0 else fl.numel() - sum(
                t.numel() for t in grads + (outs or []) if t.untyped_storage().data_ptr() == fl.untyped_storage().data_ptr()))


@pytest.mark.parametrize("n", [1, 100, 8192, 8193, 2048 * 8192, 2048 * 8192 + 5, 3 * 2048 * 8192 + 77])
def test_one_tensor(n):
    g, _ = bucket([n], [F32], n)
    check(g, 0.5)
    o, _ = bucket([n], [BF16], n + 1)
    check(g, 0.25, o)


def test_many_tensors():
    sizes = [1 + (i * 7919) % 300 for i in range(3000)]
    g, _ = bucket(sizes, [F32 if i % 3 else BF16 for i in range(3000)], 5)
    check(g, 1.0)


def test_range_of_the_norm():
    """Squares beyond fp32's range at both ends."""
    for scale in (1e30, 1e-30):
        g, _ = bucket([5000], [F32], 1, scale=scale)
        check(g, scale)


def test_no_tensors_and_zeros():
    assert grpo.grpo_clip_grad_norm_([], 1.0).item() == 0
    z = torch.zeros(100, device="cuda")
    assert grpo.grpo_clip_grad_norm_([z, z.new_empty(0)], 1.0).item() == 0 and not z.any()
    one = torch.ones(4, device="cuda")
    assert grpo.grpo_clip_grad_norm_(one, 0.0).item() == 2 and not one.any()
    one = torch.ones(4, device="cuda")
    grpo.grpo_clip_grad_norm_(one, float("inf"))
    assert torch.equal(one, torch.ones(4, device="cuda"))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    g, _ = bucket([1000, 20000], [F32, BF16], 2)
    g[1][19999] = bad
    before = [t.clone() for t in g]
    out, _ = bucket([1000, 20000], [BF16, F32], 9)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    norm = grpo.grpo_clip_grad_norm_(g, 0.1, error_flags=flags)
    assert not torch.isfinite(norm) and flags.item() == grpo.GRPO_FLAG_NONFINITE
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, before))
    grpo.grpo_clip_grad_norm_(g, 0.1, out=out)
    assert torch.equal(out[0], g[0].to(BF16)) and torch.equal(out[1].nan_to_num(0.5), g[1].float().nan_to_num(0.5))
    g[1][19999] = 0.0
    grpo.grpo_clip_grad_norm_(g, 0.1, error_flags=flags)
    assert flags.item() == 0


def test_devices_that_add_their_slots():
    """Two halves clipped by the norm of both, as after an all-reduce of the slots."""
    g, _ = bucket([50_000, 70_001], [F32, F32], 6)
    whole = [t.clone() for t in g]
    norm = grpo.grpo_clip_grad_norm_(whole, 0.7)
    parts = grpo.grpo_grad_sumsq([g[0]]) + grpo.grpo_grad_sumsq([g[1]])
    for t, w in zip(g, whole):
        n = grpo.grpo_grad_clip([t], parts, 0.7)
        assert abs(n.item() - norm.item()) <= 2.0**-23 * norm.item()
        assert ((t - w).abs() <= 2.0**-22 * w.abs()).all()


def test_same_bits_every_time():
    g, _ = bucket([3_000_001, 17], [F32, F32], 8)
    a = grpo.grpo_grad_sumsq(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = grpo.grpo_grad_sumsq(g, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_refusals():
    g = torch.ones(10, device="cuda")
    with pytest.raises(TypeError):
        grpo.GradList([g.half()])
    with pytest.raises(ValueError):
        grpo.GradList([g.cpu()])
    with pytest.raises(ValueError):
        grpo.GradList([torch.ones(4, 4, device="cuda").t()])
    with pytest.raises(ValueError):
        grpo.GradList([g], out=[g.new_empty(9)])
    with pytest.raises(ValueError):
        grpo.GradList([g], out=[])
    with pytest.raises(grpo.GrpoError):
        grpo.GradList([g, g])  # would be scaled twice
    with pytest.raises(grpo.GrpoError):
        grpo.GradList([g[:6], g[5:]])
    with pytest.raises(grpo.GrpoError):
        grpo.GradList([g[:5]], out=[g[2:7]])
    with pytest.raises(grpo.GrpoError):
        grpo.grpo_clip_grad_norm_([g], -1.0)
    with pytest.raises(grpo.GrpoError):
        grpo.grpo_clip_grad_norm_([g], float("nan"))
    with pytest.raises(TypeError):
        grpo.grpo_grad_clip([g], torch.zeros(2048, device="cuda"), 1.0)
    with pytest.raises(ValueError):
        grpo.grpo_grad_clip([g], torch.zeros(2047, device="cuda", dtype=torch.float64), 1.0)
    with pytest.raises(ValueError):
        grpo.grpo_clip_grad_norm_(grpo.GradList([g]), 1.0, out=[g])
    assert torch.equal(g, torch.ones(10, device="cuda"))


def test_memory_that_moved_is_refused():
    g = torch.ones(10, device="cuda")
    lst = grpo.GradList([g])
    assert grpo.grpo_clip_grad_norm_(lst, 100.0).item() == pytest.approx(10**0.5)
    g.data = torch.zeros(10, device="cuda")  # the list still has the old memory
    assert grpo.grpo_clip_grad_norm_(lst, 100.0).item() == pytest.approx(10**0.5)
    h = torch.ones(10, device="cuda")
    lst = grpo.GradList([h])
    h.untyped_storage().resize_(1 << 22)
    with pytest.raises(ValueError):
        grpo.grpo_clip_grad_norm_(lst, 1.0)


def test_graph_replays():
    g, _ = bucket([9000, 100_003], [F32, BF16], 3)
    out, _ = bucket([9000, 100_003], [BF16, BF16], 4)
    lst = grpo.GradList(g, out=out)
    norm = torch.empty((), device="cuda")

    def call():
        norm.copy_(grpo.grpo_clip_grad_norm_(lst, 0.5))

    call()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        call()
    for rep in range(4):
        for t in g:
            t.mul_(0.7)
        call()
        want = [o.clone() for o in out] + [norm.clone()]
        torch.cuda.synchronize()
        for o in out:
            o.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + [norm], want)), rep


def test_table_stays_until_another_stream_is_done_with_it():
    """Lists that the calls make for themselves, used on a stream that is still busy when they go."""
    n = 300
    g = [torch.full((50 + i,), 0.25, device="cuda") for i in range(n)]
    want = (sum(x.numel() for x in g) * 0.0625) ** 0.5
    table_bytes = 40 * n
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = torch.ones(4096, 4096, device="cuda")
        for _ in range(20):
            x = (x @ x).mul_(1 / 4096)
    held = []
    norm = grpo.grpo_clip_grad_norm_(g, 1e9, stream=side)
    for _ in range(20):
        held.append(torch.full((table_bytes,), 0, dtype=torch.uint8, device="cuda"))
    partials = grpo.grpo_grad_sumsq(g, stream=side)
    held.append(torch.full((table_bytes,), 0, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert abs(norm.item() - want) <= 2.0**-24 * want
    assert abs(partials.sum().item() ** 0.5 - want) <= 1e-12 * want
