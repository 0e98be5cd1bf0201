"""The workspace of the calls that reduce the tiles of few long rows in a launch of their own: one for calls one after the other,
with whatever the last call left in it, one each for calls on two streams, and calls in graphs.  Every test asks that the call
wrote to its workspace: a case that stops taking the two launches fails here."""
import numpy as np
import pytest
import torch

import paper_2606_05597_amd as grpo
from paper_2606_05597_amd import _lib
from tests.test_gpu_sampled_logp import actions
from tests.test_gpu_sampling import BF16, F32, check, make, uniform

pytestmark = pytest.mark.gpu

# what takes two launches: nothing cut, from 16,385 words on; the longest of few rows that are cut
CASES = [(1, 17001, F32, {}), (40, 20000, BF16, dict(temperature=0.7)), (191, 16385, F32, {}),
         (1, 151936, BF16, dict(top_k=50, top_p=0.95)), (64, 66001, F32, dict(temperature=0.8, top_p=0.9)),
         (9, 70001, BF16, dict(top_k=40)), (3, 70001, BF16, dict(min_p=0.02)), (2, 300_000, F32, dict(top_k=5000))]


def room(T, V):
    return int(_lib.load().grpo_sampling_workspace_bytes(T, V))


def filled(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")


def call(which, logits, u, act, par, **kw):
    if which == "draw":
        return grpo.grpo_sample(logits, u, **par, **kw)
    logp, n, rows = grpo.grpo_sampled_logp(logits, act, **par, **kw)
    return logp, n, rows


def same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.dtype == F32 else x, y.view(torch.uint8) if y.dtype == F32 else y)
               for x, y in zip(a, b))


def inputs(T, V, dtype, par, seed):
    logits, z = make("peaked", T, V, dtype, seed)
    return logits, z, uniform(z, par, seed), torch.from_numpy(actions(z, par, seed).astype(np.int32)).cuda()


def test_one_workspace_for_calls_one_after_the_other():
    """Each call finds the records of the one before it, of other rows, lengths and types, and all bits set at first."""
    ws = filled(max(room(T, V) for T, V, _, _ in CASES))
    for i, (T, V, dtype, par) in enumerate(CASES + CASES[::-1]):
        logits, z, u, act = inputs(T, V, dtype, par, i)
        before = ws.clone()
        check(logits, z, par, u, V, workspace=ws)
        assert not torch.equal(ws, before), (T, V)
        got = call("logp", logits, None, act, par, workspace=ws)
        assert same(got, call("logp", logits, None, act, par, workspace=filled(room(T, V)))), (T, V)


def test_a_workspace_of_exactly_the_size_asked_for():
    """What lies behind it stays, and less is refused."""
    for i, (T, V, dtype, par) in enumerate(CASES):
        need = room(T, V)
        buf = filled(need + 4096)
        logits, z, u, act = inputs(T, V, dtype, par, i)
        check(logits, z, par, u, V, workspace=buf[:need])
        assert (buf[need:] == 0xFF).all() and not (buf[:need] == 0xFF).all(), (T, V)
        with pytest.raises(grpo.GrpoError):
            call("logp", logits, None, act, par, workspace=buf[:need - 1])


@pytest.mark.parametrize("which", ["draw", "logp"])
def test_two_calls_at_once_on_two_streams(which):
    sets = []
    for k, (T, V, dtype, par) in enumerate([(50, 66001, F32, dict(top_p=0.9)), (64, 151936, BF16, dict(top_k=50, top_p=0.95)),
                                            (150, 60000, BF16, dict(temperature=0.8)), (33, 70001, F32, dict(top_k=30))]):
        logits, _, u, act = inputs(T, V, dtype, par, k)
        sets.append((logits, torch.from_numpy(u).cuda(), act, par, filled(room(T, V)), torch.cuda.Stream()))
    want = [call(which, x, u, a, par) for x, u, a, par, _, _ in sets]
    torch.cuda.synchronize()
    for own in (True, False):  # the caller's workspaces, or those that the calls allocate
        for _ in range(5):
            got = [call(which, x, u, a, par, stream=s, **(dict(workspace=ws) if own else {})) for x, u, a, par, ws, s in sets]
            torch.cuda.synchronize()
            assert all(same(g, w) for g, w in zip(got, want))
    assert not any((ws == 0xFF).all() for _, _, _, _, ws, _ in sets)


@pytest.mark.parametrize("T,V,dtype,par", [(9, 50000, BF16, dict(temperature=0.9)), (9, 151936, BF16, dict(top_k=50, top_p=0.95)),
                                           (20, 66001, F32, dict(temperature=0.9, top_p=0.97))], ids=str)
def test_graph_replays(T, V, dtype, par):
    logits, _, u, act = inputs(T, V, dtype, par, V)
    u = torch.from_numpy(u).cuda()
    ws, eager_ws = filled(room(T, V)), filled(room(T, V))
    outs = [t.clone() for which in ("draw", "logp") for t in call(which, logits, u, act, par)]

    def both(w):
        return [t for which in ("draw", "logp") for t in call(which, logits, u, act, par, workspace=w)]

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for o, r in zip(outs, both(ws)):
            o.copy_(r)
    for rep in range(4):
        u.copy_(torch.rand(T, device="cuda"))
        logits.mul_(0.9)
        want = [t.clone() for t in both(eager_ws)]
        torch.cuda.synchronize()
        for o in outs:
            o.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert same(outs, want), rep
        assert not (ws == 0xFF).all()


def test_two_graphs_that_were_captured_with_their_own_workspaces():
    """Replayed at once on two streams."""
    sides = []
    for k, par in enumerate((dict(top_k=50, top_p=0.95), dict(temperature=0.8))):
        T, V = 40, 100_000
        logits, _, u, _ = inputs(T, V, BF16, par, k)
        u = torch.from_numpy(u).cuda()
        want = call("draw", logits, u, None, par)
        outs = [torch.empty_like(t) for t in want]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for o, r in zip(outs, call("draw", logits, u, None, par)):
                o.copy_(r)
        sides.append((g, outs, want, torch.cuda.Stream(), logits, u))
    for _ in range(5):
        for _, outs, _, _, _, _ in sides:
            for o in outs:
                o.zero_()
        torch.cuda.synchronize()
        for g, _, _, s, _, _ in sides:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(same(outs, want) for _, outs, want, _, _, _ in sides)
